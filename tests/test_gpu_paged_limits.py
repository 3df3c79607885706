"""GPU: the paged cache where a call meets less than it needs: window pages that are gone, rooms that were refused, sums past 32 bits, weights below
a type's range."""
import pytest
import torch

from pagedcase import Paged

pytestmark = pytest.mark.gpu


def _missing(model, slot, rows):
    """Window pages that the last `rows` tokens of the slot attend by their own layers' keys and that are gone (the header's rule, key by key)."""
    n = model.lens[slot]
    i, j = torch.arange(n - rows, n)[:, None], torch.arange(n)[None]
    near = ((j <= i) & ((j < model.S) | (j > i - model.W))).any(0).nonzero().flatten() // model.ps
    return [page for page in sorted(set(near.tolist())) if model.table["w"][slot][page] < 0]


@pytest.mark.parametrize("S,W,ps", [(16, 64, 16), (0, 16, 16), (5, 33, 32), (40, 1, 16), (70, 65, 64), (3, 400, 16)])
def test_plans_over_several_extends(S, W, ps):
    """Accepted exactly where every window page that the rows attend is there, whatever the extends the rows came by."""
    p = Paged(2, 2, 2, 1, 64, S, W, 2, 900, ps, 120, 120, seed=W)
    answers = set()
    for held, parts in ((32, (16, 16)), (100, (1, 1, 1)), (200, (100, 100)), (300, (1, 30)), (150, (ps, ps, 1)), (0, (200, 200)), (63, (1, 64))):
        p.free([0, 1])
        p.extend([held, 7], [0, 1])
        for more in parts:
            p.extend([more], [0])
        n = held + sum(parts)
        for rows in {1, parts[-1], parts[-1] + 1, n - held, min(n - held + 1, n), n}:
            p.cache.pod_paged_plan(p.ints([0, 7, 7 + rows]), 7 + rows, p.ints([1, 0]))
            ok = not _missing(p.model, 0, rows)
            p.expect(ok)
            answers.add(ok)
    p.assert_books()
    assert True in answers and (False in answers or W == 400)


def test_rows_of_several_extends_attend_what_they_should_or_are_refused():
    p = Paged(4, 2, 4, 2, 64, 16, 64, 2, 900, 16, 120, 120, seed=2)
    p.extend([500, 90], [0, 1])
    p.prompt([0, 1], [500, 90])
    for more in (10, 10):
        p.extend([more], [0])
    p.prompt([0], [20])                                          # both extends' rows in one batch: their window is still there
    for more in (100, 100):
        p.extend([more], [0])
    before = [t.clone() for t in (p.cache.keys, p.cache.values, p.cache.window_keys)]
    plan = p.cache.pod_paged_plan(p.ints([0, 200]), 200, p.ints([0]))
    p.expect(False)
    q, k = p.rows(200, 4), p.rows(200, 2)
    out = torch.full_like(q, 7.0)
    p.cache.pod_paged_prefill(1, k, k, q, q, plan, p.scale, out=out)
    p.expect(False)
    assert bool((out == 7).all())
    for t, b in zip((p.cache.keys, p.cache.values, p.cache.window_keys), before):
        assert torch.equal(t.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,held,lost", [(64, 640, True), (64, 641, False), (128, 640, True), (128, 6400, True), (64, 6399, False), (64, 79, False), (64, 80, False), (64, 96, True)])
def test_a_refused_extend_never_gives_a_held_token_another_answer(d, held, lost, dtype):
    """W = 65 and pages of 16: the extend's first token no longer needs the page of tokens .. held - 65, the last held one does where that is the page's
    last.  The answer stays, or the call refuses it; layers whose keys are in context pages go on."""
    p = Paged(2, 2, 4, 2, d, 16, 65, 2, 8000, 16, 450, 450, dtype, seed=held)
    p.extend([held - 1, 50], [0, 1])
    p.prompt([0, 1], [held - 1, 50])
    p.extend([1], [0])
    k, v, q = ([p.rows(1, h) for _ in range(2)] for h in (2, 2, 4))
    for layer in range(2):
        p._note(layer, [0], [1], k[layer], v[layer])
        out = p.cache.pod_paged_decode(layer, k[layer], v[layer], q[layer], q[0] if layer else None, p.scale, p.ints([0]))
        p.check(layer, 0, 1, q[layer], q[0] if layer else None, out)
    want = out
    assert not p.extend([8000 - held], [0])
    p.assert_books()
    assert bool(_missing(p.model, 0, 1)) == lost
    both = [torch.cat([t, p.rows(1, 4)]) for t in q]
    out = p.cache.pod_paged_decode(0, None, None, both[0], None, p.scale, p.ints([0, 1]))
    p.expect(True)
    p.check(0, 0, 1, q[0], None, out[:1])
    out = p.cache.pod_paged_decode(1, None, None, both[1], both[0], p.scale, p.ints([0, 1]))
    p.expect(not lost)
    p.check(1, 1, 1, both[1][1:], both[0][1:], out[1:])
    if lost:
        assert not out[0].any()
    else:
        p.check(1, 0, 1, q[1], q[0], out[:1])
        alone = p.cache.pod_paged_decode(1, None, None, q[1], q[0], p.scale, p.ints([0]))
        assert torch.equal(alone, want)
    p.cache.pod_paged_plan(p.ints([0, 1]), 1, p.ints([0]))
    p.expect(not lost)
