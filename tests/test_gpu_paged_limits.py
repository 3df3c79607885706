"""GPU: the paged cache where a call meets less than it needs: window pages that are gone, rooms that were refused, sums past 32 bits, weights below
a type's range."""
import math

import pytest
import torch

import paper_2412_02252_amd as pod
from pagedcase import DEV, Paged

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


def _pools(p):
    return [t.clone().view(torch.int16) for t in (p.cache.keys, p.cache.values, p.cache.window_keys)]


def _unchanged(p, before):
    return all(torch.equal(t.view(torch.int16), b) for t, b in zip((p.cache.keys, p.cache.values, p.cache.window_keys), before))


def _refused(p, counts, slots):
    """An extend that the model refuses; nobody asks the cache."""
    p.cache.pod_paged_extend(p.ints(counts), p.ints(slots))
    assert not p.model.extend(counts, slots)


def _try_step(p, slots):
    """Both layers' calls of a step, rows that must go nowhere: the outputs."""
    n, outs, qs = len(slots), [], None
    for layer in range(p.L):
        k, v, q = p.rows(n, p.Hkv), p.rows(n, p.Hkv), p.rows(n, p.Hq)
        outs.append(p.cache.pod_paged_decode(layer, k, v, q, qs, p.scale, p.ints(slots)))
        qs = q
    return outs


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("shared", [64, 70])
def test_a_step_after_a_refused_extend_overwrites_nothing(shared, many):
    """Three samples of a prompt, at a page's border or inside a page; no page is left for the next token."""
    slots = 70 if many else 4                                    # (more than 64 entries: the list that is summed up in LDS)
    p = Paged(2, 2, 4, 2, 64, 5, 30, slots, 2000, 16, 9 + slots, 9 + slots, seed=shared)
    p.extend([shared], [1])
    p.prompt([1], [shared])
    p.fork([1, 1], [0, 3])
    if shared % 16:
        fill = 16 - shared % 16
        p.extend([fill] * 3, [1, 0, 3])
        p.prompt([1, 0, 3], [fill] * 3)
    free = min(p.model.refs[k].count(0) for k in "cw")
    assert p.extend([16 * (free - 1)], [2])
    p.prompt([2], [16 * (free - 1)])
    live = [3, 0, 1] + list(range(4, slots))
    before = _pools(p)
    for _ in range(2):
        _refused(p, [1] * len(live), live)
        assert not any(t.any() for t in _try_step(p, live))
        p.cache.pod_paged_plan(p.ints([0, 1]), 1, p.ints([3]))
    assert _unchanged(p, before)
    p.expect(False)
    p.assert_books()
    p.free([2])
    _refused(p, [3000], [0])                                     # one that was refused and then got room, unasked in between
    some = [3, 0, 1] if many else [3, 0, 1, 2]
    p.cache.pod_paged_extend(p.ints([1] * len(some)), p.ints(some))
    assert p.model.extend([1] * len(some), some)
    queries = []
    for layer in range(2):
        k, v, q = p.rows(len(some), 2), p.rows(len(some), 2), p.rows(len(some), 4)
        queries.append(q)
        p._note(layer, some, [1] * len(some), k, v)
        out = p.cache.pod_paged_decode(layer, k, v, q, queries[0] if layer else None, p.scale, p.ints(some))
        for e, s in enumerate(some):
            p.check(layer, s, 1, q[e:e + 1], queries[0][e:e + 1] if layer else None, out[e:e + 1])
    p.expect(False)
    p.extend([1], [0])
    p.step([0])
    p.assert_books()


def test_a_plan_after_a_refused_extend_has_the_later_rooms_only():
    p = Paged(2, 2, 4, 2, 64, 5, 30, 3, 400, 16, 20, 20, seed=8)
    p.extend([100, 40], [0, 1])
    p.prompt([0, 1], [100, 40])
    before = _pools(p)
    _refused(p, [60, 200], [0, 1])
    for rows in (1, 20, 40):
        plan = p.cache.pod_paged_plan(p.ints([0, rows]), rows, p.ints([1]))
        p.cache.pod_paged_store(0, p.rows(rows, 2), p.rows(rows, 2), plan)
    assert _unchanged(p, before)
    p.cache.pod_paged_extend(p.ints([7, 9]), p.ints([1, 0]))     # accepted, but nobody has asked about the refusal yet
    assert p.model.extend([7, 9], [1, 0])
    before = _pools(p)
    plan = p.cache.pod_paged_plan(p.ints([0, 8, 17]), 17, p.ints([1, 0]))
    p.cache.pod_paged_store(0, p.rows(17, 2), p.rows(17, 2), plan)
    assert _unchanged(p, before)
    p.expect(False)
    _refused(p, [400, 1], [0, 1])
    p.expect(False)                                              # asked: from here on every row may be written again, as long as it is there
    p.prompt([1, 0], [7, 9])
    p.extend([3, 2], [0, 1])
    p.prompt([0, 1], [3, 2], stored_first=True)
    p.assert_books()


def test_a_refused_extend_holds_back_its_own_entries_only():
    p = Paged(2, 2, 4, 2, 64, 5, 30, 5, 400, 16, 20, 20, seed=9)
    p.extend([30, 31, 32], [0, 1, 2])
    p.prompt([0, 1, 2], [30, 31, 32])
    for counts, slots in (([400, 0, 1], [1, 0, 2]), ([1, 1], [1, 9]), ([-1], [1]), ([1, 1], [1, 1])):
        p.cache.pod_paged_extend(p.ints([1]), p.ints([0]))
        assert p.model.extend([1], [0])
        before = _pools(p)
        _refused(p, counts, slots)
        assert not any(t.any() for t in _try_step(p, [1]))
        assert _unchanged(p, before)
        queries = []
        for layer in range(2):                                   # slot 0 has its token
            k, v, q = p.rows(1, 2), p.rows(1, 2), p.rows(1, 4)
            queries.append(q)
            p._note(layer, [0], [1], k, v)
            out = p.cache.pod_paged_decode(layer, k, v, q, queries[0] if layer else None, p.scale, p.ints([0]))
            p.check(layer, 0, 1, q, queries[0] if layer else None, out)
        p.expect(False)
    _refused(p, [400], [1])
    p.cache.pod_paged_fork(p.ints([1]), p.ints([3]))             # a sample of a slot without room has none either
    p.model.fork([1], [3])
    before = _pools(p)
    assert not any(t.any() for t in _try_step(p, [3, 1]))
    assert _unchanged(p, before)
    p.cache.pod_paged_free(p.ints([1, 3]))                       # a freed slot begins anew
    p.model.free([1, 3])
    p.k[1], p.v[1] = [[], []], [[], []]
    p.cache.pod_paged_extend(p.ints([20]), p.ints([1]))
    assert p.model.extend([20], [1])
    p.expect(False)
    p.prompt([1], [20])
    p.assert_books()


def test_replays_of_a_step_that_finds_no_page():
    """One graph: room for a token, both layers.  Replays without a free page change nothing; once there are pages it goes on, unasked."""
    p = Paged(2, 2, 4, 2, 64, 5, 30, 3, 400, 16, 14, 14, seed=10)
    p.extend([31, 60, 80], [0, 1, 2])
    p.prompt([0, 1, 2], [31, 60, 80])
    slots, one = p.ints([0, 1]), p.ints([1, 1])
    k, v, q = ([p.rows(2, h) for _ in range(2)] for h in (2, 2, 4))
    outs = [torch.empty_like(t) for t in q]

    def step():
        p.cache.pod_paged_extend(one, slots)
        for layer in range(2):
            p.cache.pod_paged_decode(layer, k[layer], v[layer], q[layer], q[0] if layer else None, p.scale, slots, out=outs[layer])

    def replayed(run):
        for t in k + v + q:
            t.copy_(torch.randn(t.shape, generator=p.gen).to(p.dtype))
        before = _pools(p)
        run()
        ok = p.model.extend([1, 1], [0, 1])
        for layer in range(2):
            if ok:
                p._note(layer, [0, 1], [1, 1], k[layer], v[layer])
                for s in range(2):
                    p.check(layer, s, 1, q[layer][s:s + 1], q[0][s:s + 1] if layer else None, outs[layer][s:s + 1])
            else:
                assert not outs[layer].any()
        assert ok or _unchanged(p, before)
        return ok

    assert replayed(step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    answers = [replayed(graph.replay) for _ in range(60)]
    assert answers[0] and not any(answers[-3:])
    p.cache.pod_paged_free(p.ints([2]))
    p.model.free([2])
    assert all(replayed(graph.replay) for _ in range(20))
    p.expect(False)
    p.assert_books()


@pytest.mark.parametrize("entries,last", [(128, 1 << 28), (129, 16), (257, 16)])
def test_more_pages_than_32_bits_count_are_too_few(entries, last):
    """2^24 pages for each entry but the last: 2^31 in all, 2^31 and one, 2^32 and one; tables of 8 GB and more."""
    free, total = torch.cuda.mem_get_info()
    tokens = 1 << 28
    if free < entries * tokens // 16 * 4 * 2 + (4 << 30):
        pytest.skip("the tables do not fit")
    cache = pod.PagedCache(pod.make_paged_config(1, 1, 1, 1, 64, 0, 16, entries, tokens, 16, 20, 0), DEV)
    counts = torch.full((entries,), tokens, dtype=torch.int32, device=DEV)
    counts[-1] = last
    before = cache.lens.clone(), cache.page_refs.clone()
    cache.pod_paged_extend(counts)
    with pytest.raises(pod.PodError) as e:
        cache.pod_paged_check()
    assert e.value.code == pod.binding.ERR_STATE and "too few free pages" in str(e.value)
    assert torch.equal(cache.lens, before[0]) and torch.equal(cache.page_refs, before[1])
    counts[:] = 0
    counts[[0, entries - 1]] = torch.tensor([100, 200], dtype=torch.int32, device=DEV)   # 7 + 13 pages: all there are
    cache.pod_paged_extend(counts)
    cache.pod_paged_check()
    assert cache.lens[[0, entries - 1]].tolist() == [100, 200] and bool((cache.page_refs == 1).all())
    assert cache.page_table[0, :8].tolist() == [*range(7), -1] and cache.page_table[entries - 1, :14].tolist() == [*range(7, 20), -1]


@pytest.mark.parametrize("bits", [20.0, 26.0, 30.0])
@pytest.mark.parametrize("where", ["first", "own"])
def test_many_small_weights_beside_a_large_one(where, bits):
    """fp16: 120000 keys whose weights are about 2^-bits of one key's, which has the value 0: the result is theirs alone.

    An element differs by its rounding, eps / 2 |o| or half a step of 2^-24; by that of the weights, once in the product and once in the sum that divides,
    2 eps / 2 sum_j w_j |v_j|; by weights whose packed form is below the type's normal range: off by half of 2^-24 of the largest weight's share of its
    packed form, which is at least 2^7: sum_j |v_j| 2^-32 / l; and by 32-bit sums, 2^-24 a step over n / 16 steps of products and of the sum, and of logits of
    2^5 over 64 products: 2 (n / 16 + 2^11) 2^-24 sum_j w_j |v_j|."""
    n, hq, d = 120000, 2, 64
    p = Paged(1, 1, hq, 1, d, 4, 64, 1, n + 10, 256, 500, 0, torch.float16)
    k, v = 0.2 * torch.randn((n + 3, 1, d), generator=p.gen), 1 + torch.randn((n + 3, 1, d), generator=p.gen)
    big = [0] if where == "first" else list(range(n, n + 3))
    k[:, :, 0] = 0
    k[big] = 0
    k[big, :, 0] = bits * math.log(2)                            # q k scale = bits ln 2
    v[big] = 0
    q = 0.5 * torch.randn((3, hq, d), generator=p.gen)
    q[:, :, 0] = 1 / p.scale
    k, v, q = (t.half() for t in (k, v, q))
    half = torch.finfo(torch.float16).eps / 2

    def close(out, rows, last):                                  # tokens .. last
        i, out = torch.arange(last + 1 - rows, last + 1)[:, None], out.cpu().double()
        for h in range(hq):
            a = q[last + 1 - rows - n:last + 1 - n, h].double() @ k[:last + 1, 0].double().T * p.scale
            a = torch.where(torch.arange(last + 1)[None] <= i, a, -math.inf)
            w = torch.exp(a - a.amax(-1, keepdim=True))
            l, vd = w.sum(-1, keepdim=True), v[:last + 1, 0].double()
            want, size = w @ vd / l, w @ vd.abs() / l
            tol = half * (want.abs() + 2 * size) + 2.0 ** -25 + vd.abs().sum(0) * 2.0 ** -32 / l + 2 * (last / 16 + 2 ** 11) * 2.0 ** -24 * size
            err = (out[:, h] - want).abs()
            assert bool((err <= tol).all()), (rows, h, float((err / tol).max()), float(want.abs().mean()), float(out[:, h].abs().mean()))

    dev = [t.to(DEV) for t in (k, v, q)]
    c = p.cache
    c.pod_paged_extend(p.ints([n]))
    c.pod_paged_store(0, dev[0][:n], dev[1][:n], c.pod_paged_plan(p.ints([0, n]), n))
    c.pod_paged_extend(p.ints([2]))
    plan = c.pod_paged_plan(p.ints([0, 2]), 2)
    close(c.pod_paged_prefill(0, dev[0][n:n + 2], dev[1][n:n + 2], dev[2][:2], None, plan, p.scale), 2, n + 1)
    c.pod_paged_extend(p.ints([1]))
    close(c.pod_paged_decode(0, dev[0][n + 2:], dev[1][n + 2:], dev[2][2:], None, p.scale), 1, n + 2)
    c.pod_paged_check()


def test_sums_stop_above_a_pool_of_millions_of_pages():
    """1024 entries of 2^21 pages each, as many as the pool has in all: 2^31."""
    free, total = torch.cuda.mem_get_info()
    if free < 50 << 30:
        pytest.skip("the tables and pools do not fit")
    tokens, pages = 1 << 25, 1 << 21
    cache = pod.PagedCache(pod.make_paged_config(1, 1, 1, 1, 64, 0, 16, 1024, tokens, 16, pages, 0), DEV)
    counts = torch.full((1024,), tokens, dtype=torch.int32, device=DEV)
    cache.pod_paged_extend(counts)
    with pytest.raises(pod.PodError) as e:
        cache.pod_paged_check()
    assert e.value.code == pod.binding.ERR_STATE and "too few free pages" in str(e.value)
    assert not cache.lens.any() and not cache.page_refs.any()
    counts[1:] = 0
    cache.pod_paged_extend(counts)                               # all of them for one
    cache.pod_paged_check()
    assert int(cache.lens[0]) == tokens and bool((cache.page_refs == 1).all())
    assert torch.equal(cache.page_table[0], torch.arange(pages, dtype=torch.int32, device=DEV)) and bool((cache.page_table[1:3] == -1).all())


@pytest.mark.parametrize("n", [1, 5])
def test_rows_of_one_head_may_have_any_head_stride(n):
    """A token's only head is contiguous whatever the stride between heads that are not there."""
    p = Paged(1, 1, 1, 1, 64, 4, 50, n, 100, 16, 2 * n, 0)
    p.extend([1] * n, list(range(n)))
    k, v, q = (p.rows(n, 1) for _ in range(3))
    p._note(0, list(range(n)), [1] * n, k, v)
    turned = [t.as_strided((n, 1, 64), (64, 64 * n + 8, 1)) for t in (k, v, q)]
    out = p.cache.pod_paged_decode(0, *turned, None, p.scale)
    for e in range(n):
        p.check(0, e, 1, q[e:e + 1], None, out[e:e + 1])
    plan = p.cache.pod_paged_plan(p.ints(list(range(n + 1))), n)
    p.cache.pod_paged_store(0, turned[0], turned[1], plan)
    assert torch.equal(p.cache.pod_paged_prefill(0, None, None, turned[2], None, plan, p.scale), out)
    p.expect(True)
