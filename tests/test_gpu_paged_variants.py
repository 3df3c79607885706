"""GPU: every kernel that a paged call may choose, at sizes that choose it: one key group per prompt tile, even runs of single-token calls, long prompts."""
import math
import random

import pytest
import torch

from pagedcase import DEV, Paged

pytestmark = pytest.mark.gpu

HEADWISE = [[0] * 8, [0, 1, 0, 1, 1, 0, 1, 1], [0, 1, 2, 1, 1, 2, 2, 2]]


def _cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _one_group(Hq, Hkv, counts):
    """The prompt launch has more workgroups than the device compute units: one key group per tile."""
    tiles = sum(counts) // (128 // (Hq // Hkv)) + min(len(counts), sum(counts))
    return tiles * Hkv > _cus()


def _even_runs(Hkv, lens, S, W, upper_heads):
    """The single-token launch of these lengths takes even runs (the rule of its kernel on two workgroups per compute unit)."""
    def tiles(n, upper):
        if n == 0 or not upper:
            return -(-n // 32)
        last = n - 1
        first = S // 32
        distant = (last - W) // 32 - first + 1 if last - W >= S else 0
        sink = (min(S, n) - 1) // 32 + 1 if S else 0
        begin = max(sink, (last - W + 1) // 32 if last - W + 1 > 0 else 0)
        return distant + sink + max(last // 32 - begin + 1, 0)
    if len(lens) > 64:
        return True
    wgs = min(2 * _cus(), 512)
    total = sum(upper_heads * tiles(n, True) + (Hkv - upper_heads) * tiles(n, False) for n in lens)
    room = wgs - len(lens) * Hkv
    return room <= 0 or -(-total // room) * wgs > total + 8 * wgs


def _fill(p, slots, counts):
    """New tokens whose rows are stored and attended by nobody yet."""
    p.extend(counts, slots)
    cu = [0]
    for c in counts:
        cu.append(cu[-1] + c)
    plan = p.cache.pod_paged_plan(p.ints(cu), cu[-1], p.ints(slots))
    for layer in range(p.L):
        k, v = p.rows(cu[-1], p.Hkv), p.rows(cu[-1], p.Hkv)
        p._note(layer, slots, counts, k, v)
        p.cache.pod_paged_store(layer, k, v, plan)
    p.cache.pod_paged_check()


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
def test_prompts_of_more_workgroups_than_compute_units(d, dtype, far):
    """Lowest and upper layers, prompts and a chunk behind them; far: logits up to some 200 apart, whose reference moves many times."""
    p = Paged(2, 2, 64, 8, d, 5, 70, 3, 900, 16, 160, 160, dtype, seed=d + far)
    if far:
        p.scale = 4.0
        # 4 sum |q k| < 2^(log2 d + 2); over d products, scaled and shifted, off by 2^-24 (d + 2) of that, above and below the division
        p.logit_slack = 2 * 2.0 ** -24 * (d + 2) * 4 * d
    counts = [400, 1, 250]
    assert _one_group(64, 8, counts) and _one_group(64, 8, [300, 260])
    p.extend(counts, [2, 0, 1])
    p.prompt([2, 0, 1], counts, gap=8)
    p.extend([300, 260], [1, 0])
    p.prompt([1, 0], [300, 260])


def test_head_wise_prompts_of_more_workgroups_than_compute_units():
    p = Paged(3, 1, 64, 8, 64, 6, 40, 2, 700, 16, 100, 100, block_lowest=HEADWISE)
    assert _one_group(64, 8, [420, 130])
    p.extend([420, 130], [0, 1])
    p.prompt([0, 1], [420, 130])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,n,Hkv,G,longest", [(64, 64, 8, 2, 300), (128, 64, 8, 2, 200), (64, 64, 8, 1, 150), (128, 50, 8, 2, 4000), (64, 100, 3, 2, 400), (128, 66, 5, 2, 150)])
def test_steps_with_even_runs(d, n, Hkv, G, longest, dtype):
    """Runs that end and begin anywhere in a pair's list: distant, sink and window tiles; few entries and many; one sequence far longer than the others."""
    r = random.Random(d + n)
    lens = [r.choice([0, 1, 31, 32, 70, 76, r.randint(1, min(longest, 300))]) for _ in range(n)]
    lens[r.randrange(n)] = longest
    pages = sum(-(-(x + 1) // 16) for x in lens)
    p = Paged(2, G, 2 * Hkv, Hkv, d, 5, 70, n, longest + 10, 16, pages, pages if G > 1 else 0, dtype, seed=n)
    slots = r.sample(range(n), n)
    _fill(p, slots, lens)
    assert _even_runs(Hkv, [x + 1 for x in lens], 5, 70, Hkv if G > 1 else 0)
    p.extend([1] * n, slots)
    p.step(slots)


@pytest.mark.parametrize("n", [64, 75])
def test_head_wise_steps_with_even_runs(n):
    r = random.Random(n)
    lens = [r.choice([0, 1, 40, 47, 60, r.randint(1, 250)]) for _ in range(n)]
    pages = sum(-(-(x + 1) // 16) for x in lens)
    p = Paged(3, 1, 16, 8, 64, 6, 40, n, 300, 16, pages, pages, block_lowest=HEADWISE, seed=n)
    _fill(p, list(range(n)), lens)
    assert all(_even_runs(8, [x + 1 for x in lens], 6, 40, sum(HEADWISE[layer][h] != layer for h in range(8))) for layer in range(3))
    p.extend([1] * n, list(range(n)))
    p.step(list(range(n)))


def _check_sampled(p, layer, held, q, qs, out, rows, at):
    """Rows `at` of the last `rows` tokens of a sequence; held: its keys and values per layer on the device.  As Paged.check, but for the sums: 2^-24 a step over
    n / 16 steps of products and of the sum that divides, and 2^-13 for logits of size up to 2^4 over 128 products and their exponentials.  fp16: weights below the
    type's normal range are off by half of 2^-24 of a packed largest one of at least 2^7."""
    rep, half = p.Hq // p.Hkv, torch.finfo(p.dtype).eps / 2
    k, v = held[layer]
    low, n = held[layer - layer % 2][0], len(held[layer][0])
    i, j = (n - rows + torch.tensor(at, device=DEV))[:, None], torch.arange(n, device=DEV)[None]
    near = (j < p.S) | (j > i - p.W)
    for g in range(p.Hq):
        h = g // rep
        a = q[at, g].double() @ k[:, h].double().T.contiguous()
        if layer % 2:
            a = torch.where(near, a, qs[at, g].double() @ low[:, h].double().T.contiguous())
        a = torch.where(j <= i, a * p.scale, -math.inf)
        w = torch.exp(a - a.amax(-1, keepdim=True))
        l, vd = w.sum(-1, keepdim=True), v[:, h].double()
        want, size = w @ vd / l, w @ vd.abs() / l
        tol = half * (want.abs() + 2 * size) + (2.0 ** -13 + 2 * (n / 16 + 2 ** 7) * 2.0 ** -24) * size
        if p.dtype == torch.float16:
            tol = tol + 2.0 ** -32 * vd.abs().sum(0) / l
        err = (out[at, g].double() - want).abs()
        assert bool((err <= tol).all()), (layer, g, n, rows, float((err / tol).max()), at[int((err / tol).amax(-1).argmax())])


@pytest.mark.parametrize("d,ps,dtype,counts", [(128, 64, torch.bfloat16, [16384, 1]), (64, 16, torch.float16, [9000, 7001, 1, 1]), (128, 256, torch.float16, [5000, 28000, 1])])
def test_long_prompts_chunks_and_steps(d, ps, dtype, counts):
    """One sequence in chunks of `counts` tokens (1: a single-token step as well), rows sampled at tiles' and windows' borders and elsewhere."""
    Hq, Hkv, S, W = 8, 2, 64, 2048
    n = sum(counts)
    p = Paged(2, 2, Hq, Hkv, d, S, W, 1, n, ps, -(-n // ps), -(-n // ps), dtype)
    gen = torch.Generator(device=DEV).manual_seed(d)
    r = random.Random(n)
    held = [[torch.empty((0, Hkv, d), dtype=dtype, device=DEV) for _ in range(2)] for _ in range(2)]
    for rows in counts:
        p.extend([rows], [0])
        plan = p.cache.pod_paged_plan(p.ints([0, rows]), rows)
        at = sorted({x for x in (0, 1, 31, 32, 63, 64, W - 1, W, W + S, rows // 2, rows - 2, rows - 1) if 0 <= x < rows} | {r.randrange(rows) for _ in range(24)})
        qs = None
        for layer in range(2):
            k, v, q = (torch.randn((rows, x, d), generator=gen, device=DEV).to(dtype) for x in (Hkv, Hkv, Hq))
            held[layer] = [torch.cat([a, b]) for a, b in zip(held[layer], (k, v))]
            _check_sampled(p, layer, held, q, qs, p.cache.pod_paged_prefill(layer, k, v, q, qs, plan, p.scale), rows, at)
            if rows == 1:
                _check_sampled(p, layer, held, q, qs, p.cache.pod_paged_decode(layer, k, v, q, qs, p.scale), rows, at)
            qs = q
    p.expect(True)
    p.assert_books()
