"""GPU tests of the weights of attention over 8-bit pages: what few rows round them by, and their sum beside scales of V
that lie far apart.  Against 64 bits (pages8_ref.py)."""

import math

import pytest
import torch

import batch_ref as R
import pages8_ref as R8
import test_gpu_pages8 as T
from paper_2608_00814_gb300 import binding as B
from test_gpu_batch_ops import BF16, F16, gen, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _built():
    from paper_2608_00814_gb300 import _build
    _build.build()


@pytest.mark.parametrize("dtype, kv", [(BF16, BF16), (BF16, F16), (F16, F16)])
@pytest.mark.parametrize("counts, lens, nq, width", [
    ([1, 1, 1, 1], [700, 90, 333, 16], 8, None),        # tiles of 8 rows, a block each
    ([1, 1, 1, 1], [700, 90, 333, 16], 8, 70),          # equal shares
    ([5, 2, 9, 1], [400, 90, 333, 200], 8, None),
    ([5, 2, 9, 1], [400, 90, 333, 200], 8, 70),
    ([100, 90], [300, 420], 2, 70),                     # 95 rows on average, few tiles: the same kernels
    ([200], [450], 2, None),                            # and over a short table
])
def test_few_rows_round_own_weights_to_11_bits(dtype, kv, counts, lens, nq, width):
    """Without a prefix every weight is binary16's, of bf16 queries too: half a step of 2^-11, where bf16 has 2^-8; and of q
    2^-25 of a row's largest is left out."""
    d = 128
    step = R.Step(counts, lens, 16, seed=1, width=width)
    q, _, _, cache = T.inputs8(step, 0, nq, 2, d, dtype, kv, seed=2)
    out, st = T.attend8(step, q, None, None, 0, cache)
    assert int(st) == 0
    none = torch.zeros(0, 2, d, dtype=F16, device="cuda")
    out64, mag, size, (left, _, term, v) = R8.attention(step, q, none, none, cache, 1 / math.sqrt(d))
    left = min(left, left * 2.0 ** -8) if step.n * (nq // 2) > 64 * len(counts) else left
    R8.check_attention(out, out64, mag, size, (left, R.U[F16], term, v), max(lens))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("high", [30, 110, 119])
@pytest.mark.parametrize("low", [-20, -60, -117])
@pytest.mark.parametrize("counts, lens, width", [([1, 2], [70, 300], None), ([1, 2], [70, 300], 80), ([90, 140], [400, 330], 80)])
def test_weights_count_whatever_scale_their_v_has(dtype, high, low, counts, lens, width):
    """Blocks of zeros under a large scale, and between them blocks whose scores are 2^10 of the others' and whose v is all
    but zero: they weigh as much as their scores say, which the prefix's v shows.  Their own v is below 2^-11 of what is
    added up, or lost beside the large scale: 2^-32 of that at most, as far as zeros count."""
    d, nkv, nq, prefix = 128, 2, 4, 40
    step = R.Step(counts, lens, 16, seed=3, width=width)
    g = gen(4)
    q = (1 + randn(g, step.rows, nq, d, std=0.05)).to(dtype)
    pk, pv = torch.zeros(prefix, nkv, d, dtype=dtype, device="cuda"), randn(g, prefix, nkv, d, dtype=dtype)
    k, v, ks, vs = T.pool(g, step.n_pages, 16, nkv, d)
    ks.fill_(127)
    odd = torch.arange(step.n_pages, device="cuda") % 2 == 1
    k.copy_(torch.where(odd[:, None, None, None], 1.0, 0.0).expand(k.shape).to(k.dtype))
    v.copy_(torch.where(odd[:, None, None, None], v.float(), 0.0).to(v.dtype))
    vs.copy_((127 + torch.where(odd, low, high)).to(torch.uint8)[:, None, None].expand(vs.shape))
    cache = B.PagedCache8(k, v, ks, vs)
    scale = 10 * math.log(2) / d
    out, st = T.attend8(step, q, pk, pv, prefix, cache, scale=scale)
    assert int(st) == 0
    ref, mag, size, (left, weights, _, _) = R8.attention(step, q, pk, pv, cache, scale)
    own = 448 * 2.0 ** low      # of v: at most all of it is lost
    R8.check_attention(out, ref, mag, size, (left, weights, own / (prefix + max(lens)), 0.0), prefix + max(lens))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("counts, lens, width", [([1, 2], [70, 300], None), ([1, 2], [70, 300], 80), ([90, 140], [400, 330], 80)])
def test_factors_past_fp32(dtype, counts, lens, width):
    """A key whose score is far below fp32's range beside keys of zeros, under the largest scale and with large queries, so
    that what a product of codes is multiplied by is past fp32: the zeros' scores are 0 and weigh the same (1, exactly), the
    other key nothing.  So out is v's mean: half a step of it, and of fp32 for each key of either sum."""
    d, nkv, nq = 128, 2, 4
    step = R.Step(counts, lens, 16, seed=3, width=width)
    g = gen(5)
    q = (256 * (1 + randn(g, step.rows, nq, d).abs().clamp(max=2))).to(dtype)
    k, v, ks, vs = T.pool(g, step.n_pages, 16, nkv, d, lo=-8, hi=-4)
    k.zero_()
    ks.fill_(127 + 119)
    for b in range(len(counts)):
        for s in (3, lens[b] - counts[b] - 20):
            page, at = step.where(b, s)
            k[page, at] = -448.0
    cache = B.PagedCache8(k, v, ks, vs)
    scale = 512.0
    out, st = T.attend8(step, q, None, None, 0, cache, scale=scale)
    assert int(st) == 0
    none = torch.zeros(0, nkv, d, dtype=dtype, device="cuda")
    ref, mag, _, _ = R8.attention(step, q, none, none, cache, scale)
    out = out[:step.n].double().cpu()
    assert bool(torch.isfinite(out).all())
    tol = R.U[dtype] * ref.abs() + (4 * max(lens) + 64) * R.F32 * mag + (2.0 ** -25 if dtype is F16 else 0)
    assert bool(((out - ref).abs() <= tol).all()), float(((out - ref).abs() - tol).max())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("nan", [False, True])
@pytest.mark.parametrize("counts, lens, nq, start", [
    ([90, 128], [700, 300], 8, 256),       # two row tiles a block; from the third tile of keys on
    ([128, 100], [128, 900], 2, 0),        # one, whose tiles of keys two streams take in turn
    ([128, 120], [1000, 640], 2, 384),
    ([110, 127], [5000, 4900], 2, 2300),   # several ranges of keys a sequence
    ([128], [2600], 10, 2048),
])
def test_scales_far_from_those_before(dtype, tree, nan, counts, lens, nq, start):
    """From some position on a third of V's blocks stand under scales of next to nothing and of the least there is, behind
    tiles of ordinary ones; also with trees, and with a NaN among the step's own v, which reaches the rows that see it."""
    d, nkv, prefix = 128, 2, 70
    step = R.Step(counts, lens, 16, seed=6, width=330)
    parent = [-1 if j == 0 else max(0, j - 1 - j % 3) for c in counts for j in range(c)] if tree else None
    par = torch.tensor(parent, dtype=torch.int32, device="cuda") if tree else None
    q, pk, pv, cache = T.inputs8(step, prefix, nq, nkv, d, dtype, dtype, seed=7, std=0.5)
    for b, n in enumerate(lens):
        for s in range(start // 16 * 16, n, 16):
            if (s // 16) % 3:
                page, at = step.where(b, s)
                cache.v_scale[page, at // 16] = 127 - (117 if (s // 16) % 3 == 1 else 55)
    ref = R8.attention(step, q, pk[:prefix], pv[:prefix], cache, 1 / math.sqrt(d), parent)
    want = torch.zeros(step.n, nq, dtype=torch.bool)
    if nan:
        b, node = len(counts) - 1, 40
        page, at = step.where(b, lens[b] - counts[b] + node)
        cache.v.view(torch.uint8)[page, at, 1, 9] = R8.NAN_CODE
        first = step.q_start[b]
        seen = R.ancestors(parent[first:first + counts[b]])[:, node] if tree else torch.arange(counts[b]) >= node
        want[first:first + counts[b], nq // 2:] = seen[:, None]
    out, st = T.attend8(step, q, pk, pv, prefix, cache, par)
    assert int(st) == 0
    out = out[:step.n]
    assert torch.equal(torch.isnan(out[..., 9]).cpu(), want) and int(torch.isnan(out).sum()) == int(want.sum())
    out = torch.where(torch.isnan(out), ref[0].to(dtype).cuda(), out)
    R8.check_attention(out, *ref, prefix + max(lens))
