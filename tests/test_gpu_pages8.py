"""GPU tests of the operators on 8-bit pages, and on pages between steps, against their 64-bit restatement
(pages8_ref.py)."""

import math

import numpy as np
import pytest
import torch

import batch_ref as R
import pages8_ref as R8
from paper_2608_00814_gb300 import binding as B
from test_gpu_batch_ops import BF16, F16, F32, LLAMA, TYPES, gen, randn, status

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
U8 = torch.uint8


@pytest.fixture(autouse=True)
def _built():
    from paper_2608_00814_gb300 import _build
    _build.build()


def codes(g, *shape):
    return (randn(g, *shape) * 90).clamp(-448, 448).to(E4M3)


def scales(g, *shape, lo=-8, hi=3):
    return torch.randint(127 + lo, 128 + hi, shape, generator=g, device="cuda", dtype=torch.int32).to(U8)


def pool(g, n_pages, page, nkv, d, lo=-8, hi=3):
    return [codes(g, n_pages, page, nkv, d) for _ in range(2)] + [scales(g, n_pages, page // 16, nkv, lo=lo, hi=hi) for _ in range(2)]


def clone(p):
    return [t.clone() for t in p]


# ------------------------------------------------------------------ append

STEPS = [([1], [1], 16, 0), ([1, 1, 1, 1], [17, 1, 300, 16], 16, 0), ([3, 0, 5, 1, 16], [3, 9, 100, 64, 32], 48, 2),
         ([130, 1, 0], [130, 513, 5], 64, 3), ([1] * 70, list(range(1, 71)), 16, 1), ([2] * 40, [5] * 40, 256, 0),
         ([31, 17, 2, 64], [45, 33, 17, 80], 32, 1)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("case", range(len(STEPS)))
def test_append8(dtype, case):
    """Rows into fresh blocks and among positions held before, whose scale grows or not."""
    counts, lens, page, pad = STEPS[case]
    step = R.Step(counts, lens, page, seed=case, pad=pad)
    g = gen(case)
    nkv, d = [(8, 128), (2, 64), (3, 66), (9, 80)][case % 4]
    rows = randn(g, step.rows, 3 * nkv, d, dtype=dtype)
    rows[:, 2 * nkv:] *= torch.exp2(randn(g, step.rows, nkv, 1, std=3.0).round()).to(dtype)
    k, v = rows[:, nkv:2 * nkv], rows[:, 2 * nkv:]
    if pad:
        rows[step.n:] = math.nan
    gain = 1 + randn(g, d, dtype=dtype, std=0.2)
    pos = torch.randint(0, 9000, (step.rows,), generator=g, device="cuda", dtype=torch.int32)
    p = pool(g, step.n_pages, page, nkv, d)
    for norm, rope in ((gain, (1e6,)), (None, LLAMA), (None, None)):
        before, st = clone(p), status()
        B.oos_paged_append8(B.PagedCache8(*p), step.device(B), k, v, norm, 1e-6, rope and B.OosRopeConfig(*rope), pos, st)
        assert int(st) == 0
        ref, r = R.norm_rope(k[:step.n], norm, 1e-6, rope and R.rates(d, *rope), pos[:step.n])
        tol = 32 * R.F32 * r if norm is not None or rope else torch.zeros_like(r)      # as in check_norm_rope
        R8.check_append(step, (before[0], before[2]), (p[0], p[2]), ref, tol, (dtype, case, "k", rope))
        y = v[:step.n].double().cpu()
        R8.check_append(step, (before[1], before[3]), (p[1], p[3]), y, torch.zeros_like(y), (dtype, case, "v"))
        rows[:step.n] *= 4      # the next pass needs larger scales


def test_append8_token_by_token():
    """A block that is filled one position after the other: each time the scale grows, what is there is rounded
    again; then the next block is begun."""
    nkv, d, n = 2, 128, 20
    g = gen(0)
    k, v = randn(g, n, nkv, d, dtype=BF16), randn(g, n, nkv, d, dtype=BF16)
    v *= 2.0 ** torch.tensor([0, 1, 0, 3, -5, 9, 2, 0, 0, 1, 20, 3, 1, 0, 0, 0, -30, 1, -40, 0], device="cuda")[:, None, None]
    p = pool(g, 3, 16, nkv, d, lo=30, hi=40)
    st = status()
    for i in range(n):
        step = R.Step([1], [i + 1], 16, spare_pages=1)
        step.table, step.n_pages, step.width = [[2, 0]], 3, 2
        before = clone(p)
        B.oos_paged_append8(B.PagedCache8(*p), step.device(B), k[i:i + 1], v[i:i + 1], None, 0.0, None, None, st)
        for side, y in ((0, k), (1, v)):
            y = y[i:i + 1].double().cpu()
            R8.check_append(step, (before[side], before[2 + side]), (p[side], p[2 + side]), y, torch.zeros_like(y), i)
    assert int(st) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [128, 66, 2])
def test_append8_special_values(dtype, d):
    """Zeros take the least scale; infinite and NaN elements become NaN and leave the scale to the others; values of
    any magnitude keep four bits, the largest saturate."""
    step = R.Step([5, 16, 1, 1], [5, 16, 1, 1], 16)
    g = gen(1)
    v = randn(g, step.rows, 3, d, dtype=dtype)
    v[0] = 0
    v[1, 1, 1] = math.inf
    v[2, 2, 0] = math.nan
    v[3, 1, 0] = -math.inf
    v[5:, 0] *= 2.0 ** -120
    v[5:, 1] *= 2.0 ** 100
    v[21] = 0
    v[22] = math.nan
    v[20, 2, 1] = torch.finfo(dtype).max
    for shift in (0, 1):
        flat = torch.empty(v.numel() + 1, dtype=dtype, device="cuda")      # rows that start off 16-byte boundaries
        x = flat[shift:shift + v.numel()].view_as(v).copy_(v)
        p = pool(g, step.n_pages, 16, 3, d)
        before, st = clone(p), status()
        B.oos_paged_append8(B.PagedCache8(*p), step.device(B), x, x, None, 0.0, None, None, st)
        assert int(st) == 0
        y = v.double().cpu()
        for side in (0, 1):
            R8.check_append(step, (before[side], before[2 + side]), (p[side], p[2 + side]), y, torch.zeros_like(y), shift)
    # a NaN that is held stays one when its block's scale grows
    step = R.Step([1], [2], 16)
    p = pool(g, step.n_pages, 16, 3, d)
    p[0].view(U8)[:, 0] = R8.NAN_CODE
    x = torch.full((1, 3, d), 2.0 ** 15, dtype=dtype, device="cuda")
    st = status()
    B.oos_paged_append8(B.PagedCache8(*p), step.device(B), x, x, None, 0.0, None, None, st)
    assert bool(torch.isnan(p[0][step.where(0, 0)[0], 0].float()).all()) and int(st) == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_append8_rounds_what_64_bits_give(dtype):
    """Codes next to a border.  A turned value is off by at most 6.5 half steps of its pair's length (cosine and sine 2.5
    each, their products and the sum 1.5), so by at most 8 steps of its own where it has nine tenths of that length; all
    of those within 8 steps of a border are computed in 64 bits."""
    n, nkv, d = 16384, 8, 128
    step = R.Step([n], [n], 256)
    g = gen(5)
    k = randn(g, n, nkv, d, dtype=dtype)
    pos = torch.randint(0, 100000, (n,), generator=g, device="cuda", dtype=torch.int32)
    p = pool(g, step.n_pages, 256, nkv, d)
    st = status()
    B.oos_paged_append8(B.PagedCache8(*p), step.device(B), k, k, None, 0.0, B.OosRopeConfig(1e6), pos, st)
    assert int(st) == 0
    ref, r = R.norm_rope(k, None, 0.0, R.rates(d, 1e6), pos)
    order = torch.tensor(step.table[0])
    codes = p[0].cpu().double()[order].view(n, nkv, d)
    e = R8.exps(p[2])[order].view(n // 16, nkv).repeat_interleave(16, 0)[..., None]
    want = R8.e4m3(torch.ldexp(ref, -e))
    large = ref.abs() >= 0.9 * r
    assert int(large.sum()) > n * nkv * d // 5 and not bool((codes != want)[large].any())


def test_append8_reports_rows_without_a_place():
    """A page outside the pool, a position outside the table, a length below the step's rows: those blocks are left
    out and reported, the others are appended."""
    nkv, d, page = 2, 128, 16
    for what in ("page", "negative page", "width", "length"):
        step = R.Step([20, 20, 2], [26, 38, 6], page)
        if what in ("page", "negative page"):
            step.table[1][2] = step.n_pages if what == "page" else -1
        elif what == "width":
            step.lens[1] = page * len(step.table[1]) + 2
        else:
            step.lens[1] = 1
        v = randn(gen(1), step.rows, nkv, d, dtype=BF16)
        p = pool(gen(2), step.n_pages, page, nkv, d)
        before, st = clone(p), status()
        B.oos_paged_append8(B.PagedCache8(*p), step.device(B), v, v, None, 1e-6, None, None, st)
        assert int(st) == B.OOS_EBATCH, what
        # the same step without what has no place
        y, counts, lens = v.double().cpu(), list(step.counts), list(step.lens)
        if what in ("page", "negative page"):
            counts[1], lens[1] = 14, 32
        elif what == "width":
            counts[1], lens[1] = 18, page * len(step.table[1])
        else:
            counts[1], lens[1] = 1, 1
        keep = list(range(20)) + [20 + i + (19 if what == "length" else 0) for i in range(counts[1])] + [40, 41]
        ok = R.Step(counts, lens, page)
        ok.table, ok.n_pages = step.table, step.n_pages
        for side in (0, 1):
            R8.check_append(ok, (before[side], before[2 + side]), (p[side], p[2 + side]), y[keep], torch.zeros_like(y[keep]), what)


def test_append8_offsets_out_of_order():
    """Sequences whose offsets decrease or pass the rows are left out and reported, lengths of any value do no harm."""
    g = gen(4)
    v = randn(g, 6, 1, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    for q_start, lens in (([0, 9, 1, 2], [9, 1, 1]), ([0, 2, 4, 6], [-1, 2, 2 ** 31 - 1]), ([0, 2, 4, 6], [-2 ** 31, 2, 2])):
        p = pool(g, 4, 16, 1, 64)
        before, st = clone(p), status()
        batch = B.Batch(torch.tensor(q_start, **i32), torch.tensor(lens, **i32), torch.tensor([[0], [1], [2]], **i32), 6)
        B.oos_paged_append8(B.PagedCache8(*p), batch, v, v, None, 1e-6, None, None, st)
        assert int(st) == B.OOS_EBATCH
        assert torch.equal(p[0][3].view(U8), before[0][3].view(U8)) and torch.equal(p[2][3], before[2][3])
        if q_start[1] == 2:
            assert bool(((p[0][1, :2].float() * torch.exp2(p[2][1].float() - 127)[:, :, None] - v[2:4]).abs() <= 2.0 ** -4 * v[2:4].abs() + 2.0 ** -16).all())


def test_append8_far_pages():
    """Positions past 2^32 codes of the pool."""
    nkv, d, page, n_pages = 8, 128, 64, 80000
    kp, vp = [torch.empty(n_pages, page, nkv, d, dtype=U8, device="cuda").view(E4M3) for _ in range(2)]
    sc = [torch.zeros(n_pages, page // 16, nkv, dtype=U8, device="cuda") for _ in range(2)]
    x = randn(gen(1), 2, nkv, d, dtype=BF16)
    i32 = dict(dtype=torch.int32, device="cuda")
    batch = B.Batch(torch.tensor([0, 2], **i32), torch.tensor([65], **i32), torch.tensor([[n_pages - 2, n_pages - 1]], **i32), 2)
    kp[n_pages - 2, 48:] = 0
    vp[n_pages - 2, 48:] = 0
    st = status()
    B.oos_paged_append8(B.PagedCache8(kp, vp, *sc), batch, x, x, None, 1e-6, None, None, st)
    assert int(st) == 0
    for t, s in ((kp, sc[0]), (vp, sc[1])):
        for i, (a, b) in enumerate(((n_pages - 2, 63), (n_pages - 1, 0))):
            y = R8.values(t[a, b // 16 * 16:b // 16 * 16 + 16], s[a, b // 16][None])[b % 16]
            assert bool(((y - x[i].double().cpu()).abs() <= 2.0 ** -4 * x[i].double().cpu().abs() + 2.0 ** -16).all())


# ------------------------------------------------------------------ attention

def attend8(step, q, pk, pv, prefix, cache, parent=None, scale=None, out=None, st=None, stream=None, ws=None):
    batch = step.device(B)
    st = status() if st is None else st
    out = torch.full_like(q, 7.0) if out is None else out
    n = B.oos_shared_prefix_attention8_workspace_bytes(q, prefix, cache, batch)
    ws = torch.full((n,), 255, dtype=U8, device="cuda") if ws is None else ws     # NaN where nothing is written
    B.oos_shared_prefix_attention8(q, pk, pv, prefix, cache, batch, parent, scale or 1 / math.sqrt(q.shape[-1]), out, ws,
                                   st, stream=stream)
    return out, st


def inputs8(step, prefix, nq, nkv, d, dtype, kv, seed=0, std=1.5, lo=-8, hi=-4):
    """q, prefix and a cache of codes whose slots that no row sees are NaN, with scales that are NaN's byte where a
    block has none that is."""
    g = gen(seed)
    q = randn(g, step.rows, nq, d, dtype=dtype, std=std)
    q[step.n:] = math.nan
    pk, pv = [randn(g, prefix + 3, nkv, d, dtype=kv) for _ in range(2)]
    pk[prefix:], pv[prefix:] = math.nan, math.nan
    x = pool(g, step.n_pages, step.page, nkv, d, lo=lo, hi=hi)
    seen = torch.zeros(step.n_pages, step.page, dtype=torch.bool)
    for b, n in enumerate(step.lens):
        for s in range(n):
            seen[step.where(b, s)] = True
    none = ~seen.cuda()
    for t in x[:2]:
        t.view(U8)[none] = R8.NAN_CODE
    for t in x[2:]:
        t[none.view(step.n_pages, -1, 16).all(-1)] = 255
    return q, pk, pv, B.PagedCache8(*x)


def run_case8(counts, lens, page, pad, prefix, nq, nkv, d, dtype, kv, parent=None, seed=0, std=1.5, width=None, **how):
    step = R.Step(counts, lens, page, seed=seed, pad=pad, width=width)
    q, pk, pv, cache = inputs8(step, prefix, nq, nkv, d, dtype, kv, seed, std, **how)
    par = None if parent is None else torch.tensor(parent + [0] * pad, dtype=torch.int32, device="cuda")
    out, st = attend8(step, q, pk, pv, prefix, cache, par)
    assert int(st) == 0
    ref = R8.attention(step, q, pk[:prefix], pv[:prefix], cache, 1 / math.sqrt(d), parent)
    R8.check_attention(out[:step.n], *ref, prefix + max(lens), (counts, lens, prefix))
    assert bool((out[step.n:] == 7.0).all())
    again, _ = attend8(step, q, pk, pv, prefix, cache, par)
    assert torch.equal(out, again)       # sums in a fixed order
    return out


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("prefix", [0, 1, 129, 1000])
@pytest.mark.parametrize("nq, nkv", [(16, 8), (5, 1), (6, 6)])
def test_attention8_decode(dtype, kv, prefix, nq, nkv):
    run_case8([1, 1, 1, 1, 1], [1, 16, 17, 130, 259], 16, 0, prefix, nq, nkv, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("page", [16, 48, 256])
def test_attention8_ragged(dtype, kv, page):
    """Requests of 0 to 150 rows, five heads per group, rows behind the last request."""
    run_case8([3, 0, 150, 1, 40], [3, 9, 200, 64, 40], page, 3, 200, 10, 2, 128, dtype, kv, seed=page)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("prefix", [0, 77])
def test_attention8_trees(dtype, kv, prefix):
    """Trees of 1 to 128 rows, forests among them, and a bare chain."""
    rng = np.random.RandomState(4)
    counts = [1, 64, 0, 128, 33, 128]
    parent = []
    for c in counts[:-1]:
        parent += [-1 if j == 0 or rng.rand() < 0.1 else int(rng.randint(max(0, j - 9), j)) for j in range(c)]
    parent += list(range(-1, 127))
    run_case8(counts, [1, 100, 30, 128, 333, 140], 32, 2, prefix, 8, 2, 128, dtype, kv, parent=parent, seed=3)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("counts", [[1, 4, 2, 6], [1] * 20, [16, 9, 30, 12]])
def test_attention8_small_trees(dtype, kv, counts):
    """Trees of a few rows: tiles of 8, 16 and more rows, blocks of keys that hold committed positions and nodes."""
    parent = [-1 if j == 0 else (j * 5) % j if j % 4 else -1 for c in counts for j in range(c)]
    run_case8(counts, [c + 29 * i % 75 for i, c in enumerate(counts)], 16, 1, 40, 8, 2, 128, dtype, kv, parent=parent)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("d", [2, 32, 64, 66, 80])
def test_attention8_head_sizes(dtype, kv, d):
    run_case8([2, 9, 1, 70], [50, 9, 100, 90], 16, 1, 70, 6, 2, d, dtype, kv, seed=d)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("counts, lens", [([1, 2, 1], [5000, 3, 2500]), ([100], [4100]), ([60, 200], [3000, 700])])
def test_attention8_long_sequences(dtype, kv, counts, lens):
    """Several ranges of keys a sequence, empty ones among them."""
    run_case8(counts, lens, 64, 0, 300, 8, 2, 128, dtype, kv, width=200)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("most", [1, 2])
def test_attention8_beside_a_long_prefix(dtype, kv, most):
    counts = [1 + i % most for i in range(60)]
    run_case8(counts, [c + 4 * i % 400 for i, c in enumerate(counts)], 16, 2, 9000 if kv is F32 else 20000, 8, 1, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES)
def test_attention8_many_sequences(dtype, kv):
    counts = [(i * 7) % 3 for i in range(1100)]
    run_case8(counts, [c + i % 5 for i, c in enumerate(counts)], 16, 1, 33, 20, 1, 128 if kv is not F32 else 64, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("n", [33, 64, 65])
def test_attention8_many_rows_of_many_sequences(dtype, kv, n):
    """Tiles dealt by their sequences' lengths, equal ones among them, and more sequences than that holds."""
    counts = [0 if i % 9 == 4 else 70 if i % 5 else 130 for i in range(n)]
    lens = [c + (i * 37) % 11 * 20 for i, c in enumerate(counts)]
    run_case8(counts, lens, 16, 2, 30, 2, 2, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("counts, lens", [([1, 1, 2], [100, 300, 40]), ([90, 140], [200, 300])])
@pytest.mark.parametrize("lo, hi", [(-117, -100), (-60, 30), (100, 119)])
def test_attention8_scales_of_any_size(dtype, kv, counts, lens, lo, hi):
    """Blocks whose scales lie far apart, the smallest and the largest there are: v keeps its digits whatever stands
    beside it.  The scores are kept small by the query's scale."""
    d = 128
    step = R.Step(counts, lens, 16)
    q, pk, pv, cache = inputs8(step, 0, 4, 2, d, dtype, kv, lo=lo, hi=hi)
    if hi > 110:      # sums of values near the largest stay finite, and so does out
        if dtype is F16:
            return
        cache.v.copy_((cache.v.float() / 64).to(E4M3))
    scale = 2.0 ** -max(lo + 8, hi + 8) if abs(hi) < 110 else 2.0 ** -120
    scale = min(scale, 2.0 ** 100)
    out, st = attend8(step, q, None, None, 0, cache, scale=scale)
    assert int(st) == 0
    ref, mag, size, tops = R8.attention(step, q, pk[:0], pv[:0], cache, scale)
    if dtype is F16:
        top = ref.abs() < 65000
        out, ref, mag = [torch.where(top, t.double().cpu(), 0.0).to(t.dtype) for t in (out, ref, mag)]
    R8.check_attention(out, ref, mag, size, tops, max(lens))


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("counts, lens", [([2, 5], [30, 12]), ([70, 130], [90, 150])])
def test_attention8_rows_any_stride(dtype, kv, counts, lens):
    """q a slice of a projection's rows, out a slice of wider rows that starts off 16-byte boundaries."""
    step = R.Step(counts, lens, 16)
    q, pk, pv, cache = inputs8(step, 40, 8, 2, 128, dtype, kv)
    wide_q = torch.zeros(step.rows, 12, 128, dtype=dtype, device="cuda")
    wide_q[:, 1:9] = q
    flat = torch.full((step.rows * 1031 + 1,), 7.0, dtype=dtype, device="cuda")
    out = torch.as_strided(flat, (step.rows, 8, 128), (1031, 128, 1), 1)
    attend8(step, wide_q[:, 1:9], pk, pv, 40, cache, out=out)
    plain, _ = attend8(step, q, pk, pv, 40, cache)
    assert torch.equal(out, plain)
    odd = torch.as_strided(torch.zeros(step.rows * 1031 + 1, dtype=dtype, device="cuda"), (step.rows, 8, 128), (1031, 128, 1), 1)
    odd.copy_(q)
    again, _ = attend8(step, odd, pk, pv, 40, cache, out=torch.empty_like(plain))
    assert torch.equal(again, plain)
    guard = torch.ones_like(flat, dtype=torch.bool)
    for i in range(step.rows):
        guard[1 + i * 1031:1 + i * 1031 + 1024] = False
    assert bool((flat[guard] == 7.0).all())


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("last", [3, 150])
def test_attention8_large_and_special_scores(dtype, kv, last):
    """Rows whose scores are huge in either direction; a NaN key that is seen makes its rows NaN, and only those."""
    step = R.Step([1, 1, last], [40, 3, 17 + last], 16)
    q, pk, pv, cache = inputs8(step, 130, 4, 2, 128, dtype, kv, std=60.0)
    out, _ = attend8(step, q, pk, pv, 130, cache)
    ref = R8.attention(step, q, pk[:130], pv[:130], cache, 1 / math.sqrt(128))
    R8.check_attention(out, *ref, 170)
    p, e = step.where(1, 2)
    cache.k.view(U8)[p, e, 1, 5] = R8.NAN_CODE
    out2, _ = attend8(step, q, pk, pv, 130, cache)
    nan = torch.isnan(out2).any(-1).cpu()
    want = torch.zeros(2 + last, 4, dtype=torch.bool)
    want[1, 2:] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("counts, lens, nodes", [([3, 1, 90, 30], [3, 20, 200, 31], (2, 40, 7)),
                                                 ([3, 1, 9, 5], [3, 20, 200, 31], (2, 4, 3)),
                                                 ([2, 1, 3, 1], [9, 20, 200, 31], (1, 1, 0))])
def test_attention8_masked_places_hold_anything(dtype, kv, tree, counts, lens, nodes):
    """A NaN k or v at one of the step's own positions reaches the rows that see it, and no other."""
    step = R.Step(counts, lens, 16)
    parent = ([j - 1 for j in range(counts[0])] + [-1] + [-1 if j == 0 else j // 2 for j in range(counts[2])] + [-1] * counts[3]
              if tree else None)
    par = torch.tensor(parent, dtype=torch.int32, device="cuda") if tree else None
    q, pk, pv, cache = inputs8(step, 50, 6, 2, 128, dtype, kv)
    ref = R8.attention(step, q, pk[:50], pv[:50], cache, 1 / math.sqrt(128), parent)
    for side in ("v", "k"):
        held = getattr(cache, side).view(U8).clone()
        sees = torch.zeros(step.n, dtype=torch.bool)
        for b, node in zip((0, 2, 3), nodes):
            lo, c, n = step.q_start[b], counts[b], lens[b]
            p, e = step.where(b, n - c + node)
            getattr(cache, side).view(U8)[p, e, 1, 3] = R8.NAN_CODE
            rel = R.ancestors(parent[lo:lo + c]) if tree else torch.ones(c, c).tril() > 0
            sees[lo:lo + c] |= rel[:, node]
        out, st = attend8(step, q, pk, pv, 50, cache, par)
        assert int(st) == 0
        want = torch.zeros(step.n, 6, 128, dtype=torch.bool)
        if side == "v":
            want[sees, 3:, 3] = True
        else:
            want[sees, 3:] = True
        assert torch.equal(torch.isnan(out).cpu(), want), side
        fill = torch.where(want, ref[0].to(out.dtype), out.cpu())
        R8.check_attention(fill, *ref, 250, side)
        getattr(cache, side).view(U8).copy_(held)


@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("counts", [[1, 1, 40], [70, 1, 90]])
def test_attention8_queries_of_any_size(dtype, kv, counts):
    """Queries far above and below one must neither overflow nor vanish."""
    step = R.Step(counts, [39 + counts[0], 3, 20 + counts[2]], 16)
    top = 2.0 ** 15 if dtype is F16 else 2.0 ** 60
    for factor in (top, 2.0 ** -13 if dtype is F16 else 2.0 ** -60):
        q, pk, pv, cache = inputs8(step, 200, 4, 2, 128, dtype, kv, std=0.3)
        q = (q.float() * factor).to(dtype)
        scale = 1 / math.sqrt(128) / factor
        out, _ = attend8(step, q, pk, pv, 200, cache, scale=scale)
        ref = R8.attention(step, q, pk[:200], pv[:200], cache, scale)
        R8.check_attention(out, *ref, 200 + max(step.lens), factor)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("rows", [2, 60])
def test_attention8_reports_bad_batches(dtype, kv, rows):
    """A page outside the pool is not seen; a length below the step's rows leaves rows without keys (zeros); a
    malformed parent counts as a root.  All are reported, other sequences keep their results."""
    nq, nkv, d, page = 4, 2, 128, 16
    good = R.Step([1, rows, 1], [40, rows, 30], page)
    q, _, _, cache = inputs8(good, 0, nq, nkv, d, dtype, kv)
    base, st = attend8(good, q, None, None, 0, cache)
    last = rows + 1
    assert int(st) == 0
    for what in ("page", "length", "width"):
        step = R.Step([1, rows, 1], [40, rows, 30], page)
        if what == "page":
            step.table[0][1] = step.n_pages + 5
        elif what == "length":
            step.lens[1] = rows - 1
        else:
            step.lens[0] = 10 ** 6
        out, st = attend8(step, q, None, None, 0, cache)
        assert int(st) == B.OOS_EBATCH, what
        assert torch.equal(out[last], base[last])
        if what == "length":
            assert bool((out[1] == 0).all()) and torch.equal(out[0], base[0])     # the first row would be position -1
        if what == "page":
            k, v = [torch.cat([t[good.table[0][0]], t[good.table[0][2]][:8]]) for t in
                    (R8.values(cache.k, cache.k_scale), R8.values(cache.v, cache.v_scale))]
            for h in range(nq):
                w = torch.softmax(k[:, h // 2] @ q[0, h].double().cpu() / math.sqrt(d), 0)
                assert float((w @ v[:, h // 2] - out[0, h].double().cpu()).abs().max()) < 0.05 * float(v.abs().max())
    roots = [-1] * (rows + 2)
    bad = torch.tensor(roots[:2] + [5] + roots[3:], dtype=torch.int32, device="cuda")
    out, st = attend8(good, q, None, None, 0, cache, parent=bad)
    assert int(st) == B.OOS_ETREE
    fine = torch.tensor(roots, dtype=torch.int32, device="cuda")
    ref, st = attend8(good, q, None, None, 0, cache, parent=fine)
    assert int(st) == 0 and torch.equal(ref, out)
    for n in (-1, -2 ** 31, 2 ** 31 - 1):
        for parents in (None, fine):
            step = R.Step([1, rows, 1], [40, rows, 30], page)
            ref, st = attend8(step, q, None, None, 0, cache, parent=parents)
            step.lens[1] = n
            out, st = attend8(step, q, None, None, 0, cache, parent=parents)
            assert int(st) == B.OOS_EBATCH
            assert torch.equal(out[0], ref[0]) and torch.equal(out[last], ref[last])
    step = R.Step([1, rows, 1], [40, rows, 30], page)
    step.q_start = [0, 1, 99, 4]
    out, st = attend8(step, q, None, None, 0, cache)
    assert int(st) == B.OOS_EBATCH and torch.equal(out[0], base[0])


def test_attention8_refuses_a_small_workspace():
    step = R.Step([1], [5], 16)
    q, pk, pv, cache = inputs8(step, 10, 4, 2, 128, BF16, BF16)
    n = B.oos_shared_prefix_attention8_workspace_bytes(q, 10, cache, step.device(B))
    assert n > 0
    for ws in (torch.empty(n - 1, dtype=U8, device="cuda"), torch.empty(n + 256, dtype=U8, device="cuda")[1:]):
        with pytest.raises(B.OosError) as e:
            attend8(step, q, pk, pv, 10, cache, ws=ws)
        assert e.value.code == B.OOS_EWORKSPACE


@pytest.mark.parametrize("rows", [1, 60])
def test_attention8_far_pages(rows):
    """Pages past 2^32 codes of the pool."""
    nkv, d, page, n_pages = 8, 128, 64, 80000
    far_kv = [torch.empty(n_pages, page, nkv, d, dtype=U8, device="cuda").view(E4M3) for _ in range(2)]
    far_sc = [torch.zeros(n_pages, page // 16, nkv, dtype=U8, device="cuda") for _ in range(2)]
    near_p = pool(gen(1), 2, page, nkv, d, lo=-8, hi=-5)
    for a, b in zip(far_kv + far_sc, near_p):
        a[n_pages - 2:] = b
    q = randn(gen(3), rows, 16, d, dtype=BF16)
    far, near = R.Step([rows], [100], page), R.Step([rows], [100], page)
    far.n_pages, far.table = n_pages, [[n_pages - 2, n_pages - 1]]
    near.n_pages, near.table = 2, [[0, 1]]
    a, st = attend8(far, q, None, None, 0, B.PagedCache8(*far_kv, *far_sc))
    b, _ = attend8(near, q, None, None, 0, B.PagedCache8(*near_p))
    assert int(st) == 0 and torch.equal(a, b)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("shape", ["decode", "ragged", "tree"])
def test_attention8_repeats_bit_for_bit(dtype, kv, shape):
    """Passes over cold and warm caches, next to another stream's traffic: a copy that is read before it has landed
    shows as a difference."""
    counts = {"decode": [1] * 40, "ragged": [100, 300, 17, 64, 33], "tree": [64, 128, 30, 90]}[shape]
    lens = [c + 37 * (i + 1) % 400 for i, c in enumerate(counts)]
    d = 64 if kv is F32 else 128
    parent = [j - 1 if j % 3 else max(-1, j - 3) for c in counts for j in range(c)] if shape == "tree" else None
    par = torch.tensor(parent, dtype=torch.int32, device="cuda") if parent else None
    for prefix in (0, 1300):
        step = R.Step(counts, lens, 16, seed=7)
        q, pk, pv, cache = inputs8(step, prefix, 8, 2, d, dtype, kv)
        base, st = attend8(step, q, pk, pv, prefix, cache, par)
        ref = R8.attention(step, q, pk[:prefix], pv[:prefix], cache, 1 / math.sqrt(d), parent)
        R8.check_attention(base, *ref, prefix + max(lens), shape)
        flush = torch.empty(1 << 28, dtype=U8, device="cuda")
        side = torch.cuda.Stream()
        outs = []
        for i in range(12):
            flush.fill_(i)
            if i >= 6:
                with torch.cuda.stream(side):
                    flush[:1 << 27].copy_(flush[1 << 27:])
            outs.append(attend8(step, q, pk, pv, prefix, cache, par)[0])
            side.synchronize()
        torch.cuda.synchronize()
        assert int(st) == 0 and all(torch.equal(base, o) for o in outs)


# ------------------------------------------------------------------ pages between steps

def paths_of(rng, counts, most):
    return [[0] + sorted(rng.choice(np.arange(1, c), min(c, int(rng.randint(1, most + 1))) - 1, replace=False).tolist())
            if c and rng.rand() < 0.9 else [] for c in counts]


def as_tensors(step, paths):
    flat = torch.full((step.rows,), -1, dtype=torch.int32)
    for b, p in enumerate(paths):
        flat[step.q_start[b]:step.q_start[b] + len(p)] = torch.tensor(p, dtype=torch.int32)
    return flat.cuda(), torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")


COMPACT = [([1], [1], 16, 1), ([64, 5, 0, 128, 30], [70, 5, 9, 333, 31], 16, 128), ([9] * 50, [9 + i for i in range(50)], 48, 9),
           ([128, 100], [128, 109], 64, 40)]


@pytest.mark.parametrize("kind", [F32, BF16, F16, E4M3])
@pytest.mark.parametrize("case", range(len(COMPACT)))
@pytest.mark.parametrize("nkv, d, layers", [(8, 128, 2), (3, 66, 3), (1, 2, 70), (2, 80, 1)])
def test_compact(kind, case, nkv, d, layers):
    counts, lens, page, most = COMPACT[case]
    if kind is not E4M3 and page == 48:
        page = 7
    step = R.Step(counts, lens, page, seed=case, pad=2)
    g, rng = gen(case), np.random.RandomState(case)
    paths = paths_of(rng, counts, most)
    if kind is E4M3:
        data = [pool(g, step.n_pages, page, nkv, d) for _ in range(layers)]
        held = B.PagedLayers([B.PagedCache8(*p) for p in data])
        run = B.oos_paged_compact8
    else:
        data = [[randn(g, step.n_pages, page, nkv, d, dtype=kind) for _ in range(2)] + [None, None] for _ in range(layers)]
        held = B.PagedLayers([B.PagedCache(*p[:2]) for p in data])
        run = B.oos_paged_compact
    before = [[None if t is None else t.clone() for t in p] for p in data]
    nodes, n = as_tensors(step, paths)
    new, st = torch.full((len(counts),), -5, dtype=torch.int32, device="cuda"), status()
    run(held, step.device(B), nodes, n, new, st)
    assert int(st) == 0
    assert new.tolist() == [m - c + len(p) for c, m, p in zip(counts, lens, paths)]
    for i in (0, layers // 2, layers - 1):
        for s in (0, 1):
            x, e = R8.compacted(step, paths, (before[i][s], before[i][2 + s]))
            assert R8.same(x, data[i][s].cpu().double())
            if e is not None:
                assert torch.equal(e, R8.exps(data[i][2 + s]))


@pytest.mark.parametrize("kind", [BF16, E4M3])
def test_compact_reports_bad_sequences(kind):
    """Nodes that do not ascend or are not the sequence's, counts, offsets and pages out of range: the sequence stays
    as it is and is reported, the others are moved."""
    nkv, d, page, counts, lens = 2, 128, 16, [6, 8, 5], [26, 40, 9]
    good = [[0, 2, 5], [0, 3, 4, 7], [0, 4]]
    for what in ("order", "twice", "far", "negative", "many", "negative count", "page", "length", "offsets"):
        step = R.Step(counts, lens, page, seed=1)
        paths = [list(p) for p in good]
        if what in ("order", "twice", "far", "negative"):
            paths[1] = {"order": [0, 4, 3], "twice": [0, 3, 3], "far": [0, 8], "negative": [-1, 2]}[what]
        nodes, n = as_tensors(step, paths)
        if what == "many":
            n[1] = 9
        elif what == "negative count":
            n[1] = -1
        elif what == "page":
            step.table[1][2] = step.n_pages
        elif what == "length":
            step.lens[1] = 7
        elif what == "offsets":
            step.q_start[2] = 10 ** 6
        p = pool(gen(2), step.n_pages, page, nkv, d) if kind is E4M3 else [randn(gen(2), step.n_pages, page, nkv, d, dtype=kind) for _ in range(2)] + [None] * 2
        before = [None if t is None else t.clone() for t in p]
        new, st = torch.zeros(3, dtype=torch.int32, device="cuda"), status()
        if kind is E4M3:
            B.oos_paged_compact8(B.PagedLayers([B.PagedCache8(*p)]), step.device(B), nodes, n, new, st)
        else:
            B.oos_paged_compact(B.PagedLayers([B.PagedCache(*p[:2])]), step.device(B), nodes, n, new, st)
        assert int(st) == B.OOS_EBATCH, what
        moved = [good[0], [], [] if what == "offsets" else good[2]]
        whole = R.Step(counts, lens, page, seed=1)
        assert new.tolist() == [23, step.lens[1], 9 if what == "offsets" else 6], what
        for s in (0, 1):
            x, e = R8.compacted(whole, moved, (before[s], before[2 + s]))
            assert R8.same(x, p[s].cpu().double()), what


@pytest.mark.parametrize("kind", [F32, BF16, E4M3])
@pytest.mark.parametrize("nkv, d, page, layers, shift", [(8, 128, 16, 3, 0), (3, 66, 32, 2, 1), (1, 2, 16, 70, 0), (2, 128, 512, 1, 2)])
def test_pages_copy(kind, nkv, d, page, layers, shift):
    """Whole pages, one source for several; pools that start off 16-byte boundaries; pairs out of range."""
    g, n = gen(1), 9
    order = torch.randperm(n, generator=torch.Generator().manual_seed(3)).tolist()
    src, dst = [order[0], order[0], order[1], order[2], n, -1, order[2]], order[3:7] + [order[7], order[7], n]

    def shifted(t):
        flat = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
        return flat[shift:].view(t.shape).copy_(t)

    if kind is E4M3:
        data = [[shifted(t) for t in pool(g, n, page, nkv, d)] for _ in range(layers)]
        held, run = B.PagedLayers([B.PagedCache8(*p) for p in data]), B.oos_pages_copy8
    else:
        data = [[shifted(randn(g, n, page, nkv, d, dtype=kind)) for _ in range(2)] for _ in range(layers)]
        held, run = B.PagedLayers([B.PagedCache(*p) for p in data]), B.oos_pages_copy
    want = [clone(p) for p in data]
    for p in want:
        for t in p:
            for a, b in list(zip(src, dst))[:4]:
                t.view(U8)[b] = t.view(U8)[a]
    for bad in (False, True):
        k = len(src) if bad else 4
        st = status()
        run(held, *(torch.tensor(x[:k], dtype=torch.int32, device="cuda") for x in (src, dst)), st)
        assert int(st) == (B.OOS_EBATCH if bad else 0)
        for a, b in zip(data, want):
            for x, y in zip(a, b):
                assert torch.equal(x.contiguous().view(U8), y.contiguous().view(U8))
    run(held, *(torch.zeros(0, dtype=torch.int32, device="cuda") for _ in range(2)), st)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype, kv", TYPES)
def test_steps_of_a_session(dtype, kv):
    """Prompts, a step with trees, the accepted nodes' move, forks of the pages in use, a step of the forks: the
    attention of each is the 64-bit one over what the pages hold then, which is what was appended, rounded; and the
    whole runs from a CUDA graph on another stream with the same bits."""
    nq, nkv, d, page, prefix = 8, 2, 128, 32, 150
    g = gen(9)
    pk, pv = randn(g, prefix, nkv, d, dtype=kv), randn(g, prefix, nkv, d, dtype=kv)
    kn = 1 + randn(g, d, dtype=dtype, std=0.1)
    rope = B.OosRopeConfig(1e6)
    prompts, trees, paths = [5, 40, 20], [12, 30, 1], [[0, 2, 3], [0, 5, 6, 29], [0]]
    parent = [-1 if j == 0 else j - 1 if j % 3 == 0 else j // 2 for c in trees for j in range(c)]
    for b, path in enumerate(paths):      # a path's nodes follow each other
        for a, j in zip(path, path[1:]):
            parent[sum(trees[:b]) + j] = a
    table = [[0, 3, 7], [5, 1, 8], [2, 4, 6]]
    lens = [prompts, [p + t for p, t in zip(prompts, trees)]]
    held = [p + len(x) for p, x in zip(prompts, paths)]
    # a fork of each: the last page in use is copied, the ones before are shared
    forks = [t[:h // page] + [9 + b] + [11 + b] * 0 for b, (t, h) in enumerate(zip(table, held))]
    steps = []
    for counts, n, tab in ((prompts, lens[0], table), (trees, lens[1], table),
                           ([1] * 6, [h + 1 for h in held] * 2, table + [f + [12 + b] for b, f in enumerate(forks)])):
        s = R.Step(counts, n, page, pad=1)
        s.table, s.n_pages = [list(t) + [0] * (3 - len(t)) for t in tab], 16
        s.table = [t[:3] for t in s.table]
        s.width = 3
        steps.append(s)
    src = torch.tensor([t[h // page] for t, h in zip(table, held)], dtype=torch.int32, device="cuda")
    dst = torch.tensor([9 + b for b in range(3)], dtype=torch.int32, device="cuda")
    rows = [randn(g, s.rows, nq + 2 * nkv, d, dtype=dtype) for s in steps]
    par = torch.tensor(parent + [0], dtype=torch.int32, device="cuda")
    pos = [torch.tensor([prefix + n - c + j for c, n in zip(s.counts, s.lens) for j in range(c)] + [0], dtype=torch.int32,
                        device="cuda") for s in steps]
    start = pool(g, 16, page, nkv, d)
    p = clone(start)
    cache = B.PagedCache8(*p)
    layers = B.PagedLayers([cache])
    outs = [torch.zeros(s.rows, nq, d, dtype=dtype, device="cuda") for s in steps]
    batches = [s.device(B) for s in steps]
    ws = torch.empty(max(B.oos_shared_prefix_attention8_workspace_bytes(o, prefix, cache, b) for o, b in zip(outs, batches)),
                     dtype=U8, device="cuda")
    nodes, n_nodes = as_tensors(steps[1], paths)
    new, st = torch.zeros(3, dtype=torch.int32, device="cuda"), status()

    def one(i, look):
        k, v = rows[i][:, nq:nq + nkv], rows[i][:, nq + nkv:]
        before = clone(p) if look else None
        B.oos_paged_append8(cache, batches[i], k, v, kn, 1e-6, rope, pos[i], st)
        if look:
            s = steps[i]
            ref, r = R.norm_rope(k[:s.n], kn, 1e-6, R.rates(d), pos[i][:s.n])
            R8.check_append(s, (before[0], before[2]), (p[0], p[2]), ref, 32 * R.F32 * r, i)
            y = v[:s.n].double().cpu()
            R8.check_append(s, (before[1], before[3]), (p[1], p[3]), y, torch.zeros_like(y), i)
        B.oos_shared_prefix_attention8(rows[i][:, :nq], pk, pv, prefix, cache, batches[i], par if i == 1 else None,
                                       1 / math.sqrt(d), outs[i], ws, st)
        if look:
            ref = R8.attention(s, rows[i][:, :nq], pk, pv, cache, 1 / math.sqrt(d), parent if i == 1 else None)
            R8.check_attention(outs[i][:s.n], *ref, prefix + max(s.lens), i)

    def session(look):
        for a, b in zip(p, start):
            a.copy_(b)
        one(0, look)
        one(1, look)
        before = clone(p) if look else None
        B.oos_paged_compact8(layers, batches[1], nodes, n_nodes, new, st)
        if look:
            assert new.tolist() == held
            for s in (0, 1):
                x, e = R8.compacted(steps[1], paths, (before[s], before[2 + s]))
                assert R8.same(x, p[s].cpu().double()) and torch.equal(e, R8.exps(p[2 + s]))
        B.oos_pages_copy8(layers, src, dst, st)
        one(2, look)

    session(True)
    assert int(st) == 0
    first, pages = [o.clone() for o in outs], clone(p)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        session(False)
    for o in outs:
        o.fill_(3.0)
    for _ in range(2):
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            graph.replay()
        torch.cuda.synchronize()
        assert int(st) == 0
        for s, a, b in zip(steps, outs, first):
            assert torch.equal(a[:s.n], b[:s.n])
        assert all(torch.equal(a.view(U8), b.view(U8)) for a, b in zip(p, pages))


@pytest.mark.parametrize("kind", [BF16, E4M3])
def test_compact_is_append_again(kind):
    """The move does what appending the accepted rows again does, where no scale differs."""
    nkv, d, page = 2, 128, 16
    step = R.Step([30, 8], [50, 8], page, seed=2)
    paths = [[0, 4, 9, 28], [0, 7]]
    g = gen(3)
    x = randn(g, step.rows, nkv, d, dtype=BF16).clamp(-3, 3)
    x[:, :, 0] = 3.5      # every position needs the same scale
    sides = []
    for again in (False, True):
        if kind is E4M3:
            p = [torch.zeros(step.n_pages, page, nkv, d, dtype=U8, device="cuda").view(E4M3) for _ in range(2)]
            p += [torch.full((step.n_pages, 1, nkv), 127 - 7, dtype=U8, device="cuda") for _ in range(2)]
            cache, append, move = B.PagedCache8(*p), B.oos_paged_append8, B.oos_paged_compact8
        else:
            cache, append, move = B.PagedCache.empty(step.n_pages, page, nkv, d, dtype=kind), B.oos_paged_append, B.oos_paged_compact
        st, new = status(), torch.zeros(2, dtype=torch.int32, device="cuda")
        append(cache, step.device(B), x, x, None, 0.0, None, None, st)
        if again:
            s2 = R.Step([4, 2], [24, 2], page, seed=2)
            s2.table, s2.width = step.table, step.width
            rows = torch.stack([x[step.q_start[b] + j] for b, q in enumerate(paths) for j in q])
            append(cache, s2.device(B), rows, rows, None, 0.0, None, None, st)
        else:
            nodes, n = as_tensors(step, paths)
            move(B.PagedLayers([cache]), step.device(B), nodes, n, new, st)
            assert new.tolist() == [24, 2]
        assert int(st) == 0
        k = cache.dequantized()[0] if kind is E4M3 else cache.k.float()
        sides.append([torch.stack([k[step.where(b, s)] for s in range(n)]) for b, n in enumerate((24, 2))])
    assert all(torch.equal(a, b) for a, b in zip(*sides))


def test_two_attention8_calls_at_once():
    """Calls on two streams with workspaces of their own do not disturb each other."""
    step = R.Step([1] * 20, list(range(1, 400, 20)), 16)
    sets = [inputs8(step, 900, 8, 2, 128, BF16, BF16, seed=s) for s in (1, 2)]
    want = [attend8(step, *(s[:3]), 900, s[3])[0] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    batch = step.device(B)
    ws = [torch.empty(B.oos_shared_prefix_attention8_workspace_bytes(sets[0][0], 900, s[3], batch), dtype=U8, device="cuda") for s in sets]
    outs, st = [torch.empty_like(w) for w in want], status()
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(sets):
            B.oos_shared_prefix_attention8(s[0], s[1], s[2], 900, s[3], batch, None, 1 / math.sqrt(128), outs[i], ws[i], st,
                                           stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want)) and int(st) == 0
