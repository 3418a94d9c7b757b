"""GPU tests of the batch operators against their 64-bit restatement (batch_ref.py)."""

import math

import numpy as np
import pytest
import torch

import batch_ref as R
from paper_2608_00814_gb300 import binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
LLAMA = (5e5, 8.0, 1.0, 4.0, 8192)


@pytest.fixture(autouse=True)
def _built():
    from paper_2608_00814_gb300 import _build
    _build.build()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ head norms and rotation

@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("n, nq, nkv, d", [(1, 16, 8, 128), (7, 5, 1, 64), (300, 3, 3, 80), (33, 4, 2, 66), (2, 1, 0, 2),
                                           (5, 0, 2, 128), (3000, 9, 3, 32), (4, 2, 2, 126)])
def test_norm_rope(dtype, n, nq, nkv, d):
    for seed, (norm, rope) in enumerate([(True, (1e6,)), (False, LLAMA), (True, None)]):
        g = gen(seed)
        rows = randn(g, n, nq + 2 * nkv, d, dtype=dtype, std=3.0)
        q = rows[:, :nq] if nq else None                   # slices of one projection's rows
        k = rows[:, nq:nq + nkv] if nkv else None
        before = rows.clone()
        gains = [1 + randn(g, d, dtype=dtype, std=0.2) if norm else None for _ in range(2)]
        pos = torch.randint(0, 100000, (n,), generator=g, device="cuda", dtype=torch.int32)
        outs = [torch.full((n, h + 1, d), 7.0, dtype=dtype, device="cuda") for h in (nq, nkv)]   # a guard head
        views = [o[:, :h] for o, h in zip(outs, (nq, nkv))]
        B.oos_qk_norm_rope(q, k, gains[0], gains[1], 1e-6, rope and B.OosRopeConfig(*rope), pos,
                           views[0] if nq else None, views[1] if nkv else None)
        assert torch.equal(rows, before)
        for x, o, v, gain, h in zip((q, k), outs, views, gains, (nq, nkv)):
            assert bool((o[:, h:] == 7.0).all())
            if x is not None:
                ref, r = R.norm_rope(x, gain, 1e-6, rope and R.rates(d, *rope), pos)
                R.check_norm_rope(v, ref, r, (dtype, n, d, seed))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_rope_in_place_and_unaligned(dtype):
    """q_out = q, and rows that start one element past a 16-byte boundary (narrow loads)."""
    g = gen(5)
    n, h, d = 37, 4, 128
    flat = randn(g, n * h * d + 1, dtype=dtype)
    pos = torch.arange(n, device="cuda", dtype=torch.int32) * 997
    for off in (0, 1):
        x = flat[off:off + n * h * d].view(n, h, d).clone() if off == 0 else None
        if off:
            buf = torch.empty(n * h * d + 1, dtype=dtype, device="cuda")
            x = buf[1:].view(n, h, d)
            x.copy_(flat[:-1].view(n, h, d))
        ref, r = R.norm_rope(x, None, 1e-6, R.rates(d), pos)
        B.oos_qk_norm_rope(x, None, None, None, 1e-6, B.OosRopeConfig(1e6), pos, x, None)
        R.check_norm_rope(x, ref, r, off)


def test_norm_rope_far_and_negative_positions():
    d = 128
    pos = torch.tensor([0, 1, -1, 4095, 1000003, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    n = pos.numel()
    x = randn(gen(3), n, 2, d)
    y = torch.empty_like(x)
    B.oos_qk_norm_rope(x, None, None, None, 0.0, B.OosRopeConfig(1e4), pos, y, None)
    # the 64-bit angle itself is off by 2^-53 of up to 2^31 radians: 2^-22, taken out by exact products of integers
    f = R.rates(d, 1e4)
    turns = torch.zeros(n, d // 2, dtype=torch.float64)
    for i, p in enumerate(pos.tolist()):
        for m in range(d // 2):
            num, den = (float(f[m]) / (2 * math.pi)).as_integer_ratio()
            turns[i, m] = (p * num % den) / den
    c, s = torch.cos(2 * math.pi * turns)[:, None], torch.sin(2 * math.pi * turns)[:, None]
    xd = x.double().cpu()
    h = d // 2
    ref = torch.cat((xd[..., :h] * c - xd[..., h:] * s, xd[..., h:] * c + xd[..., :h] * s), -1)
    R.check_norm_rope(y, ref, torch.hypot(xd[..., :h], xd[..., h:]).repeat(1, 1, 2))


def test_norm_rope_special_values():
    """Zeros stay zero, an infinite or NaN element makes its own head NaN and no other."""
    x = torch.ones(3, 4, 64, device="cuda")
    x[0, 1] = 0
    x[1, 2, 5] = math.inf
    x[2, 3, 7] = math.nan
    y = torch.empty_like(x)
    gain = torch.ones(64, device="cuda")
    B.oos_qk_norm_rope(x, None, gain, None, 1e-6, B.OosRopeConfig(1e6), torch.zeros(3, dtype=torch.int32, device="cuda"), y, None)
    assert bool((y[0, 1] == 0).all())
    nan = torch.isnan(y).any(-1).cpu()
    want = torch.zeros(3, 4, dtype=torch.bool)
    want[1, 2] = want[2, 3] = True
    assert torch.equal(nan, want)


# ------------------------------------------------------------------ append

STEPS = [([1], [1], 16, 0), ([1, 1, 1], [17, 1, 300], 16, 0), ([3, 0, 5, 1], [3, 9, 100, 64], 7, 2),
         ([130, 1, 0], [130, 513, 5], 64, 3), ([1] * 70, list(range(1, 71)), 1, 1), ([2] * 40, [5] * 40, 256, 0)]


@pytest.mark.parametrize("src, dst", [(F32, F32), (BF16, BF16), (BF16, F16), (F16, F16), (F32, BF16), (F32, F16),
                                      (BF16, F32)])
@pytest.mark.parametrize("case", range(len(STEPS)))
def test_append(src, dst, case):
    counts, lens, page, pad = STEPS[case]
    step = R.Step(counts, lens, page, seed=case, pad=pad)
    g = gen(case)
    nkv, d = [(8, 128), (2, 64), (3, 66)][case % 3]
    rows = randn(g, step.rows, 3 * nkv, d, dtype=src)
    k, v = rows[:, nkv:2 * nkv], rows[:, 2 * nkv:]
    if pad:
        k[step.n:] = math.nan
    gain = 1 + randn(g, d, dtype=src, std=0.2)
    pos = torch.randint(0, 9000, (step.rows,), generator=g, device="cuda", dtype=torch.int32)
    kp, vp = randn(g, step.n_pages, page, nkv, d, dtype=dst), randn(g, step.n_pages, page, nkv, d, dtype=dst)
    want_k, want_v = kp.clone(), vp.clone()
    for norm, rope in ((gain, (1e6,)), (None, LLAMA), (None, None)):
        st = status()
        B.oos_paged_append(B.PagedCache(kp, vp), step.device(B), k, v, norm, 1e-6, rope and B.OosRopeConfig(*rope),
                           pos, st)
        assert int(st) == 0
        ref, r = R.norm_rope(k[:step.n], norm, 1e-6, rope and R.rates(d, *rope), pos[:step.n])
        spots = [step.where(b, n - c + j) for b, (c, n) in enumerate(zip(counts, lens)) for j in range(c)]
        pi, ei = [torch.tensor(x, device="cuda") for x in zip(*spots)]
        R.check_norm_rope(kp[pi, ei], ref, r, (src, dst, case))
        want_v[pi, ei] = v[:step.n].to(dst)
        want_k[pi, ei] = kp[pi, ei]
        assert torch.equal(vp, want_v) and torch.equal(kp, want_k)     # nothing else was written


def test_append_reports_rows_without_a_place():
    """A page outside the pool, a position outside the table, a length below the step's rows: those rows
    are left out and reported, the others are appended."""
    nkv, d, page = 2, 128, 4
    for what in ("page", "negative page", "width", "length"):
        step = R.Step([2, 2, 2], [6, 8, 6], page, pad=0)
        if what == "page":
            step.table[1][1] = step.n_pages
        elif what == "negative page":
            step.table[1][1] = -1
        elif what == "width":
            step.lens[1] = 4 * len(step.table[1]) + 2
        else:
            step.lens[1] = 1
        k, v = randn(gen(1), 6, nkv, d, dtype=BF16), randn(gen(2), 6, nkv, d, dtype=BF16)
        kp = torch.zeros(step.n_pages, page, nkv, d, dtype=BF16, device="cuda")
        vp = torch.zeros_like(kp)
        st = status()
        B.oos_paged_append(B.PagedCache(kp, vp), step.device(B), k, v, None, 1e-6, None, None, st)
        assert int(st) == B.OOS_EBATCH, what
        want = torch.zeros_like(kp)
        rows = [(0, 4, 0), (0, 5, 1), (2, 4, 4), (2, 5, 5)] + ([(1, 0, 3)] if what == "length" else [])
        for b, s, i in rows:
            p, e = step.where(b, s)
            want[p, e] = k[i]
        assert torch.equal(kp, want), what


def test_append_offsets_out_of_order():
    """A row that its sequence's offsets do not hold is left out and reported, whatever the search finds."""
    k, v = randn(gen(1), 6, 1, 64, dtype=F32), randn(gen(2), 6, 1, 64, dtype=F32)
    kp = torch.zeros(4, 16, 1, 64, device="cuda")
    vp = torch.zeros_like(kp)
    i32 = dict(dtype=torch.int32, device="cuda")
    # row 5 counts two offsets not above it, and so falls to sequence 2, whose only row is row 1
    batch = B.Batch(torch.tensor([0, 9, 1, 2], **i32), torch.tensor([9, 1, 1], **i32),
                    torch.tensor([[0], [1], [2]], **i32), 6)
    st = status()
    B.oos_paged_append(B.PagedCache(kp, vp), batch, k, v, None, 1e-6, None, None, st)
    assert int(st) == B.OOS_EBATCH
    assert bool((kp[2, 1:] == 0).all()) and bool((vp[2, 1:] == 0).all())


def test_append_far_pages():
    """Positions past 2^31 elements of the pool."""
    nkv, d, page = 8, 128, 64
    n_pages = 40000                                  # 2.6e9 elements, 5.2 GB a side
    k, v = randn(gen(1), 2, nkv, d, dtype=BF16), randn(gen(2), 2, nkv, d, dtype=BF16)
    kp = torch.empty(n_pages, page, nkv, d, dtype=BF16, device="cuda")
    vp = torch.empty_like(kp)
    i32 = dict(dtype=torch.int32, device="cuda")
    batch = B.Batch(torch.tensor([0, 2], **i32), torch.tensor([65], **i32),
                    torch.tensor([[n_pages - 2, n_pages - 1]], **i32), 2)
    st = status()
    B.oos_paged_append(B.PagedCache(kp, vp), batch, k, v, None, 1e-6, None, None, st)
    assert int(st) == 0
    assert torch.equal(kp[n_pages - 2, 63], k[0]) and torch.equal(kp[n_pages - 1, 0], k[1])
    assert torch.equal(vp[n_pages - 2, 63], v[0]) and torch.equal(vp[n_pages - 1, 0], v[1])


# ------------------------------------------------------------------ attention

TYPES = [(F32, F32), (BF16, BF16), (BF16, F16), (F16, F16)]


def attend(step, q, pk, pv, prefix, kp, vp, parent=None, scale=None, out=None, st=None, stream=None, ws=None):
    cache, batch = B.PagedCache(kp, vp), step.device(B)
    st = status() if st is None else st
    out = torch.full_like(q, 7.0) if out is None else out
    n = B.oos_shared_prefix_attention_workspace_bytes(q, prefix, cache, batch)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if ws is None else ws     # NaN where nothing is written
    B.oos_shared_prefix_attention(q, pk, pv, prefix, cache, batch, parent, scale or 1 / math.sqrt(q.shape[-1]), out, ws,
                                  st, stream=stream)
    return out, st


def inputs(step, prefix, nq, nkv, d, dtype, kv, seed=0, std=1.5):
    """q, prefix and pages; every slot that no row sees is NaN."""
    g = gen(seed)
    q = randn(g, step.rows, nq, d, dtype=dtype, std=std)
    q[step.n:] = math.nan
    pk, pv = [randn(g, prefix + 3, nkv, d, dtype=kv) for _ in range(2)]
    pk[prefix:], pv[prefix:] = math.nan, math.nan
    pages = []
    for _ in range(2):
        p = torch.full((step.n_pages, step.page, nkv, d), math.nan, dtype=kv, device="cuda")
        x = randn(g, step.n_pages, step.page, nkv, d, dtype=kv)
        for b, n in enumerate(step.lens):
            for s in range(n):
                pi, ei = step.where(b, s)
                p[pi, ei] = x[pi, ei]
        pages.append(p)
    return q, pk, pv, pages[0], pages[1]


def run_case(counts, lens, page, pad, prefix, nq, nkv, d, dtype, kv, parent=None, seed=0, std=1.5):
    step = R.Step(counts, lens, page, seed=seed, pad=pad)
    q, pk, pv, kp, vp = inputs(step, prefix, nq, nkv, d, dtype, kv, seed, std)
    par = None if parent is None else torch.tensor(parent + [0] * pad, dtype=torch.int32, device="cuda")
    out, st = attend(step, q, pk, pv, prefix, kp, vp, par)
    assert int(st) == 0
    ref, mag, size = R.attention(step, q, pk[:prefix], pv[:prefix], kp, vp, 1 / math.sqrt(d), parent)
    keys = prefix + max(lens)
    R.check_attention(out[:step.n], ref, mag, size, keys, F32 if kv is F32 else kv, (counts, lens, prefix))
    assert bool((out[step.n:] == 7.0).all())
    again, _ = attend(step, q, pk, pv, prefix, kp, vp, par)
    assert torch.equal(out, again)       # sums in a fixed order
    return out


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("prefix", [0, 1, 63, 128, 129, 1000])
@pytest.mark.parametrize("nq, nkv", [(16, 8), (5, 1), (6, 6)])
def test_attention_decode(dtype, kv, prefix, nq, nkv):
    run_case([1, 1, 1, 1, 1], [1, 16, 17, 130, 259], 16, 0, prefix, nq, nkv, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("page", [1, 7, 64, 100])
def test_attention_ragged(dtype, kv, page):
    """Requests of 0 to 150 rows, five heads per group, rows behind the last request."""
    run_case([3, 0, 150, 1, 40], [3, 9, 200, 64, 40], page, 3, 200, 10, 2, 128, dtype, kv, seed=page)


@pytest.mark.parametrize("dtype, kv", TYPES)
def test_attention_trees(dtype, kv):
    """Trees of 1 to 128 rows, forests among them, and a bare chain."""
    rng = np.random.RandomState(4)
    counts = [1, 64, 0, 128, 33, 128]
    parent = []
    for c in counts[:-1]:
        parent += [-1 if j == 0 or rng.rand() < 0.1 else int(rng.randint(max(0, j - 9), j)) for j in range(c)]
    parent += list(range(-1, 127))
    run_case(counts, [1, 100, 30, 128, 333, 140], 32, 2, 77, 8, 2, 128, dtype, kv, parent=parent, seed=3)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("d", [2, 32, 64, 66, 80])
def test_attention_head_sizes(dtype, kv, d):
    run_case([2, 9, 1], [50, 9, 100], 16, 1, 70, 6, 2, d, dtype, kv, seed=d)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("d", [66, 96])
@pytest.mark.parametrize("most", [1, 2])
def test_attention_many_sequences_of_few_rows(dtype, kv, d, most):
    """Small tiles over the own keys, larger ones over the prefix."""
    counts = [1 + i % most for i in range(40)]
    run_case(counts, [c + 13 * i % 120 for i, c in enumerate(counts)], 16, 2, 150, 9, 3, d, dtype, kv, seed=d)


@pytest.mark.parametrize("dtype, kv", TYPES)
def test_attention_many_sequences(dtype, kv):
    """More sequences than one round of the search takes, one wide group of heads."""
    counts = [(i * 7) % 3 for i in range(1100)]
    run_case(counts, [c + i % 5 for i, c in enumerate(counts)], 4, 1, 33, 20, 1, 128 if kv is not F32 else 64, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES)
def test_attention_long_prefix_few_rows(dtype, kv):
    run_case([1, 2], [5000, 3], 64, 0, 9001, 4, 2, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("n_seqs, most", [(64, 9), (3, 16), (16, 16)])
@pytest.mark.parametrize("tree", [False, True])
def test_attention_several_tiles_of_few_rows(dtype, kv, n_seqs, most, tree):
    """Sequences of one to `most` tokens of five heads a group: a few 16-row tiles each, or one large one."""
    rng = np.random.RandomState(n_seqs)
    counts = [int(c) for c in rng.randint(1, most + 1, n_seqs)]
    parent = [-1 if j == 0 else int(rng.randint(-1, j)) for c in counts for j in range(c)] if tree else None
    run_case(counts, [c + int(rng.randint(0, 300)) for c in counts], 16, 1, 100, 10, 2, 128, dtype, kv, parent=parent)


@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("most", [1, 2])
def test_attention_pages_beside_a_long_prefix(dtype, kv, most):
    """The prefix's kernel leaves SMs free for long, and the sequences' own keys leave parts for a join."""
    counts = [1 + i % most for i in range(100)]
    run_case(counts, [c + 4 * i % 400 for i, c in enumerate(counts)], 16, 2, 20000, 8, 1, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", TYPES[1:])
def test_attention_many_rows_long_prefix(dtype, kv):
    """Several row tiles and several splits of the prefix; scores far enough apart that maxima move."""
    run_case([90, 1, 200, 77], [90, 300, 210, 500], 16, 1, 1501, 8, 2, 128, dtype, kv, std=6.0)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("shape", ["decode", "ragged", "tree"])
def test_attention_repeats_bit_for_bit(dtype, kv, shape):
    """Passes over cold and warm caches, next to another stream's traffic: a copy that is read before it has
    landed shows as a difference."""
    counts = {"decode": [1] * 40, "ragged": [100, 300, 17, 64, 33], "tree": [64, 128, 30, 90]}[shape]
    lens = [c + 37 * (i + 1) % 400 for i, c in enumerate(counts)]
    d = 64 if kv is F32 else 128
    parent = [j - 1 if j % 3 else max(-1, j - 3) for c in counts for j in range(c)] if shape == "tree" else None
    par = torch.tensor(parent, dtype=torch.int32, device="cuda") if parent else None
    for prefix in (0, 1300):
        step = R.Step(counts, lens, 16, seed=7)
        q, pk, pv, kp, vp = inputs(step, prefix, 8, 2, d, dtype, kv)
        base, st = attend(step, q, pk, pv, prefix, kp, vp, par)
        ref, mag, size = R.attention(step, q, pk[:prefix], pv[:prefix], kp, vp, 1 / math.sqrt(d), parent)
        R.check_attention(base, ref, mag, size, prefix + max(lens), F32 if kv is F32 else kv, shape)
        flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
        side = torch.cuda.Stream()
        outs = []
        for i in range(12):
            flush.fill_(i)
            if i >= 6:
                with torch.cuda.stream(side):
                    flush[:1 << 27].copy_(flush[1 << 27:])
            outs.append(attend(step, q, pk, pv, prefix, kp, vp, par)[0])
            side.synchronize()
        torch.cuda.synchronize()
        assert int(st) == 0 and all(torch.equal(base, o) for o in outs)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("counts, lens", [([2, 5], [30, 12]), ([70, 130], [90, 150])])
def test_attention_rows_any_stride(dtype, kv, counts, lens):
    """q a slice of a projection's rows, out a slice of wider rows that starts off 16-byte boundaries."""
    step = R.Step(counts, lens, 16)
    q, pk, pv, kp, vp = inputs(step, 40, 8, 2, 128, dtype, kv)
    wide_q = torch.zeros(step.rows, 12, 128, dtype=dtype, device="cuda")
    wide_q[:, 1:9] = q
    flat = torch.full((step.rows * 1031 + 1,), 7.0, dtype=dtype, device="cuda")
    out = torch.as_strided(flat, (step.rows, 8, 128), (1031, 128, 1), 1)
    attend(step, wide_q[:, 1:9], pk, pv, 40, kp, vp, out=out)
    plain, _ = attend(step, q, pk, pv, 40, kp, vp)
    assert torch.equal(out, plain)
    odd = torch.as_strided(torch.zeros(step.rows * 1031 + 1, dtype=dtype, device="cuda"), (step.rows, 8, 128), (1031, 128, 1), 1)
    odd.copy_(q)
    again, _ = attend(step, odd, pk, pv, 40, kp, vp, out=torch.empty_like(plain))
    assert torch.equal(again, plain)
    guard = torch.ones_like(flat, dtype=torch.bool)
    for i in range(step.rows):
        guard[1 + i * 1031:1 + i * 1031 + 1024] = False
    assert bool((flat[guard] == 7.0).all())


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("last", [3, 150])
def test_attention_large_and_special_scores(dtype, kv, last):
    """Rows whose scores are huge in either direction; a NaN key that is seen makes its rows NaN, and only those."""
    step = R.Step([1, 1, last], [40, 3, 17 + last], 16)
    q, pk, pv, kp, vp = inputs(step, 130, 4, 2, 128, dtype, kv, std=60.0)
    out, _ = attend(step, q, pk, pv, 130, kp, vp)
    ref, mag, size = R.attention(step, q, pk[:130], pv[:130], kp, vp, 1 / math.sqrt(128))
    R.check_attention(out, ref, mag, size, 170, F32 if kv is F32 else kv)
    p, e = step.where(1, 2)
    kp[p, e, 1, 5] = math.nan
    out2, _ = attend(step, q, pk, pv, 130, kp, vp)
    nan = torch.isnan(out2).any(-1).cpu()
    want = torch.zeros(2 + last, 4, dtype=torch.bool)
    want[1, 2:] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("counts, lens, nodes", [([3, 1, 90, 30], [3, 20, 200, 31], (2, 40, 7)),
                                                 ([3, 1, 9, 5], [3, 20, 200, 31], (2, 4, 3)),
                                                 ([2, 1, 3, 1], [9, 20, 200, 31], (1, 1, 0))])
def test_attention_masked_places_hold_anything(dtype, kv, tree, value, counts, lens, nodes):
    """A v or k that is not finite at one of the step's own positions reaches the rows that see it, and no other."""
    step = R.Step(counts, lens, 16)
    parent = ([j - 1 for j in range(counts[0])] + [-1] + [-1 if j == 0 else j // 2 for j in range(counts[2])] + [-1] * counts[3]
              if tree else None)
    par = torch.tensor(parent, dtype=torch.int32, device="cuda") if tree else None
    q, pk, pv, kp, vp = inputs(step, 50, 6, 2, 128, dtype, kv)
    base, _ = attend(step, q, pk, pv, 50, kp, vp, par)
    sees = torch.zeros(step.n, dtype=torch.bool)
    for b, node in zip((0, 2, 3), nodes):
        lo, c, n = step.q_start[b], counts[b], lens[b]
        p, e = step.where(b, n - c + node)
        vp[p, e, 1, 3] = value
        rel = R.ancestors(parent[lo:lo + c]) if tree else torch.ones(c, c).tril() > 0
        sees[lo:lo + c] |= rel[:, node]
    out, st = attend(step, q, pk, pv, 50, kp, vp, par)
    assert int(st) == 0
    got, want = out.float().cpu(), base.float().cpu()
    want[sees, 3:, 3] = value
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    same = torch.isfinite(want)
    assert torch.equal(got[~same & ~torch.isnan(want)], want[~same & ~torch.isnan(want)])
    # both sums are within their bounds of the exact one; compare with twice a loose one
    assert float((got - want)[same].abs().max()) <= 0.05 * float(want[same].abs().max())


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("counts", [[1, 1, 1], [1, 90, 60]])
@pytest.mark.parametrize("value", [math.inf, -math.inf])
def test_attention_infinite_values_stay_infinite(dtype, kv, counts, value):
    """An infinite v long before the step, where no row's weight vanishes: infinite in all rows, not NaN."""
    step = R.Step(counts, [40, 130, 90], 16)
    q, pk, pv, kp, vp = inputs(step, 50, 6, 2, 128, dtype, kv, std=0.2)
    p, e = step.where(0, 3)
    vp[p, e, 1, 3] = value
    pv[7, 0, 5] = value
    out, st = attend(step, q, pk, pv, 50, kp, vp)
    assert int(st) == 0
    want = torch.isfinite(out)
    assert bool((out[:counts[0], 3:, 3] == value).all()) and bool((out[:step.n, :3, 5] == value).all())
    want[:counts[0], 3:, 3] = True
    want[:step.n, :3, 5] = True
    assert bool(want[:step.n].all())


@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("counts", [[1, 1, 40], [70, 1, 90]])
def test_attention_queries_of_any_size(dtype, kv, counts):
    """Queries far above and below one: with binary16 pages they must neither overflow nor vanish."""
    step = R.Step(counts, [39 + counts[0], 3, 20 + counts[2]], 16)
    top = 2.0 ** 15 if dtype is F16 else 2.0 ** 60
    for factor in (top, 2.0 ** -13 if dtype is F16 else 2.0 ** -60):
        q, pk, pv, kp, vp = inputs(step, 200, 4, 2, 128, dtype, kv, std=0.3)
        q = (q.float() * factor).to(dtype)
        scale = 1 / math.sqrt(128) / factor
        out, _ = attend(step, q, pk, pv, 200, kp, vp, scale=scale)
        ref, mag, size = R.attention(step, q, pk[:200], pv[:200], kp, vp, scale)
        R.check_attention(out, ref, mag, size, 200 + max(step.lens), kv, factor)


@pytest.mark.parametrize("dtype, kv", TYPES)
def test_attention_reports_bad_batches(dtype, kv):
    """A page outside the pool is not seen; a length below the step's rows leaves rows without keys (zeros);
    a malformed parent counts as a root.  All are reported, other sequences keep their results."""
    nq, nkv, d, page = 4, 2, 128, 16
    good = R.Step([1, 2, 1], [40, 2, 30], page)
    q, _, _, kp, vp = inputs(good, 0, nq, nkv, d, dtype, kv)
    base, st = attend(good, q, None, None, 0, kp, vp)
    assert int(st) == 0
    for what in ("page", "length", "width"):
        step = R.Step([1, 2, 1], [40, 2, 30], page)
        if what == "page":
            step.table[0][1] = step.n_pages + 5
        elif what == "length":
            step.lens[1] = 1
        else:
            step.lens[0] = 10 ** 6
        out, st = attend(step, q, None, None, 0, kp, vp)
        assert int(st) == B.OOS_EBATCH, what
        assert torch.equal(out[3], base[3])
        if what == "length":
            assert bool((out[1] == 0).all())               # row 0 of two would be position -1
            assert torch.equal(out[2, :], out[2, :]) and torch.equal(out[0], base[0])
        if what == "page":
            k = torch.cat([kp[good.table[0][0]], kp[good.table[0][2]][:8]]).double().cpu()
            v = torch.cat([vp[good.table[0][0]], vp[good.table[0][2]][:8]]).double().cpu()
            for h in range(nq):
                w = torch.softmax(k[:, h // 2] @ q[0, h].double().cpu() / math.sqrt(d), 0)
                assert float((w @ v[:, h // 2] - out[0, h].double().cpu()).abs().max()) < 0.05
    bad = torch.tensor([-1, -1, 5, -1], dtype=torch.int32, device="cuda")
    out, st = attend(good, q, None, None, 0, kp, vp, parent=bad)
    assert int(st) == B.OOS_ETREE
    fine = torch.tensor([-1, -1, -1, -1], dtype=torch.int32, device="cuda")
    ref, st = attend(good, q, None, None, 0, kp, vp, parent=fine)
    assert int(st) == 0 and torch.equal(ref, out)
    # a length of any value: only the extremes' own rows are affected
    for n in (-1, -2 ** 31, 2 ** 31 - 1):
        for parents in (None, fine):
            step = R.Step([1, 2, 1], [40, 2, 30], page)
            ref, st = attend(step, q, None, None, 0, kp, vp, parent=parents)
            step.lens[1] = n
            out, st = attend(step, q, None, None, 0, kp, vp, parent=parents)
            assert int(st) == B.OOS_EBATCH
            assert torch.equal(out[0], ref[0]) and torch.equal(out[3], ref[3])
    # offsets that decrease or pass the rows: reported, and the sequence in order keeps its result
    step = R.Step([1, 2, 1], [40, 2, 30], page)
    step.q_start = [0, 1, 9, 4]
    out, st = attend(step, q, None, None, 0, kp, vp)
    assert int(st) == B.OOS_EBATCH and torch.equal(out[0], base[0])


def test_attention_refuses_a_small_workspace():
    step = R.Step([1], [5], 16)
    q, pk, pv, kp, vp = inputs(step, 10, 4, 2, 128, BF16, BF16)
    n = B.oos_shared_prefix_attention_workspace_bytes(q, 10, B.PagedCache(kp, vp), step.device(B))
    assert n > 0
    for ws in (torch.empty(n - 1, dtype=torch.uint8, device="cuda"), torch.empty(n + 256, dtype=torch.uint8, device="cuda")[1:]):
        with pytest.raises(B.OosError) as e:
            attend(step, q, pk, pv, 10, kp, vp, ws=ws)
        assert e.value.code == B.OOS_EWORKSPACE


def test_attention_far_pages():
    """Pages past 2^31 elements of the pool."""
    nkv, d, page, n_pages = 8, 128, 64, 40000
    kp = torch.empty(n_pages, page, nkv, d, dtype=BF16, device="cuda")
    vp = torch.empty_like(kp)
    near_k, near_v = randn(gen(1), 2, page, nkv, d, dtype=BF16), randn(gen(2), 2, page, nkv, d, dtype=BF16)
    kp[n_pages - 2:], vp[n_pages - 2:] = near_k, near_v
    q = randn(gen(3), 2, 16, d, dtype=BF16)
    far, near = R.Step([2], [100], page), R.Step([2], [100], page)
    far.n_pages, far.table = n_pages, [[n_pages - 2, n_pages - 1]]
    near.n_pages, near.table = 2, [[0, 1]]
    a, st = attend(far, q, None, None, 0, kp, vp)
    b, _ = attend(near, q, None, None, 0, near_k, near_v)
    assert int(st) == 0 and torch.equal(a, b)


# ------------------------------------------------------------------ together

def layer_step(step, g, nq, nkv, d, dtype, kv, prefix):
    q = randn(g, step.rows, nq + 2 * nkv, d, dtype=dtype)
    pos = [prefix + n - c + j for c, n in zip(step.counts, step.lens) for j in range(c)] + [0] * (step.rows - step.n)
    return q, torch.tensor(pos, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype, kv", TYPES)
def test_three_steps_of_a_layer(dtype, kv):
    """Prompts, then two decoding steps: norms and rotation, append, attention, as a layer runs them; replayed
    from a CUDA graph on another stream with new inputs, the results are the same bits."""
    nq, nkv, d, page, prefix = 8, 2, 128, 16, 150
    g = gen(9)
    pk, pv = randn(g, prefix, nkv, d, dtype=kv), randn(g, prefix, nkv, d, dtype=kv)
    qn, kn = 1 + randn(g, d, dtype=dtype, std=0.1), 1 + randn(g, d, dtype=dtype, std=0.1)
    rope = B.OosRopeConfig(1e6)
    lens0 = [5, 40, 1]
    full = R.Step([1, 1, 1], [n + 2 for n in lens0], page, pad=0)
    kp, vp = [torch.full((full.n_pages, page, nkv, d), math.nan, dtype=kv, device="cuda") for _ in range(2)]
    hist_k, hist_v = [[] for _ in lens0], [[] for _ in lens0]
    for t in range(3):
        counts = lens0 if t == 0 else [1, 1, 1]
        step = R.Step(counts, [n + t for n in lens0], page, pad=1)
        step.table, step.n_pages, step.width = full.table, full.n_pages, full.width
        rows, pos = layer_step(step, g, nq, nkv, d, dtype, kv, prefix)
        k, v = rows[:, nq:nq + nkv], rows[:, nq + nkv:]
        # the definition
        qr, _ = R.norm_rope(rows[:, :nq], qn, 1e-6, R.rates(d), pos)
        kr, _ = R.norm_rope(k, kn, 1e-6, R.rates(d), pos)
        q = torch.empty(step.rows, nq, d, dtype=dtype, device="cuda")
        out = torch.full((step.rows, nq, d), 7.0, dtype=dtype, device="cuda")
        st, cache, batch = status(), B.PagedCache(kp, vp), step.device(B)
        ws = torch.empty(B.oos_shared_prefix_attention_workspace_bytes(q, prefix, cache, batch), dtype=torch.uint8, device="cuda")

        def layer(stream):
            B.oos_qk_norm_rope(rows[:, :nq], None, qn, None, 1e-6, rope, pos, q, None, stream=stream)
            B.oos_paged_append(cache, batch, k, v, kn, 1e-6, rope, pos, st, stream=stream)
            B.oos_shared_prefix_attention(q, pk, pv, prefix, cache, batch, None, 1 / math.sqrt(d), out, ws, st, stream=stream)

        torch.cuda.synchronize()
        layer(None)
        torch.cuda.synchronize()
        assert int(st) == 0
        first = out.clone()
        ref_k, ref_v = [], []
        for b, c in enumerate(counts):
            for j in range(c):
                i = step.q_start[b] + j
                hist_k[b].append(kr[i])
                hist_v[b].append(v[i].double().cpu())
        for b in range(3):
            kk = torch.cat([pk.double().cpu(), torch.stack(hist_k[b])])
            vv = torch.cat([pv.double().cpu(), torch.stack(hist_v[b])])
            for j in range(counts[b]):
                i, seen = step.q_start[b] + j, prefix + step.lens[b] - counts[b] + j + 1
                for h in range(nq):
                    s = kk[:seen, h // 4] @ qr[i, h] / math.sqrt(d)
                    w = torch.softmax(s, 0)
                    got = out[i, h].double().cpu()
                    want = w @ vv[:seen, h // 4]
                    # rounding q and k to their types moves a score by (u_q + u_k) sum |q k|, that a weight
                    # by twice it; V, P and the output by half a step each
                    size = float((kk[:seen, h // 4].abs() @ qr[i, h].abs()).max()) / math.sqrt(d)
                    u, uk = R.U[dtype], R.U[kv]
                    mag = w @ vv[:seen, h // 4].abs()
                    tol = u * want.abs() + mag * (2 * (u + uk) * size + 2 * uk + 4 * 400 * R.F32)
                    assert bool(((got - want).abs() <= tol).all()), (t, b, j, h)
        # the same step from a graph, on its own stream
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer(torch.cuda.current_stream())
        out.fill_(3.0)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:step.n], first[:step.n])


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("prefix", [0, 700])
@pytest.mark.parametrize("counts", [[1] * 9, [40, 0, 7, 90]])
def test_calls_that_follow_each_other(dtype, kv, prefix, counts):
    """Layers whose queries are the layer's before, over the same pages, workspace and rows, with torch's kernels
    and fills between them: the same bits whether each call is waited for, none is, or a graph with a second
    stream in it runs them."""
    nq, nkv, d, page, layers = 8, 2, 128, 16, 6
    step = R.Step(counts, [c + 150 + 11 * i for i, c in enumerate(counts)], page, pad=1)
    g = gen(5)
    pk, pv = [randn(g, prefix + 1, nkv, d, dtype=kv) for _ in range(2)]
    pages = [randn(g, step.n_pages, page, nkv, d, dtype=kv) for _ in range(2)]
    start = randn(g, step.rows, nq + 2 * nkv, d, dtype=dtype)
    gain, pos = 1 + randn(g, d, dtype=dtype, std=0.1), torch.arange(step.rows, dtype=torch.int32, device="cuda")
    rope, batch, st = B.OosRopeConfig(1e6), step.device(B), status()
    kp, vp, rows = torch.empty_like(pages[0]), torch.empty_like(pages[1]), torch.empty_like(start)
    q, out = [torch.empty(step.rows, nq, d, dtype=dtype, device="cuda") for _ in range(2)]
    outs = torch.empty(layers, step.rows, nq, d, dtype=dtype, device="cuda")
    cache = B.PagedCache(kp, vp)
    ws = torch.empty(B.oos_shared_prefix_attention_workspace_bytes(q, prefix, cache, batch), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()

    def run(after):
        kp.copy_(pages[0]), vp.copy_(pages[1]), rows.copy_(start)
        for i in range(layers):
            fork, join = torch.cuda.Event(), torch.cuda.Event()
            out.zero_()
            fork.record()
            with torch.cuda.stream(side):
                side.wait_event(fork)
                rows[:, nq:].mul_(-1)
                join.record()
            after()
            B.oos_qk_norm_rope(rows[:, :nq], None, gain, None, 1e-6, rope, pos, q, None)
            after()
            torch.cuda.current_stream().wait_event(join)
            B.oos_paged_append(cache, batch, rows[:, nq:nq + nkv], rows[:, nq + nkv:], gain, 1e-6, rope, pos, st)
            after()
            B.oos_shared_prefix_attention(q, pk, pv, prefix, cache, batch, None, 1 / math.sqrt(d), out, ws, st)
            after()
            rows[:, :nq].copy_(out)
            outs[i].copy_(out)
            after()

    run(torch.cuda.synchronize)
    want = outs.clone()
    assert int(st) == 0 and not torch.equal(want[0], want[1])
    for _ in range(3):
        outs.zero_()
        run(lambda: None)
        torch.cuda.synchronize()
        assert torch.equal(outs, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(lambda: None)
    for _ in range(3):
        outs.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs, want)
    assert int(st) == 0


def test_two_calls_at_once():
    """Calls on two streams with workspaces of their own do not disturb each other."""
    step = R.Step([1] * 20, list(range(1, 400, 20)), 16)
    sets = [inputs(step, 900, 8, 2, 128, BF16, BF16, seed=s) for s in (1, 2)]
    want = [attend(step, *(s[:3]), 900, *s[3:])[0] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        outs = [torch.empty_like(w) for w in want]
        cache = [B.PagedCache(*s[3:]) for s in sets]
        batch = step.device(B)
        ws = [torch.empty(B.oos_shared_prefix_attention_workspace_bytes(sets[0][0], 900, cache[0], batch),
                          dtype=torch.uint8, device="cuda") for _ in sets]
        st = status()
        torch.cuda.synchronize()
        for _ in range(10):
            for i, s in enumerate(sets):
                B.oos_shared_prefix_attention(s[0], s[1], s[2], 900, cache[i], batch, None, 1 / math.sqrt(128), outs[i],
                                              ws[i], st, stream=streams[i])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("name", ["tiny", "mini-bf16", "mini-f16kv"])
def test_pages_hold_what_the_model_writes(name):
    """K and V of a prompt's first layer, projected here and appended to pages, against those that
    oos_prefill leaves in its cache."""
    import dataclasses

    from cases import build_case
    case = build_case("mini-bf16" if name == "mini-f16kv" else name, 0)
    if name == "mini-f16kv":
        case.cfg = dataclasses.replace(case.cfg, cache_dtype="f16")
    cfg = case.cfg
    from synth.device import upload_model
    w = upload_model(case.model)
    model = B.OosModel(cfg, w, max_T=128, use_graph=False)
    n, nkv, d = 100, cfg.n_kv_heads, cfg.head_dim
    kv = B.KVCache.empty(cfg, n + 8)
    tokens = torch.randint(0, cfg.vocab, (n,), generator=gen(2), device="cuda", dtype=torch.int32)
    B.oos_prefill(model, kv, 0, tokens, n)
    assert B.oos_last_status(model) == B.OOS_OK
    lw = w["layers"][0]
    x = w["embed"][tokens.long()].double()
    xn = x / torch.sqrt((x * x).mean(-1, keepdim=True) + cfg.rms_eps) * lw["attn_norm"].double()
    k = (xn @ lw["w_k"].double().T).float().view(n, nkv, d)
    v = (xn @ lw["w_v"].double().T).float().view(n, nkv, d)
    step = R.Step([60, 40], [60, 40], 16)
    cache = B.PagedCache.empty(step.n_pages, 16, nkv, d, dtype=kv.k[0].dtype)
    gain = lw["k_norm"].float() if cfg.qk_norm else None
    st = status()
    B.oos_paged_append(cache, step.device(B), k, v, gain, cfg.rms_eps, B.make_rope(cfg),
                       torch.arange(n, dtype=torch.int32, device="cuda"), st)
    assert int(st) == 0
    for j in range(n):
        p, e = step.where(0, j) if j < 60 else step.where(1, j - 60)
        for mine, theirs in ((cache.k, kv.k[0]), (cache.v, kv.v[0])):
            a, b = mine[p, e].double(), theirs[j].double()
            tol = 1e-4 if cfg.dtype == "f32" else 2e-2
            assert float((a - b).abs().max()) <= tol * max(1.0, float(b.abs().max()))
