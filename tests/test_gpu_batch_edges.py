"""GPU tests of the batch operators at edges of their contract: what a status says, where weights
and scores lose digits, and calls over several steps."""

import math
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

import batch_ref as R
from paper_2608_00814_gb300 import binding as B
from test_gpu_batch_ops import BF16, F16, F32, TYPES, attend, gen, inputs, randn, status

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _built():
    from paper_2608_00814_gb300 import _build
    _build.build()


# ------------------------------------------------------------------ weights

@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("prefix", [0, 2048])
@pytest.mark.parametrize("counts", [[1] * 40, [90, 200, 64, 140, 90, 200, 64, 140]])
def test_attention_returns_a_constant_v(dtype, kv, prefix, counts):
    """Where every key has the same v, out is that v: a row's weights, as they are multiplied, add up to the sum
    that it is divided by.  v is a power of two, below which half a step is smallest: 2^-9 of the value for bf16 and
    2^-12 for binary16.  Both sums are of the same positive numbers, at most `keys` of them and 64 in the joins, each
    rounded or truncated to 2^-23 of it, but few of them count: one key in 128 (16 of own keys with few rows) has a
    score 2^1 to 2^4 times, by row, the one before's and the others have none.  At most 64 count, so the sums are off
    by 2^-23 (64 + 64) < 2^-12, and nothing but the value itself may come out (bf16 weights of two halves are off by
    2^-16 at most besides)."""
    apart = 16 if counts[0] == 1 else 128
    step = R.Step(counts, [c + apart * (2 + i % 7) + 5 * i for i, c in enumerate(counts)], 16)
    q, pk, pv, kp, vp = inputs(step, prefix, 8, 2, 128, dtype, kv)
    q.zero_()
    q[..., 0] = 1 + 3 * torch.rand(step.rows, 8, generator=gen(1), device="cuda")      # powers of two per step
    q[..., 1] = 2.0 ** 12

    def ramp(n, apart):
        k = torch.zeros(n, 2, 128, device="cuda")
        i = torch.arange(n, device="cuda")
        k[..., 0] = (i // apart)[:, None]
        k[..., 1] = -1.0 * (i % apart != apart - 1)[:, None]
        return k.to(kv)

    pk[:prefix] = ramp(prefix, 128)
    for b, n in enumerate(step.lens):
        own = ramp(n, apart)
        if prefix:
            own[..., 1] = -1
        for s in range(n):
            kp[step.where(b, s)] = own[s]
    v = torch.tensor([1.0, -1.0, 2.0, 0.5], device="cuda", dtype=kv).repeat(32)
    pv[:prefix], vp[:] = v, v
    out, st = attend(step, q, pk, pv, prefix, kp, vp, scale=math.log(2))
    assert int(st) == 0
    if dtype is F32:      # rounded sums divided, without a type's rounding after it
        assert float((out / v - 1).abs().max()) <= 128 * 2.0 ** -23
    else:
        assert torch.equal(out, v.to(dtype).expand_as(out))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("far", [18.5, 20.5, 22.5])
@pytest.mark.parametrize("where", ["prefix", "own, few rows", "own, many rows"])
def test_attention_small_weights_of_binary16(dtype, far, where):
    """One key in 16 has all the weight but a v of zero; what comes out is the others', each 2^-far of it.  A weight
    is a binary16 number below the row's largest, which stands at 2^7 or above: half a step is 2^-11 of a weight, or
    2^-25 / 2^7 = 2^-32 of the largest where it is subnormal.  A score of `far` from two fp32 roundings is off by
    far 2^-23, the rest as in check_attention."""
    n = 2048
    i32 = dict(dtype=torch.int32, device="cuda")
    heavy = torch.arange(n, device="cuda") % 16 == 0
    k, v = torch.zeros(n, 2, 128, dtype=F16, device="cuda"), torch.full((n, 2, 128), 2.0 ** 14, dtype=F16, device="cuda")
    k[heavy, :, 0], v[heavy] = 16.0, 0.0
    seqs, rows = (5, 1) if where != "own, many rows" else (2, 100)
    q = torch.zeros(seqs * rows, 8, 128, dtype=dtype, device="cuda")
    q[:, :, 0] = 1
    scale = far * math.log(2) / 16
    q_start = torch.arange(seqs + 1, **i32) * rows
    pk = pv = None
    if where == "prefix":
        pk, pv, prefix = k, v, n
        # one own key of weight zero: -2^13 scale
        kp = torch.zeros(1, 16, 2, 128, dtype=F16, device="cuda")
        kp[..., 0] = -(2.0 ** 13)
        vp, lens = torch.zeros_like(kp), 1
    else:       # every sequence reads the same page; rows of the step see it whole but for their successors
        prefix = 0
        kp, vp, lens = k[None], v[None], n
    batch = B.Batch(q_start, torch.full((seqs,), lens, **i32), torch.zeros(seqs, 1, **i32), seqs * rows)
    cache, st, out = B.PagedCache(kp.contiguous(), vp.contiguous()), status(), torch.empty_like(q)
    ws = torch.empty(B.oos_shared_prefix_attention_workspace_bytes(q, prefix, cache, batch), dtype=torch.uint8, device="cuda")
    B.oos_shared_prefix_attention(q, pk, pv, prefix, cache, batch, None, scale, out, ws, st)
    assert int(st) == 0
    w = 2.0 ** -far
    seen = torch.full((seqs * rows,), n)
    if where != "prefix":
        seen = (n - rows + 1 + torch.arange(rows)).repeat(seqs)
    big = (seen + 15) // 16
    want = ((seen - big) * w * 2.0 ** 14 / (big + (seen - big) * w))[:, None, None].double()
    rel = R.U[dtype] + max(R.U[F16], 2.0 ** -32 / w) + far * 2.0 ** -23 + (4 * n + 64) * R.F32
    got = out.double().cpu()
    assert bool(((got - want).abs() <= rel * want).all()), float(((got - want).abs() / want).max() / rel)


@pytest.mark.parametrize("counts, heads", [([1] * 6, 8), ([3, 1, 2], 4), ([2, 7], 8)])
def test_attention_own_keys_in_two_bf16_halves(counts, heads):
    """Few rows over bf16 pages without a prefix: weights are multiplied as two bf16 halves, 2^-16 of a weight
    together, and not as one, 2^-8.  Other terms as in check_attention."""
    step = R.Step(counts, [c + 40 + i for i, c in enumerate(counts)], 16)
    q, pk, pv, kp, vp = inputs(step, 0, heads, 1, 128, BF16, BF16, std=0.1)
    out, st = attend(step, q, None, None, 0, kp, vp)
    assert int(st) == 0
    ref, mag, size = R.attention(step, q, pk[:0], pv[:0], kp, vp, 1 / math.sqrt(128))
    rel = 2.0 ** -16 + 2 * (131 * R.F32 * size + 4 * R.F32) + (4 * max(step.lens) + 64) * R.F32 + 256 * R.F32 * size
    tol = R.U[BF16] * ref.abs() + rel * mag
    assert bool(((out.double().cpu() - ref).abs() <= tol).all())
    # a bound that one bf16 half would not keep
    assert rel < 2.0 ** -12


# ------------------------------------------------------------------ scores that are not finite

@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("own", [1, 16, 17, 100])
def test_attention_nan_key_beside_a_long_prefix(dtype, kv, own):
    """Own keys that leave parts for a join with the prefix's: a NaN key that is seen makes its rows NaN, and only
    those, wherever among the own keys it is."""
    counts, victims = [1 + i % 2 for i in range(100)], (3, 40, 99)
    lens = [c + 4 * i % 400 for i, c in enumerate(counts)]
    for b in victims:
        lens[b] = max(own, counts[b])
    step = R.Step(counts, lens, 16)
    q, pk, pv, kp, vp = inputs(step, 20000, 8, 1, 128, dtype, kv)
    want = torch.zeros(step.n, dtype=torch.bool)
    for b, key in zip(victims, (0, lens[40] // 2, lens[99] - counts[99])):   # all rows of a sequence see its key
        p, e = step.where(b, min(key, lens[b] - counts[b]))
        kp[p, e, 0, 9] = math.nan
        want[step.q_start[b]:step.q_start[b + 1]] = True
    out, st = attend(step, q, pk, pv, 20000, kp, vp)
    assert int(st) == 0
    nan = torch.isnan(out).cpu()
    assert torch.equal(nan.all(-1).all(-1), want) and torch.equal(nan.any(-1).any(-1), want)


# ------------------------------------------------------------------ what a status says

@pytest.mark.parametrize("dtype, kv", TYPES)
def test_attention_bad_offsets_with_trees(dtype, kv):
    """Offsets out of range are a bad batch with a tree, too; more than 128 rows of a sequence with a tree are a
    bad tree."""
    good = R.Step([1, 2, 1], [40, 2, 30], 16)
    q, _, _, kp, vp = inputs(good, 0, 4, 2, 128, dtype, kv)
    parent = torch.tensor([-1, -1, 0, -1], dtype=torch.int32, device="cuda")
    base, st = attend(good, q, None, None, 0, kp, vp, parent=parent)
    assert int(st) == 0
    for starts in ([0, 1, 9, 4], [0, 1, 3, 5], [0, 1, 0, 4], [0, 1, -3, 4]):
        step = R.Step([1, 2, 1], [40, 2, 30], 16)
        step.q_start = starts
        for parents in (None, parent):
            out, st = attend(step, q, None, None, 0, kp, vp, parent=parents)
            assert int(st) == B.OOS_EBATCH, (starts, parents is None)
        if starts[2] != 0:      # there sequence 2, from row 0 on, claims sequence 0's row as well
            assert torch.equal(out[0], base[0])
    big = R.Step([129], [140], 16)
    q, _, _, kp, vp = inputs(big, 0, 4, 2, 128, dtype, kv)
    chain = torch.arange(-1, 128, dtype=torch.int32, device="cuda")
    _, st = attend(big, q, None, None, 0, kp, vp, parent=chain)
    assert int(st) == B.OOS_ETREE


@pytest.mark.parametrize("dtype, kv", TYPES)
@pytest.mark.parametrize("counts", [[1, 0, 2], [70, 0, 90]])
def test_attention_bad_length_of_a_waiting_sequence(dtype, kv, counts):
    """A sequence without rows in the step: its length is checked all the same, the others keep their results."""
    step = R.Step(counts, [counts[0] + 9, 5, counts[2]], 16)
    q, _, _, kp, vp = inputs(step, 0, 4, 2, 128, dtype, kv)
    base, st = attend(step, q, None, None, 0, kp, vp)
    assert int(st) == 0
    for n in (-1, -2 ** 31, 2 ** 31 - 1):
        step.lens[1] = n
        out, st = attend(step, q, None, None, 0, kp, vp)
        assert int(st) == B.OOS_EBATCH and torch.equal(out, base), n


def test_attention_row_with_one_key():
    """A length below the step's rows: the row that is left at position 0 sees that key alone, and gives its v."""
    for dtype, kv in TYPES:
        step = R.Step([1, 2, 1], [40, 2, 30], 16)
        q, _, _, kp, vp = inputs(step, 0, 4, 2, 128, dtype, kv)
        step.lens[1] = 1
        out, st = attend(step, q, None, None, 0, kp, vp)
        assert int(st) == B.OOS_EBATCH
        p, e = step.where(1, 0)
        assert torch.equal(out[2], vp[p, e].repeat_interleave(2, 0).to(dtype))
        assert bool((out[1] == 0).all())


# ------------------------------------------------------------------ how a call is cut up

@pytest.mark.parametrize("dtype, kv", TYPES[1:])
@pytest.mark.parametrize("n_seqs, rows, heads, prefix, own, tree, parts", [(1, 16, 8, 0, 1100, True, 4), (1, 16, 16, 1000, 1100, True, 8),
                                                                           (16, 33, 16, 9000, 1100, False, 6)])
def test_attention_many_rows_over_long_own_keys(dtype, kv, n_seqs, rows, heads, prefix, own, tree, parts):
    """Ranges of own keys as parts, with the prefix among them, and beside its parts of a launch of its own; `parts` is
    what a GPU of 152 SMs cuts the call into.  Lengths differ, down to sequences whose later ranges hold no key."""
    lens = [own - (own - rows) * i // n_seqs for i in range(n_seqs)]
    nkv = heads // 8
    step = R.Step([rows] * n_seqs, lens, 16, pad=1)
    rng = np.random.RandomState(1)
    parent = [-1 if j == 0 else int(rng.randint(-1, j)) for _ in range(n_seqs) for j in range(rows)] if tree else None
    q, pk, pv, kp, vp = inputs(step, prefix, heads, nkv, 128, dtype, kv)
    par = None if parent is None else torch.tensor(parent + [-1], dtype=torch.int32, device="cuda")
    size = B.oos_shared_prefix_attention_workspace_bytes(q, prefix, B.PagedCache(kp, vp), step.device(B))
    if torch.cuda.get_device_properties(0).multi_processor_count == 152:
        assert size // (step.rows * heads * 132 * 4) == parts
    out, st = attend(step, q, pk, pv, prefix, kp, vp, par)
    assert int(st) == 0
    ref, mag, top = R.attention(step, q, pk[:prefix], pv[:prefix], kp, vp, 1 / math.sqrt(128), parent)
    R.check_attention(out[:step.n], ref, mag, top, prefix + own, kv)
    assert bool((out[step.n:] == 7.0).all())
    again, _ = attend(step, q, pk, pv, prefix, kp, vp, par)
    assert torch.equal(out, again)


# ------------------------------------------------------------------ angles

@pytest.mark.parametrize("theta", [1e4, 5e5, 1e6])
@pytest.mark.parametrize("d", [128, 66])
def test_norm_rope_angles_against_exact_rates(theta, d):
    """Rates theta^(-2m/d) to 50 digits: the angle is off by at most 2^-55 of a turn per position, which moves a
    pair by 2 pi of that; the rest as in check_norm_rope."""
    turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937511")
    pos = [1, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31]
    angle = torch.zeros(len(pos), d // 2, dtype=torch.float64)
    with localcontext() as digits:
        digits.prec = 50
        for m in range(d // 2):
            rate = (Decimal(theta).ln() * Decimal(-2 * m) / Decimal(d)).exp() / turn
            for i, p in enumerate(pos):
                angle[i, m] = float((p * rate) % 1 * turn)
    x = randn(gen(3), len(pos), 2, d)
    y = torch.empty_like(x)
    B.oos_qk_norm_rope(x, None, None, None, 0.0, B.OosRopeConfig(theta), torch.tensor(pos, dtype=torch.int32, device="cuda"), y, None)
    c, s, xd, h = torch.cos(angle)[:, None], torch.sin(angle)[:, None], x.double().cpu(), d // 2
    ref = torch.cat((xd[..., :h] * c - xd[..., h:] * s, xd[..., h:] * c + xd[..., :h] * s), -1)
    r = torch.hypot(xd[..., :h], xd[..., h:]).repeat(1, 1, 2)
    far = torch.tensor(pos, dtype=torch.float64).abs()[:, None, None] * 2.0 ** -55 * 2 * math.pi
    tol = R.F32 * ref.abs() + (32 * R.F32 + far) * r
    assert bool(((y.double().cpu() - ref).abs() <= tol).all())


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("heads", [1 << 20, 1 << 22, 1 << 23])
def test_append_of_many_heads(heads):
    """As many heads of two elements as a call may have: all are appended."""
    k, v = randn(gen(1), 1, heads, 2, dtype=BF16), randn(gen(2), 1, heads, 2, dtype=BF16)
    kp = torch.full((2, 1, heads, 2), 7.0, dtype=BF16, device="cuda")
    vp = torch.full_like(kp, 7.0)
    i32 = dict(dtype=torch.int32, device="cuda")
    batch = B.Batch(torch.tensor([0, 1], **i32), torch.tensor([1], **i32), torch.tensor([[1]], **i32), 1)
    st = status()
    B.oos_paged_append(B.PagedCache(kp, vp), batch, k, v, None, 1e-6, None, None, st)
    assert int(st) == 0
    assert torch.equal(kp[1], k) and torch.equal(vp[1], v)
    assert bool((kp[0] == 7.0).all()) and bool((vp[0] == 7.0).all())


def test_append_of_a_length_below_every_row():
    """A length so far below zero that a row's position would wrap to a large one: left out and reported, also where
    the table reaches that far."""
    page = 1 << 30
    k, v = randn(gen(1), 2, 1, 2, dtype=BF16), randn(gen(2), 2, 1, 2, dtype=BF16)
    kp = torch.zeros(1, page, 1, 2, dtype=BF16, device="cuda")
    vp = torch.zeros_like(kp)
    i32 = dict(dtype=torch.int32, device="cuda")
    for n in (-2 ** 31, -2 ** 31 + 1, -1, 0):
        batch = B.Batch(torch.tensor([0, 2], **i32), torch.tensor([n], **i32), torch.tensor([[0, 0]], **i32), 2)
        st = status()
        B.oos_paged_append(B.PagedCache(kp, vp), batch, k, v, None, 1e-6, None, None, st)
        assert int(st) == B.OOS_EBATCH
        assert int(torch.count_nonzero(kp)) == 0 and int(torch.count_nonzero(vp)) == 0, n


# ------------------------------------------------------------------ sizes past 32 bits

def test_binding_refuses_sizes_past_32_bits():
    """The library takes sizes of 32 bits: a larger one is refused, not cut to what is left of it."""
    wide = 2 ** 32
    x = torch.ones(wide + 3, 1, 2, dtype=BF16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    for t in (x, x.view(1, wide + 3, 2), x.view(-1)[:wide + 4].view(1, 1, wide + 4)):
        with pytest.raises(B.OosError) as e:
            B.oos_qk_norm_rope(t, None, None, None, 1e-6, None, None, t, None)
        assert e.value.code == B.OOS_EINVAL
    assert int((x != 1).sum()) == 0
    for shape in ((wide + 1, 1, 1, 2), (1, wide + 1, 1, 2)):
        pages = x.view(-1)[:2 * (wide + 1)].view(shape)
        with pytest.raises(B.OosError) as e:
            B.PagedCache(pages, pages)
        assert e.value.code == B.OOS_EINVAL
    starts, lens, table = torch.tensor([0, 1], **i32), torch.tensor([1], **i32), torch.zeros(1, 1, **i32)
    for n in (wide + 1, 2 ** 31, -wide + 1):
        with pytest.raises(B.OosError) as e:
            B.Batch(starts, lens, table, n)
        assert e.value.code == B.OOS_EINVAL
    cache, batch = B.PagedCache(x[:16].view(1, 16, 1, 2), x[16:32].view(1, 16, 1, 2)), B.Batch(starts, lens, table, 1)
    q = torch.ones(1, 1, 2, dtype=BF16, device="cuda")
    ws, st, out = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), status(), torch.zeros_like(q)
    for prefix in (wide + 1, 2 ** 31, -wide + 1, -wide):
        with pytest.raises(B.OosError) as e:
            B.oos_shared_prefix_attention(q, x, x, prefix, cache, batch, None, 1.0, out, ws, st)
        assert e.value.code == B.OOS_EINVAL
        assert B.oos_shared_prefix_attention_workspace_bytes(q, prefix, cache, batch) == 0
    many = x[:wide].view(1, wide, 2)
    with pytest.raises(B.OosError):
        B.oos_shared_prefix_attention(many, None, None, 0, cache, batch, None, 1.0, many, ws, st)
    assert B.oos_shared_prefix_attention_workspace_bytes(many, 0, cache, batch) == 0


# ------------------------------------------------------------------ steps with trees

@pytest.mark.parametrize("dtype, kv", TYPES)
def test_steps_with_trees_follow_each_other(dtype, kv):
    """Three steps with trees.  After each, a path of every tree is accepted (none of one tree's) and its rows are
    appended again, where the next step takes committed positions to be: the rows of all steps see the accepted
    history and their own ancestors, as if K and V lay in order."""
    nq, nkv, d, page, prefix = 8, 2, 128, 16, 70
    g, rng, i32 = gen(4), np.random.RandomState(7), dict(dtype=torch.int32, device="cuda")
    pk, pv = [randn(g, prefix, nkv, d, dtype=kv) for _ in range(2)]
    gain, rope = 1 + randn(g, d, dtype=dtype, std=0.1), B.OosRopeConfig(1e6)
    held = [0, 5, 33]                                  # committed positions behind the prefix
    pool = R.Step([1] * 3, [128] * 3, page)
    kp, vp = [randn(g, pool.n_pages, page, nkv, d, dtype=kv) for _ in range(2)]
    hist = [[[t[pool.where(b, s)].clone() for s in range(n)] for b, n in enumerate(held)] for t in (kp, vp)]
    cache, st = B.PagedCache(kp, vp), status()

    def on_pool(counts, lens):
        step = R.Step(counts, lens, page)
        step.table, step.n_pages, step.width = pool.table, pool.n_pages, pool.width
        return step

    for t in range(3):
        counts = [int(c) for c in rng.randint(1, 30, 3)]
        trees = [[-1 if j == 0 else int(rng.randint(max(-1, j - 4), j)) for j in range(c)] for c in counts]
        depth = [R.ancestors(p).sum(1).tolist() for p in trees]
        step = on_pool(counts, [n + c for n, c in zip(held, counts)])
        pos = torch.tensor([prefix + held[b] + x - 1 for b in range(3) for x in depth[b]], **i32)
        rows = randn(g, step.n, nq + 2 * nkv, d, dtype=dtype)
        k, v = rows[:, nq:nq + nkv].contiguous(), rows[:, nq + nkv:].contiguous()
        q, out = [torch.empty(step.n, nq, d, dtype=dtype, device="cuda") for _ in range(2)]
        parent = [p for x in trees for p in x]
        batch = step.device(B)
        ws = torch.empty(B.oos_shared_prefix_attention_workspace_bytes(q, prefix, cache, batch), dtype=torch.uint8, device="cuda")
        B.oos_qk_norm_rope(rows[:, :nq], None, gain, None, 1e-6, rope, pos, q, None)
        B.oos_paged_append(cache, batch, k, v, gain, 1e-6, rope, pos, st)
        B.oos_shared_prefix_attention(q, pk, pv, prefix, cache, batch, torch.tensor(parent, **i32), 1 / math.sqrt(d), out, ws, st)
        assert int(st) == 0
        # the definition over pages in order: the history, then the step's K and V
        flat = R.Step(counts, step.lens, page)
        fk, fv = [torch.zeros(flat.n_pages, page, nkv, d, dtype=kv, device="cuda") for _ in range(2)]
        for f, h, src in ((fk, hist[0], kp), (fv, hist[1], vp)):
            for b in range(3):
                for s in range(step.lens[b]):
                    f[flat.where(b, s)] = h[b][s] if s < held[b] else src[step.where(b, s)]
        ref, mag, size = R.attention(flat, q, pk, pv, fk, fv, 1 / math.sqrt(d), parent)
        R.check_attention(out, ref, mag, size, prefix + max(step.lens), F32 if kv is F32 else kv, t)
        # accept a path of each tree, none of one
        path = []
        for b, p in enumerate(trees):
            j, nodes = int(rng.randint(len(p))) if b != t else -1, []
            while j >= 0:
                nodes.insert(0, j)
                j = p[j]
            path.append(nodes)
        for i, src in ((0, kp), (1, vp)):
            for b in range(3):
                hist[i][b] += [src[step.where(b, held[b] + j)].clone() for j in path[b]]
        taken = torch.tensor([step.q_start[b] + j for b in range(3) for j in path[b]], dtype=torch.long, device="cuda")
        held = [n + len(x) for n, x in zip(held, path)]
        again = on_pool([len(x) for x in path], held)
        B.oos_paged_append(cache, again.device(B), k[taken], v[taken], gain, 1e-6, rope, pos[taken], st)
        assert int(st) == 0
        for i, src in ((0, kp), (1, vp)):
            for b in range(3):
                assert all(torch.equal(src[pool.where(b, s)], hist[i][b][s]) for s in range(held[b])), (t, b)
