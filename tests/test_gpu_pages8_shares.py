"""GPU tests of attention over 8-bit pages where every warp takes an equal share of all keys: tables of more than
1024 positions, up to 256 sequences of few rows.  Against the 64-bit restatement (pages8_ref.py)."""

import math
import random

import pytest
import torch

import batch_ref as R
import pages8_ref as R8
import test_gpu_pages8 as T
from paper_2608_00814_gb300 import binding as B
from test_gpu_batch_ops import BF16, F16, TYPES, gen, randn, status

pytestmark = pytest.mark.gpu
HALVES = TYPES[1:]


@pytest.fixture(autouse=True)
def _built():
    from paper_2608_00814_gb300 import _build
    _build.build()


def lengths(seed, counts, most):
    rng = random.Random(seed)
    return [c + int(most * rng.random() ** 3) if c else rng.randint(0, 40) for c in counts]


MANY = [0 if i % 7 == 3 else 1 for i in range(100)]
SOME = [(i * 5) % 4 + (i % 6 == 0) for i in range(30)]


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("counts, most, page, nq, nkv, prefix", [
    (MANY, 2500, 16, 8, 2, 0), (MANY, 2500, 48, 4, 4, 700), (SOME, 3000, 32, 16, 4, 0), (SOME, 3000, 16, 12, 2, 333),
    ([16, 9, 16, 12], 4000, 64, 8, 2, 60), ([1], 3000, 256, 6, 6, 0), ([0, 0, 1], 1500, 16, 2, 2, 1)])
def test_shares(dtype, kv, counts, most, page, nq, nkv, prefix):
    """Sequences of no and of many keys, waiting ones among them, tiles of 8 and of 16 rows, several tiles of one
    sequence; rows behind the last are left as they were."""
    lens = lengths(len(counts), counts, most)
    lens[-1] = max(lens[-1], 1100)
    T.run_case8(counts, lens, page, 3, prefix, nq, nkv, 128, dtype, kv, seed=5)


@pytest.mark.parametrize("counts, lens, nq, nkv", [([1, 1], [1100, 30], 460, 460), ([1, 0, 1], [2000, 7, 70], 64, 1),
                                                   ([1, 2], [1030, 500], 48, 3)])
def test_more_heads_than_blocks_and_wide_groups(counts, lens, nq, nkv):
    """A block for each kv head where there are more of them than the chip holds blocks; groups of several tiles."""
    T.run_case8(counts, lens, 16, 1, 40, nq, nkv, 128, BF16, BF16)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("n", [256, 257])
def test_as_many_sequences_as_the_table_holds(dtype, kv, n):
    counts = [1] * n
    lens = [1 + 3 * (i % 50) for i in range(n)]
    lens[n // 2], lens[-1] = 1300, 1
    T.run_case8(counts, lens, 16, 1, 20, 4, 2, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", HALVES)
def test_one_sequence_of_more_keys_than_places(dtype, kv):
    """40000 keys of one kv head: shares are as large as keeps a row's sums to some 256."""
    T.run_case8([1], [40000], 256, 0, 0, 4, 1, 128, dtype, kv, std=0.5)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("counts, lens, nq", [([100, 3, 5, 1], [1300, 3, 1500, 900], 2), ([6, 2, 9, 1], [1400, 2, 2000, 33], 8)])
def test_trees(dtype, kv, counts, lens, nq):
    """A chain, a bush, roots alone; nodes among and behind a long committed past."""
    shapes = [lambda j: j - 1, lambda j: -1 if j == 0 else (j - 1) // 2, lambda j: max(-1, j - 3), lambda j: -1]
    parent = [f(j) for c, f in zip(counts, shapes) for j in range(c)]
    T.run_case8(counts, lens, 16, 2, 90, nq, 2, 128, dtype, kv, parent=parent)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("rows", [2, 60])
def test_bad_batches_are_reported(dtype, kv, rows, monkeypatch):
    step = R.Step
    monkeypatch.setattr(R, "Step", lambda *a, **k: step(*a, **dict(k, width=70)))
    T.test_attention8_reports_bad_batches(dtype, kv, rows)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("tree", [False, True])
def test_masked_places_hold_anything(dtype, kv, tree, monkeypatch):
    step = R.Step
    monkeypatch.setattr(R, "Step", lambda *a, **k: step(*a, **dict(k, width=70)))
    T.test_attention8_masked_places_hold_anything(dtype, kv, tree, [3, 1, 9, 5], [3, 20, 200, 31], (2, 4, 3))


def test_offsets_out_of_order_stay_within_the_workspace():
    """The same rows claimed by several sequences: reported, and nothing is written outside out's rows and the
    workspace (its end and what lies behind it are looked at)."""
    step = R.Step([1] * 6, [1200] * 6, 16)
    q, _, _, cache = T.inputs8(step, 0, 8, 2, 128, BF16, BF16)
    n = B.oos_shared_prefix_attention8_workspace_bytes(q, 0, cache, step.device(B))
    room = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    step.q_start = [0, 6, 0, 6, 0, 6, 6]
    out, st = T.attend8(step, q, None, None, 0, cache, ws=room)
    assert int(st) == B.OOS_EBATCH and bool((room[n:] == 77).all())


@pytest.mark.parametrize("dtype, kv", HALVES)
def test_values_of_any_scale_beside_each_other(dtype, kv):
    """Blocks of zeros and of the smallest scale beside large ones: the weights of the zeros count in full."""
    step = R.Step([1, 2], [1300, 1100], 16)
    q, _, _, cache = T.inputs8(step, 0, 4, 2, 128, dtype, kv, std=0.3)
    flat_v, flat_s = cache.v.view(torch.uint8).view(-1, 16, 2, 128), cache.v_scale.view(-1, 2)
    flat_v[::2], flat_s[::2] = 0, 127 - 117
    flat_s[1::2] = 127 + (6 if dtype is F16 else 40)
    out, st = T.attend8(step, q, None, None, 0, cache)
    ref = R8.attention(step, q, torch.zeros(0, 2, 128, dtype=kv, device="cuda"), torch.zeros(0, 2, 128, dtype=kv, device="cuda"),
                       cache, 1 / math.sqrt(128))
    assert int(st) == 0
    R8.check_attention(out, *ref, 1300)


def test_a_graph_follows_the_lengths():
    """A captured call, replayed after the lengths, the offsets and the table have changed; and two graphs that share
    one workspace, one after the other."""
    nq, nkv, page, width = 8, 2, 16, 100
    sets = []
    for seed, (counts, lens) in enumerate([([1, 2, 1, 0], [1500, 2, 40, 3]), ([0, 1, 1, 2], [5, 1600, 333, 1000])]):
        step = R.Step(counts, lens, page, seed=seed, width=width)
        step.n_pages = 220
        sets.append(step)
    g = gen(4)
    x = T.pool(g, 220, page, nkv, 128, lo=-8, hi=-4)
    cache = B.PagedCache8(*x)
    q = randn(g, 4, nq, 128, dtype=BF16)
    want = [T.attend8(s, q, None, None, 0, cache)[0] for s in sets]
    batch, st, out = sets[0].device(B), status(), [torch.zeros_like(q) for _ in range(2)]
    ws = torch.empty(B.oos_shared_prefix_attention8_workspace_bytes(q, 0, cache, batch), dtype=torch.uint8, device="cuda")
    graphs = []
    for o in out:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.oos_shared_prefix_attention8(q, None, None, 0, cache, batch, None, 1 / math.sqrt(128), o, ws, st)
        graphs.append(graph)
    for i in (0, 1, 0):
        other = sets[i].device(B)
        batch.q_start.copy_(other.q_start)
        batch.seq_len.copy_(other.seq_len)
        batch.block_table.copy_(other.block_table)
        for graph, o in zip(graphs, out):
            o.fill_(5.0)
            graph.replay()
        torch.cuda.synchronize()
        assert int(st) == 0 and all(torch.equal(o, want[i]) for o in out)


def test_two_calls_at_once():
    step = R.Step([1] * 20, list(range(1, 2000, 100)), 16)
    sets = [T.inputs8(step, 900, 8, 2, 128, BF16, BF16, seed=s) for s in (1, 2)]
    want = [T.attend8(step, *(s[:3]), 900, s[3])[0] for s in sets]
    torch.cuda.synchronize()
    streams, batch, st = [torch.cuda.Stream() for _ in sets], step.device(B), status()
    ws = [torch.empty(B.oos_shared_prefix_attention8_workspace_bytes(s[0], 900, s[3], batch), dtype=torch.uint8, device="cuda")
          for s in sets]
    outs = [torch.empty_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(sets):
            B.oos_shared_prefix_attention8(s[0], s[1], s[2], 900, s[3], batch, None, 1 / math.sqrt(128), outs[i], ws[i], st,
                                           stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want)) and int(st) == 0


@pytest.mark.parametrize("dtype, kv", HALVES)
def test_repeats_bit_for_bit(dtype, kv):
    """Passes over cold and warm caches, next to another stream's traffic."""
    counts = [1, 3, 1, 0, 2] * 8
    step = R.Step(counts, lengths(3, counts, 2500), 16, seed=7, width=200)
    q, pk, pv, cache = T.inputs8(step, 500, 8, 2, 128, dtype, kv)
    base, st = T.attend8(step, q, pk, pv, 500, cache)
    flush, side = torch.empty(1 << 28, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    for i in range(12):
        flush.fill_(i)
        if i >= 6:
            with torch.cuda.stream(side):
                flush[:1 << 27].copy_(flush[1 << 27:])
        assert torch.equal(base, T.attend8(step, q, pk, pv, 500, cache)[0])
        side.synchronize()
    assert int(st) == 0


def test_calls_over_pages_of_both_kinds_in_turn():
    """A call over 16-bit pages right behind one over 8-bit pages takes nothing of its plan."""
    step = R.Step([1, 1, 2], [1200, 30, 500], 16)
    q, pk, pv, cache = T.inputs8(step, 70, 8, 2, 128, BF16, BF16)
    k, v = [torch.nan_to_num(t).to(BF16) for t in cache.dequantized()]
    pages, batch, st = B.PagedCache(k, v), step.device(B), status()
    ws = torch.empty(B.oos_shared_prefix_attention_workspace_bytes(q, 70, pages, batch), dtype=torch.uint8, device="cuda")

    def wide():
        out = torch.zeros_like(q)
        B.oos_shared_prefix_attention(q, pk, pv, 70, pages, batch, None, 1 / math.sqrt(128), out, ws, st)
        return out
    base, base8 = wide(), T.attend8(step, q, pk, pv, 70, cache)[0]
    for _ in range(3):
        assert torch.equal(T.attend8(step, q, pk, pv, 70, cache)[0], base8)
        assert torch.equal(wide(), base)
    assert int(st) == 0
    R.check_attention(base, *R.attention(step, q, pk[:70], pv[:70], k, v, 1 / math.sqrt(128)), 1270, BF16)
