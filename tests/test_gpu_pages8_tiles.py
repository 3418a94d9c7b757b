"""GPU tests of attention over 8-bit pages in sequences of many rows: more than 128 (token, head of a group) on average,
and tables of more than 1024 positions.  Against the 64-bit restatement (pages8_ref.py)."""

import math

import pytest
import torch

import batch_ref as R
import test_gpu_pages8 as T
from paper_2608_00814_gb300 import binding as B
from test_gpu_batch_ops import BF16, TYPES

pytestmark = pytest.mark.gpu
HALVES = TYPES[1:]


@pytest.fixture(autouse=True)
def _wide(monkeypatch):
    from paper_2608_00814_gb300 import _build
    _build.build()
    step = R.Step

    def wide(counts, lens, page, *a, **k):
        k["width"] = k.get("width") or max(1100 // page + 1, *[(n + page - 1) // page for n in lens])
        return step(counts, lens, page, *a, **k)
    monkeypatch.setattr(R, "Step", wide)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("page", [16, 48, 256])
@pytest.mark.parametrize("prefix", [0, 129, 1000])
def test_ragged(dtype, kv, page, prefix):
    T.run_case8([0, 150, 97, 1, 60], [3, 150, 300, 1, 475], page, 3, prefix, 10, 2, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("prefix", [0, 77])
def test_trees(dtype, kv, prefix):
    """A chain, a forest, bushes of 1 to 128 nodes, behind no and many committed positions."""
    counts = [128, 1, 100, 77]
    shapes = [lambda j: j - 1, lambda j: -1, lambda j: max(-1, j - 3), lambda j: -1 if j == 0 else (j - 1) // 2]
    parent = [f(j) for c, f in zip(counts, shapes) for j in range(c)]
    T.run_case8(counts, [128, 60, 213, 500], 16, 1, prefix, 8, 2, 128, dtype, kv, parent=parent)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("counts, lens, nq", [([60, 200], [3000, 700], 8), ([200], [4100], 2), ([129], [129], 2), ([1], [2500], 300)])
def test_long_sequences(dtype, kv, counts, lens, nq):
    T.run_case8(counts, lens, 64, 0, 33, nq, 2, 128, dtype, kv)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("lo, hi", [(-117, -100), (-60, 30), (100, 119)])
def test_scales_of_any_size(dtype, kv, lo, hi):
    T.test_attention8_scales_of_any_size(dtype, kv, [90, 140], [200, 300], lo, hi)


@pytest.mark.parametrize("dtype, kv", HALVES)
def test_rows_any_stride(dtype, kv):
    T.test_attention8_rows_any_stride(dtype, kv, [70, 130], [90, 150])


@pytest.mark.parametrize("dtype, kv", HALVES)
def test_large_and_special_scores(dtype, kv):
    T.test_attention8_large_and_special_scores(dtype, kv, 250)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("tree", [False, True])
def test_masked_places_hold_anything(dtype, kv, tree):
    T.test_attention8_masked_places_hold_anything(dtype, kv, tree, [3, 1, 128, 100], [3, 20, 260, 101], (2, 40, 7))


@pytest.mark.parametrize("dtype, kv", HALVES)
def test_queries_of_any_size(dtype, kv):
    T.test_attention8_queries_of_any_size(dtype, kv, [130, 1, 128])


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("shape", ["ragged", "tree"])
def test_repeats_bit_for_bit(dtype, kv, shape):
    T.test_attention8_repeats_bit_for_bit(dtype, kv, shape)


@pytest.mark.parametrize("dtype, kv", HALVES)
@pytest.mark.parametrize("n", [3, 70])
def test_bad_batches_are_reported(dtype, kv, n):
    """A page outside the pool, lengths below the rows or past the table, offsets out of order, a malformed parent and
    more rows than a tree may have; other sequences keep their bits.  In a step of few sequences, whose tiles are dealt
    by length, and of many."""
    nq, nkv, rows = 4, 2, 100
    counts, lens = [rows] * n, [rows + 40] * n
    good = R.Step(counts, lens, 16)
    q, _, _, cache = T.inputs8(good, 0, nq, nkv, 128, dtype, kv)
    base, st = T.attend8(good, q, None, None, 0, cache)
    assert int(st) == 0
    first, last = slice(0, rows), slice((n - 1) * rows, n * rows)
    for what in ("page", "negative page", "length", "width", "lowest"):
        step = R.Step(counts, lens, 16)
        if "page" in what:
            step.table[1][2] = -1 if "neg" in what else step.n_pages
        else:
            step.lens[1] = {"length": rows - 1, "width": 10 ** 6, "lowest": -2 ** 31}[what]
            if what == "width":
                step.table[1] = [0 if p < 0 else p for p in step.table[1]]
        out, st = T.attend8(step, q, None, None, 0, cache)
        assert int(st) == B.OOS_EBATCH, what
        assert torch.equal(out[first], base[first]) and torch.equal(out[last], base[last]), what
        if what == "length":
            assert bool((out[rows] == 0).all())      # the first row would be position -1
        if what == "lowest":
            assert bool((out[rows:2 * rows] == 0).all())
    step = R.Step(counts, lens, 16)
    step.q_start[2] = 99 if n == 3 else -5
    out, st = T.attend8(step, q, None, None, 0, cache)
    assert int(st) == B.OOS_EBATCH and torch.equal(out[first], base[first])
    roots = [-1] * (rows * n)
    for at, to in ((rows + 4, 4), (rows + 4, -2)):
        bad, fine = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in (roots[:at] + [to] + roots[at + 1:], roots)]
        out, st = T.attend8(good, q, None, None, 0, cache, parent=bad)
        ref, st2 = T.attend8(good, q, None, None, 0, cache, parent=fine)
        assert int(st) == B.OOS_ETREE and int(st2) == 0 and torch.equal(out, ref)
    many = R.Step([129] + counts[1:], [140] + lens[1:], 16)
    q2, _, _, cache2 = T.inputs8(many, 0, nq, nkv, 128, dtype, kv)
    parents = torch.tensor([-1] * many.rows, dtype=torch.int32, device="cuda")
    out, st = T.attend8(many, q2, None, None, 0, cache2, parent=parents)
    assert int(st) == B.OOS_ETREE and not bool(torch.isnan(out[129:many.n]).any())      # the first's rows are not valid


def test_two_graphs_share_a_workspace():
    """Captured calls on one workspace, replayed in turn after lengths have changed."""
    step = R.Step([150, 60, 90], [300, 60, 700], 16)
    q, pk, pv, cache = T.inputs8(step, 300, 8, 2, 128, BF16, BF16)
    other = R.Step([150, 60, 90], [200, 60, 690], 16)
    other.table = step.table
    want = [T.attend8(s, q, pk, pv, 300, cache)[0] for s in (step, other)]
    batch, st, outs, graphs = step.device(B), T.status(), [torch.zeros_like(q) for _ in range(2)], []
    ws = torch.empty(B.oos_shared_prefix_attention8_workspace_bytes(q, 300, cache, batch), dtype=torch.uint8, device="cuda")
    for o in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.oos_shared_prefix_attention8(q, pk, pv, 300, cache, batch, None, 1 / math.sqrt(128), o, ws, st)
        graphs.append(graph)
    for i in (0, 1, 0):
        batch.seq_len.copy_((step, other)[i].device(B).seq_len)
        for graph, o in zip(graphs, outs):
            o.fill_(5.0)
            graph.replay()
        torch.cuda.synchronize()
        assert int(st) == 0 and all(torch.equal(o, want[i]) for o in outs)
