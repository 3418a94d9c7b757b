"""What the operators on 8-bit pages, and on pages between steps, refuse on the host (no GPU)."""

import ctypes

import pytest
import torch

from paper_2608_00814_gb300 import binding as B
from test_batch_refusals import BAD_BATCHES, L, NULL, P, batch, cache, rope  # noqa: F401


def cache8(nkv=2, d=128, page=16, n_pages=4, k=P, v=P, ks=P, vs=P):
    return B.OosPagedCache8(nkv, d, page, n_pages, k, v, ks, vs)


BAD8 = [dict(nkv=0), dict(page=0), dict(page=24), dict(n_pages=0), dict(k=NULL), dict(v=NULL), dict(ks=NULL), dict(vs=NULL)]


def append8(L, c=None, b=None, dtype=B.OOS_DTYPE_BF16, k=P, ks=256, v=P, vs=256, eps=1e-6, r=None, positions=P, status=P):
    c, b, r = c or cache8(), b or batch(), r or rope()
    return L.oos_paged_append8(ctypes.byref(c), ctypes.byref(b), dtype, k, ks, v, vs, NULL, eps, ctypes.byref(r),
                               positions, status, NULL)


@pytest.mark.parametrize("bad", [dict(k=NULL), dict(v=NULL), dict(ks=255), dict(vs=255), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(r=rope(theta=-1.0)), dict(positions=NULL), dict(status=NULL),
                                 dict(c=cache8(nkv=65536, d=2), ks=1 << 20, vs=1 << 20),
                                 dict(b=batch(n_seqs=1 << 30))] +
                         [dict(c=cache8(**x)) for x in BAD8] + [dict(b=batch(**x)) for x in BAD_BATCHES])
def test_append8_invalid(L, bad):
    assert append8(L, **bad) == B.OOS_EINVAL


@pytest.mark.parametrize("bad", [dict(dtype=7), dict(dtype=-1), dict(c=cache8(d=129)), dict(c=cache8(d=256)), dict(c=cache8(d=0))])
def test_append8_unsupported(L, bad):
    assert append8(L, **bad) == B.OOS_EUNSUPPORTED


def attention8(L, c=None, b=None, dtype=B.OOS_DTYPE_BF16, nq=4, q=P, qs=512, pt=B.OOS_DTYPE_BF16, pk=P, pv=P, prefix=5,
               scale=0.1, out=P, os_=512, ws=P, ws_bytes=1 << 30, status=P):
    c, b = c or cache8(), b or batch()
    return L.oos_shared_prefix_attention8(dtype, nq, q, qs, pt, pk, pv, prefix, ctypes.byref(c), ctypes.byref(b), NULL,
                                          scale, out, os_, ws, ws_bytes, status, NULL)


@pytest.mark.parametrize("bad", [dict(nq=0), dict(nq=5), dict(prefix=-1), dict(prefix=2 ** 31 - 1), dict(pk=NULL),
                                 dict(pv=NULL), dict(q=NULL), dict(out=NULL), dict(qs=511), dict(os_=511),
                                 dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(status=NULL), dict(pk=P + 8), dict(pv=P + 2), dict(c=cache8(k=P + 8)),
                                 dict(c=cache8(v=P + 1)), dict(b=batch(n_tokens=1 << 30))] +
                         [dict(c=cache8(**x)) for x in BAD8] + [dict(b=batch(**x)) for x in BAD_BATCHES])
def test_attention8_invalid(L, bad):
    assert attention8(L, **bad) == B.OOS_EINVAL


@pytest.mark.parametrize("dtype, prefix", [(B.OOS_DTYPE_F32, B.OOS_DTYPE_BF16), (B.OOS_DTYPE_BF16, B.OOS_DTYPE_F32),
                                           (B.OOS_DTYPE_F16, B.OOS_DTYPE_BF16), (9, 9), (B.OOS_DTYPE_BF16, -1)])
def test_attention8_unsupported_types(L, dtype, prefix):
    assert attention8(L, dtype=dtype, pt=prefix) == B.OOS_EUNSUPPORTED


def test_attention8_unsupported_head(L):
    for d in (0, 1, 63, 130):
        assert attention8(L, c=cache8(d=d)) == B.OOS_EUNSUPPORTED


def test_workspace8_of_a_bad_shape_is_zero(L):
    f = L.oos_shared_prefix_attention8_workspace_bytes
    good = cache8(), batch()
    t = B.OOS_DTYPE_BF16
    assert f(t, 5, 10, ctypes.byref(good[0]), ctypes.byref(good[1])) == 0
    assert f(t, 4, -1, ctypes.byref(good[0]), ctypes.byref(good[1])) == 0
    assert f(9, 4, 10, ctypes.byref(good[0]), ctypes.byref(good[1])) == 0
    assert f(t, 4, 10, None, ctypes.byref(good[1])) == 0
    assert f(t, 4, 10, ctypes.byref(good[0]), None) == 0
    for x in (dict(d=200), dict(page=24), dict(page=0)):
        assert f(t, 4, 10, ctypes.byref(cache8(**x)), ctypes.byref(good[1])) == 0


def layers(kind, n=3, **other):
    """n layers, the last one with other fields."""
    make = cache8 if kind == 8 else cache
    return (B.OosPagedCache8 if kind == 8 else B.OosPagedCache) * n, [make() for _ in range(n - 1)] + [make(**other)]


def compact(L, kind, n=3, b=None, nodes=P, length=P, new=P, status=P, none=False, **other):
    t, c = layers(kind, max(n, 1) if n < 2000 else 1, **other)
    f = L.oos_paged_compact8 if kind == 8 else L.oos_paged_compact
    return f(NULL if none else t(*c), n, ctypes.byref(b or batch()), nodes, length, new, status, NULL)


OTHER = [dict(nkv=3), dict(d=64), dict(page=32), dict(n_pages=5), dict(k=NULL), dict(v=NULL)]


@pytest.mark.parametrize("kind", [8, 16])
@pytest.mark.parametrize("bad", [dict(n=0), dict(n=-1), dict(n=1 << 20), dict(none=True), dict(nodes=NULL), dict(length=NULL),
                                 dict(new=NULL), dict(status=NULL)] + OTHER + [dict(b=batch(**x)) for x in BAD_BATCHES])
def test_compact_invalid(L, kind, bad):
    assert compact(L, kind, **bad) == B.OOS_EINVAL


def copy(L, kind, n_layers=3, n=2, src=P, dst=P, status=P, none=False, **other):
    t, c = layers(kind, max(n_layers, 1) if n_layers < 2000 else 1, **other)
    f = L.oos_pages_copy8 if kind == 8 else L.oos_pages_copy
    return f(NULL if none else t(*c), n_layers, src, dst, n, status, NULL)


@pytest.mark.parametrize("kind", [8, 16])
@pytest.mark.parametrize("bad", [dict(n_layers=0), dict(n_layers=1025), dict(none=True), dict(n=-1), dict(n=(1 << 20) + 1),
                                 dict(src=NULL), dict(dst=NULL), dict(status=NULL)] + OTHER)
def test_copy_invalid(L, kind, bad):
    assert copy(L, kind, **bad) == B.OOS_EINVAL


def test_layers_unsupported(L):
    for f in (compact, copy):
        assert f(L, 16, dtype=B.OOS_DTYPE_F32) == B.OOS_EINVAL       # the last layer's differs
        assert f(L, 16, 1, dtype=9) == B.OOS_EUNSUPPORTED
        assert f(L, 16, 1, d=256) == B.OOS_EUNSUPPORTED
        assert f(L, 8, 1, d=7) == B.OOS_EUNSUPPORTED
        assert f(L, 8, 1, page=24) == B.OOS_EINVAL


def test_no_rows_or_pairs_is_no_work(L):
    assert append8(L, b=batch(n_tokens=0), k=NULL, v=NULL) == B.OOS_OK
    assert attention8(L, b=batch(n_tokens=0), q=NULL, out=NULL, ws=NULL, ws_bytes=0) == B.OOS_OK
    for kind in (8, 16):
        assert copy(L, kind, n=0, src=NULL, dst=NULL) == B.OOS_OK


def test_binding_refuses_other_tensors():
    t = torch.zeros(2, 16, 2, 128, dtype=torch.uint8).view(torch.float8_e4m3fn)      # not on a GPU
    s = torch.zeros(2, 1, 2, dtype=torch.uint8)
    for args in ((t, t, s, s), (t.float(), t.float(), s, s), (t[0], t[0], s, s)):
        with pytest.raises(B.OosError):
            B.PagedCache8(*args)
    with pytest.raises(B.OosError):
        B.PagedLayers([])
    with pytest.raises(B.OosError):
        B.PagedLayers([t])
    with pytest.raises(B.OosError):
        B.PagedCache8.empty(4, 24, 2, 128, device="cpu")
