"""What the batch operators refuse on the host, before anything is enqueued (no GPU)."""

import ctypes

import pytest
import torch

from paper_2608_00814_gb300 import _build
from paper_2608_00814_gb300 import binding as B

P = 0x1000      # an address that no call may touch: every call here is refused
NULL = None


@pytest.fixture(scope="module")
def L():
    _build.build()
    return B.lib()


def rope(theta=1e6, factor=0.0, lo=1.0, hi=4.0, orig=8192):
    return B.OosRopeConfig(theta, factor, lo, hi, orig)


def cache(dtype=B.OOS_DTYPE_BF16, nkv=2, d=128, page=16, n_pages=4, k=P, v=P):
    return B.OosPagedCache(dtype, nkv, d, page, n_pages, k, v)


def batch(n_seqs=2, n_tokens=3, width=4, q_start=P, seq_len=P, table=P):
    return B.OosBatch(n_seqs, n_tokens, width, q_start, seq_len, table)


def test_new_status_has_a_text():
    assert B.oos_status_string(B.OOS_EBATCH) != "unknown status"


def norm_rope(L, dtype=B.OOS_DTYPE_BF16, n=3, nq=4, nkv=2, d=128, q=P, qs=512, k=P, ks=256, eps=1e-6, r=None,
              positions=P, qo=P, qos=512, ko=P, kos=256):
    r = rope() if r is None else r
    return L.oos_qk_norm_rope(dtype, n, nq, nkv, d, q, qs, k, ks, NULL, NULL, eps, r and ctypes.byref(r), positions,
                              qo, qos, ko, kos, NULL)


@pytest.mark.parametrize("bad", [dict(n=-1), dict(nq=-1), dict(nq=0, nkv=0), dict(q=NULL), dict(qo=NULL), dict(k=NULL),
                                 dict(ko=NULL), dict(qs=511), dict(ks=255), dict(qos=511), dict(kos=0),
                                 dict(eps=-1e-6), dict(eps=float("nan")), dict(positions=NULL),
                                 dict(r=rope(theta=0.0)), dict(r=rope(theta=float("nan"))),
                                 dict(r=rope(factor=float("nan"))), dict(r=rope(factor=8.0, lo=4.0)),
                                 dict(r=rope(factor=8.0, lo=0.0)), dict(r=rope(factor=8.0, orig=0))])
def test_norm_rope_invalid(L, bad):
    assert norm_rope(L, **bad) == B.OOS_EINVAL


@pytest.mark.parametrize("bad", [dict(dtype=-1), dict(dtype=3), dict(d=0), dict(d=127), dict(d=130)])
def test_norm_rope_unsupported(L, bad):
    assert norm_rope(L, **bad) == B.OOS_EUNSUPPORTED


def test_no_rows_is_no_work(L):
    assert norm_rope(L, n=0, q=NULL, k=NULL, qo=NULL, ko=NULL, positions=NULL) == B.OOS_OK
    c, b = cache(), batch(n_tokens=0)
    assert L.oos_paged_append(ctypes.byref(c), ctypes.byref(b), B.OOS_DTYPE_BF16, NULL, 0, NULL, 0, NULL, 1e-6, None,
                              NULL, P, NULL) == B.OOS_OK
    assert attention(L, b=b, q=NULL, out=NULL, ws=NULL, ws_bytes=0) == B.OOS_OK


def append(L, c=None, b=None, dtype=B.OOS_DTYPE_BF16, k=P, ks=256, v=P, vs=256, eps=1e-6, r=None, positions=P, status=P):
    c, b, r = c or cache(), b or batch(), r or rope()
    return L.oos_paged_append(ctypes.byref(c), ctypes.byref(b), dtype, k, ks, v, vs, NULL, eps, ctypes.byref(r),
                              positions, status, NULL)


BAD_CACHES = [dict(nkv=0), dict(page=0), dict(n_pages=0), dict(k=NULL), dict(v=NULL)]
BAD_BATCHES = [dict(n_seqs=0), dict(n_seqs=2 ** 31 - 1), dict(n_tokens=-1), dict(width=0), dict(q_start=NULL), dict(seq_len=NULL), dict(table=NULL)]


@pytest.mark.parametrize("bad", [dict(k=NULL), dict(v=NULL), dict(ks=255), dict(vs=255), dict(eps=-1.0),
                                 dict(r=rope(theta=-1.0)), dict(positions=NULL), dict(status=NULL)] +
                         [dict(c=cache(**x)) for x in BAD_CACHES] + [dict(b=batch(**x)) for x in BAD_BATCHES])
def test_append_invalid(L, bad):
    assert append(L, **bad) == B.OOS_EINVAL


@pytest.mark.parametrize("bad", [dict(dtype=7), dict(c=cache(dtype=3)), dict(c=cache(d=129)), dict(c=cache(d=256))])
def test_append_unsupported(L, bad):
    assert append(L, **bad) == B.OOS_EUNSUPPORTED


def attention(L, c=None, b=None, dtype=B.OOS_DTYPE_BF16, nq=4, q=P, qs=512, pk=P, pv=P, prefix=5, scale=0.1, out=P,
              os_=512, ws=P, ws_bytes=1 << 30, status=P):
    c, b = c or cache(), b or batch()
    return L.oos_shared_prefix_attention(dtype, nq, q, qs, pk, pv, prefix, ctypes.byref(c), ctypes.byref(b), NULL, scale,
                                         out, os_, ws, ws_bytes, status, NULL)


@pytest.mark.parametrize("bad", [dict(nq=0), dict(nq=5), dict(prefix=-1), dict(prefix=2 ** 31 - 1), dict(pk=NULL), dict(pv=NULL), dict(q=NULL),
                                 dict(out=NULL), dict(qs=511), dict(os_=511), dict(scale=0.0), dict(scale=-1.0),
                                 dict(scale=float("nan")), dict(scale=float("inf")), dict(status=NULL),
                                 dict(pk=P + 8), dict(pv=P + 2), dict(c=cache(k=P + 8)), dict(c=cache(v=P + 4)),
                                 dict(b=batch(n_tokens=1 << 30))] +
                         [dict(c=cache(**x)) for x in BAD_CACHES] + [dict(b=batch(**x)) for x in BAD_BATCHES])
def test_attention_invalid(L, bad):
    assert attention(L, **bad) == B.OOS_EINVAL


@pytest.mark.parametrize("dtype, kv", [(B.OOS_DTYPE_F32, B.OOS_DTYPE_BF16), (B.OOS_DTYPE_BF16, B.OOS_DTYPE_F32),
                                       (B.OOS_DTYPE_F16, B.OOS_DTYPE_BF16), (B.OOS_DTYPE_F32, B.OOS_DTYPE_F16),
                                       (9, B.OOS_DTYPE_BF16), (B.OOS_DTYPE_BF16, -1)])
def test_attention_unsupported_types(L, dtype, kv):
    assert attention(L, dtype=dtype, c=cache(dtype=kv)) == B.OOS_EUNSUPPORTED


def test_attention_unsupported_head(L):
    for d in (0, 1, 63, 130):
        assert attention(L, c=cache(d=d)) == B.OOS_EUNSUPPORTED


def test_workspace_of_a_bad_shape_is_zero(L):
    f = L.oos_shared_prefix_attention_workspace_bytes
    good = cache(), batch()
    assert f(5, 10, ctypes.byref(good[0]), ctypes.byref(good[1])) == 0
    assert f(4, -1, ctypes.byref(good[0]), ctypes.byref(good[1])) == 0
    assert f(4, 10, None, ctypes.byref(good[1])) == 0
    assert f(4, 10, ctypes.byref(good[0]), None) == 0
    assert f(4, 10, ctypes.byref(cache(d=200)), ctypes.byref(good[1])) == 0


def test_binding_refuses_what_c_cannot_see():
    t = torch.zeros(2, 16, 2, 128, dtype=torch.bfloat16)      # not on a GPU
    for args in ((t, t), (t.double(), t.double()), (t[0], t[0])):
        with pytest.raises(B.OosError):
            B.PagedCache(*args)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(B.OosError):
        B.Batch(i, i[:2], torch.zeros(2, 4, dtype=torch.int32), 3)
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(B.OosError):
        B.oos_qk_norm_rope(q, None, None, None, 1e-6, None, None, q, None)
    with pytest.raises(B.OosError):
        B.oos_qk_norm_rope(None, None, None, None, 1e-6, None, None, None, None)
