"""GPU tests of what an append to 8-bit pages does next to the border of two codes, against 64 bits (pages8_ref.py)."""

import pytest
import torch

import batch_ref as R
import pages8_ref as R8
from paper_2608_00814_gb300 import binding as B
from test_gpu_batch_ops import gen, status
from test_gpu_pages8 import pool

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _built():
    from paper_2608_00814_gb300 import _build
    _build.build()


def append_k(k, gain, eps, theta, pos, page=64):
    """(K's codes [n, nkv, d] as float64, exponents [n, nkv, 1]) of one sequence of n positions."""
    n, nkv, d = k.shape
    step = R.Step([n], [n], page)
    p, st = pool(gen(9), step.n_pages, page, nkv, d), status()
    B.oos_paged_append8(B.PagedCache8(*p), step.device(B), k, k, gain, eps, theta and B.OosRopeConfig(theta), pos, st)
    assert int(st) == 0
    order = torch.tensor(step.table[0])
    codes = p[0].cpu().double()[order].view(-1, nkv, d)[:n]
    e = R8.exps(p[2])[order].view(-1, nkv).repeat_interleave(16, 0)[:n, :, None]
    return codes, e


def check_codes(codes, e, ref, r):
    """Every code is the one of the 64-bit value, but where the restatement itself does not know: angles of up to 2^12
    radians are off by 2^-40 in 64 bits, so a value by 2^-40 of its pair's length r (twice that: both sides')."""
    y = torch.ldexp(ref, -e)
    off = torch.ldexp(r, -e) * 2.0 ** -39
    lo, hi = R8.e4m3(y - off), R8.e4m3(y + off)
    bad = ~((codes == lo) | (codes == hi))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist())
    return int((lo == hi).sum()) / codes.numel()


def test_what_fp32_passes_stays_nan():
    """An element whose product with the gain is past fp32 is NaN, whatever stands beside it: its partner within eight
    steps of a border (1.0625 of a power of two) is a number still."""
    nkv, d, m = 2, 128, 3
    gain = torch.ones(d)
    gain[m] = 3e38
    k = torch.ones(16, nkv, d, dtype=torch.float64)
    k[..., m] = 4.0
    rest = (k * k).sum(-1) - 1.0
    want = 1.0625 * (1 + torch.arange(-8, 8).double()[:, None] * 2.0 ** -23)      # of the partner, normed
    k[..., m + d // 2] = want * torch.sqrt(rest / (d - want * want))
    codes, e = append_k(k.float().cuda(), gain.cuda(), 0.0, None, None, page=16)
    nan = torch.isnan(codes)
    assert bool(nan[..., m].all()) and int(nan.sum()) == 16 * nkv
    ref, r = R.norm_rope(k.float(), gain, 0.0, None, None)
    ref[..., m] = r[..., m] = 0.0
    r[..., m + d // 2] = ref[..., m + d // 2].abs()
    codes[..., m] = 0.0
    check_codes(codes, e, ref, r)
