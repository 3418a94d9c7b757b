"""GPU tests of what an append to 8-bit pages does next to the border of two codes, against 64 bits (pages8_ref.py)."""

import math

import pytest
import torch

import batch_ref as R
import pages8_ref as R8
from paper_2608_00814_gb300 import binding as B
from test_gpu_batch_ops import BF16, F16, gen, randn, status
from test_gpu_pages8 import pool

pytestmark = pytest.mark.gpu

VALUES = torch.arange(0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).double()      # of the codes, ascending


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


def check_codes(codes, e, ref, r, norm, theta, nan=None):
    """Every code is that of a value within the error of fp32: in half steps, 13.5 of a normed value (a sum of squares of
    at most 13 roundings in turn, the mean and eps 2, half of all that after the root, the root 4, two products 2), and
    6.5 of a turned pair's length r (cosine and sine 2.5 each, products and sum 1.5).  Without norms the larger element
    of a turned pair, where its code is a normal one, has the code of its 64-bit value; the restatement knows that but
    for 2^-39 of r (angles of up to 2^12 radians are off by 2^-40 in 64 bits, on either side)."""
    y = torch.ldexp(ref, -e)
    off = R.F32 * torch.ldexp((13.5 * r if norm else 0) + (6.5 * r if theta else 0), -e)
    lo, hi = R8.e4m3(y - off), R8.e4m3(y + off)
    ok = (lo <= codes) & (codes <= hi) if nan is None else torch.where(nan, torch.isnan(codes), (lo <= codes) & (codes <= hi))
    assert bool(ok.all()), (int((~ok).sum()), (~ok).nonzero()[:3].tolist())
    if theta and not norm:
        h = ref.shape[-1] // 2
        larger = (y.abs() >= torch.cat((y[..., h:], y[..., :h]), -1).abs()) & (y.abs() >= 2.0 ** -6)
        off = torch.ldexp(r, -e) * 2.0 ** -39
        lo, hi = R8.e4m3(y - off), R8.e4m3(y + off)
        bad = larger & (codes != lo) & (codes != hi) & (~nan if nan is not None else True)
        assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist())
        assert float((lo == hi)[larger].double().mean()) > 0.99


def near_borders(n, nkv, d, norm, theta, seed):
    """fp32 rows (with their gain and positions) of whose normed and turned values a third lie within a few steps of fp32 of
    a border of two codes, subnormal ones too, beside partners of any size.  The first pair gives its row the length that
    it needs."""
    g = torch.Generator().manual_seed(seed)
    idx = torch.randint(0, 0x60, (n, nkv, d), generator=g)
    y = (VALUES[idx] + VALUES[idx + 1]) / 2 * (torch.randint(0, 2, (n, nkv, d), generator=g) * 2 - 1)
    far = torch.randint(0, 2, (n, nkv, d // 2), generator=g).bool()      # one of each pair, and more
    y *= torch.where(torch.cat((far, ~far), -1) | (torch.rand(n, nkv, d, generator=g) < 0.3), 1.01, 1.0)
    pos = torch.randint(0, 4096, (n,), generator=g, dtype=torch.int32)
    h, eps, ms = d // 2, 1e-6, 9.0      # the mean square of a row
    gain = (40 * (1 + 0.2 * torch.randn(d, generator=g))).clamp(20, 60)
    gain[0] = gain[h] = 40.0
    a = (pos.double()[:, None] * R.rates(d, theta))[:, None] if theta else torch.zeros(n, 1, h, dtype=torch.float64)
    c, s = torch.cos(a), torch.sin(a)

    def unturned():
        return torch.cat((y[..., :h] * c + y[..., h:] * s, y[..., h:] * c - y[..., :h] * s), -1)
    y[..., 0], y[..., h] = 0.0 if norm else 300.0, 0.0
    z = unturned()
    if norm:
        z = z / gain.double()
        y[..., 0] = 40.0 * torch.sqrt(d * ms / (ms + eps) - (z * z).sum(-1))
        z = unturned() / gain.double() * math.sqrt(ms + eps)
    return z.float(), gain if norm else None, eps, pos


@pytest.mark.parametrize("d, nkv", [(128, 2), (64, 3), (128, 9), (96, 1), (66, 2), (4, 1)])
@pytest.mark.parametrize("norm, theta", [(True, 1e6), (True, None), (False, 1e6)])
def test_values_next_to_a_border(norm, theta, d, nkv):
    """Pairs that nearly cancel and values of subnormal codes among them; also from rows off 16-byte boundaries."""
    k, gain, eps, pos = near_borders(512, nkv, d, norm, theta, d)
    ref, r = R.norm_rope(k, gain, eps, theta and R.rates(d, theta), pos)
    for shift in (0, 1):
        flat = torch.empty(k.numel() + 1, device="cuda")
        x = flat[shift:shift + k.numel()].view(k.shape).copy_(k)
        codes, e = append_k(x, gain.cuda() if norm else None, eps, theta, pos.cuda())
        check_codes(codes, e, ref, r if theta else ref.abs(), norm, theta)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("norm, theta", [(True, 1e6), (True, None), (False, 1e6)])
def test_many_values(dtype, norm, theta):
    """Rows as they come, some elements far larger than the others, so that those take subnormal codes."""
    n, nkv, d = 8192, 8, 128
    g = gen(11)
    k = randn(g, n, nkv, d, dtype=dtype)
    gain = 1 + randn(g, d, dtype=dtype, std=0.2)
    gain[7] = 200.0
    k[::3, :, 9] *= 200
    pos = torch.randint(0, 4096, (n,), generator=g, device="cuda", dtype=torch.int32)
    codes, e = append_k(k, gain if norm else None, 1e-6, theta, pos)
    ref, r = R.norm_rope(k, gain if norm else None, 1e-6, theta and R.rates(d, theta), pos)
    check_codes(codes, e, ref, r if theta else ref.abs(), norm, theta)


@pytest.mark.parametrize("norm", [False, True])
def test_a_step_of_few_rows(norm):
    """Rows among positions held before: the border is of the scale that the block has."""
    nkv, d, n = 3, 128, 16
    k, gain, eps, pos = near_borders(n, nkv, d, norm, 1e6, 5)
    ref, r = R.norm_rope(k, gain, eps, R.rates(d, 1e6), pos)
    p, st = pool(gen(9), 3, 16, nkv, d, lo=-3, hi=-1), status()
    for i in range(n):
        step = R.Step([1], [i + 1], 16, spare_pages=1)
        step.table, step.n_pages, step.width = [[2]], 3, 1
        x = k[i:i + 1].cuda()
        B.oos_paged_append8(B.PagedCache8(*p), step.device(B), x, x, gain.cuda() if norm else None, eps, B.OosRopeConfig(1e6),
                            pos[i:i + 1].cuda(), st)
        codes, e = p[0][2, i:i + 1].cpu().double(), R8.exps(p[2])[2, 0][None, :, None]
        check_codes(codes, e, ref[i:i + 1], r[i:i + 1], norm, 1e6)
    assert int(st) == 0


def test_infinite_elements_stay_nan():
    """Pairs with an infinite element are NaN, also beside pairs of the same row that are computed again."""
    k, _, eps, pos = near_borders(512, 2, 128, False, 1e6, 6)
    k[..., 4:60:8] = math.inf
    k[..., 66:128:16] = -math.inf
    codes, e = append_k(k.cuda(), None, eps, 1e6, pos.cuda())
    nan = torch.isinf(k[..., :64]) | torch.isinf(k[..., 64:])
    nan = torch.cat((nan, nan), -1)
    ref, r = R.norm_rope(torch.where(nan, 0.0, k), None, eps, R.rates(128, 1e6), pos)
    check_codes(codes, e, ref, r, False, 1e6, nan)


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
    nan = torch.zeros(k.shape, dtype=torch.bool)
    nan[..., m] = True
    ref, _ = R.norm_rope(k.float(), gain, 0.0, None, None)
    ref[..., m] = 0.0
    check_codes(codes, e, ref, ref.abs(), True, None, nan)
