"""64-bit restatement of the batch operators (plain loops over sequences) and the
inputs of their tests."""

import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step, relative
F32 = U[torch.float32]


def rates(d, theta=1e6, factor=0.0, lo=1.0, hi=4.0, orig=8192):
    f = torch.tensor([theta ** (-2.0 * m / d) for m in range(d // 2)], dtype=torch.float64)
    if factor > 1:
        wave = 2 * math.pi / f
        w = ((orig / wave - lo) / (hi - lo)).clamp(0, 1)
        f = (1 - w) * f / factor + w * f
    return f


def norm_rope(x, gain, eps, f, positions):
    """(result, length of each rotated pair) in float64; f None: no rotation."""
    x = x.double().cpu()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double().cpu()
    h = x.shape[-1] // 2
    r = torch.hypot(x[..., :h], x[..., h:]).repeat(1, 1, 2)
    if f is None:
        return x, r
    a = (positions.cpu().double()[:, None] * f)[:, None]
    c, s = torch.cos(a), torch.sin(a)
    return torch.cat((x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s), -1), r


def check_norm_rope(got, ref, r, what=""):
    """Half a step of the output's type, and for the fp32 arithmetic before it: the sum of squares
    adds at most 21 terms in turn (10.5 half steps after the root), rsqrt and its operands 8, the gain
    2, cosine and sine (2 ulp each, an angle rounded once) at most 7 over both terms, their products
    and the sum 3: under 32 half steps of the pair's length."""
    got, t = got.double().cpu(), got.dtype
    tiny = torch.finfo(t).tiny
    tol = U[t] * ref.abs().clamp(min=tiny) + 32 * F32 * r
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((got - ref).abs().max()))


def ancestors(parent):
    n = len(parent)
    a = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        j = i
        while j >= 0:
            a[i, j] = True
            j = parent[j]
    return a


class Step:
    """A ragged step: counts[b] rows of sequence b, lens[b] positions after them, pages dealt in a random
    order; `pad` rows behind the last sequence."""

    def __init__(self, counts, lens, page, seed=0, pad=0, spare_pages=2, width=None):
        g = torch.Generator().manual_seed(seed)
        need = [(n + page - 1) // page for n in lens]
        self.counts, self.lens, self.page = list(counts), list(lens), page
        self.n_pages = sum(need) + spare_pages
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.width = width or max(1, max(need))
        self.table, at = [], 0
        for n in need:
            self.table.append(order[at:at + n] + [-7] * (self.width - n))
            at += n
        self.q_start = [0]
        for c in counts:
            self.q_start.append(self.q_start[-1] + c)
        self.n = self.q_start[-1]
        self.rows = self.n + pad

    def where(self, b, s):
        return self.table[b][s // self.page], s % self.page

    def device(self, B, dev="cuda"):
        i32 = dict(dtype=torch.int32, device=dev)
        return B.Batch(torch.tensor(self.q_start, **i32), torch.tensor(self.lens, **i32),
                       torch.tensor(self.table, **i32), self.rows)


def attention(step, q, pk, pv, kp, vp, scale, parent=None):
    """(out, sum of weights times |v|, largest sum |q k| scale of a row) in float64, [n, nq, d]; kp, vp:
    page tensors.  A row that sees no key is zero."""
    nq, d = q.shape[1:]
    nkv = kp.shape[2]
    G = nq // nkv
    q, pk, pv, kp, vp = (t.double().cpu() for t in (q, pk, pv, kp, vp))
    out = torch.zeros(step.n, nq, d, dtype=torch.float64)
    mag, size = torch.zeros_like(out), 0.0
    for b, (c, n) in enumerate(zip(step.counts, step.lens)):
        if c == 0:
            continue
        own = [step.where(b, s) for s in range(n)]
        k = torch.cat([pk] + [kp[p, e][None] for p, e in own])
        v = torch.cat([pv] + [vp[p, e][None] for p, e in own])
        P, first, lo = pk.shape[0], n - c, step.q_start[b]
        see = torch.ones(c, P + n, dtype=torch.bool)
        if parent is None:
            for j in range(c):
                see[j, P + max(0, first + j + 1):] = False
        else:
            see[:, P + first:] = ancestors(parent[lo:lo + c])
        for h in range(nq):
            kh, vh = k[:, h // G], v[:, h // G]
            x = q[lo:lo + c, h]
            s = (x @ kh.T * scale).masked_fill(~see, -math.inf)
            m = s.max(-1, keepdim=True).values if P + n else torch.zeros(c, 1, dtype=torch.float64)
            e = torch.where(see, torch.exp(s - m.masked_fill(m == -math.inf, 0)), 0.0)
            z = e.sum(-1, keepdim=True)
            w = torch.where(z > 0, e / z.clamp(min=1e-300), 0.0)
            out[lo:lo + c, h], mag[lo:lo + c, h] = w @ vh, w @ vh.abs()
            if P + n:
                size = max(size, float((x.abs() @ kh.abs().T * scale).max()))
    return out, mag, size


def check_attention(got, ref, mag, size, keys, weights, what=""):
    """got [n, nq, d] against (ref, mag, size).  With A = sum of the exact weights times |v|:
      - half a step of the output's type of the value;
      - the weights' own rounding for P.V, half a step of `weights` (torch type) times A;
      - a score's error, at most (d + 3) half steps of fp32 of sum |q k| scale, twice that as a
        relative error of a weight and of the sum it is divided by, and the exponential's 4 twice;
      - one half step (two where the tensor cores truncate) per key for either sum, and 64 for the joins.
    """
    got, t = got.double().cpu(), got.dtype
    d = got.shape[-1]
    rel = 2 * ((d + 3) * F32 * size + 4 * F32) + (4 * keys + 64) * F32
    if weights is not torch.float32:
        rel += U[weights] + d * F32 * 2 * size      # truncated sums of the scores
    tol = U[t] * ref.abs().clamp(min=torch.finfo(t).tiny) + rel * mag
    bad = ~((got - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), float((got - ref).abs().max()))
