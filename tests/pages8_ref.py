"""64-bit restatement of the operators on 8-bit pages, and the inputs of their tests."""

import math

import torch

import batch_ref as R

LOW, HIGH, BLOCK = -117, 119, 16
NAN_CODE = 0x7F


def e4m3(x):
    """x (float64, magnitudes up to 448 after saturation) to four significant bits and steps of 2^-9 at least."""
    x = x.double().clamp(-448, 448)
    step = torch.ldexp(torch.ones_like(x), torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.where(torch.isnan(x), x, (x / step).round() * step)


def needed(top):
    """Least exponent with top <= 448 2^e."""
    if not top > 0:
        return LOW
    m, e = math.frexp(top)
    return max(LOW, min(HIGH, e - 9 + (m > 0.875)))


def exps(scale):
    return (scale.view(torch.uint8).cpu().int() - 127).clamp(LOW, HIGH)


def values(codes, scale):
    """What pages hold, float64 on the CPU, of codes [.., page, nkv, d] and scales [.., page / 16, nkv]."""
    p = torch.ldexp(torch.ones(scale.shape, dtype=torch.float64), exps(scale))
    return codes.cpu().double() * p.repeat_interleave(BLOCK, -2)[..., None]


def rescaled(codes, d):
    """Codes (float64) after a growth of their scale by 2^d."""
    return e4m3(codes * 2.0 ** -d)


def same(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


def check_append(step, before, after, y, tol, what=""):
    """One side of an append: before, after = (codes, scale) of the pool; y [n, nkv, d] the exact rows, tol
    [n, nkv, d] what the fp32 arithmetic before the rounding may be off by.  The scale is the least for some
    values within tol of y; every code is the rounding of a value within tol, so it is off by half a step of the
    value (2^-4, or 2^-10 of the scale's unit) and tol; codes from before are rounded again exactly; nothing
    else changes."""
    c0, c1 = before[0].cpu().double(), after[0].cpu().double()
    e0, e1 = exps(before[1]), exps(after[1])
    touched = torch.zeros(c0.shape[:2], dtype=torch.bool)
    touched_scale = torch.zeros(e0.shape[:2], dtype=torch.bool)
    nkv = c0.shape[2]
    for b, (c, n) in enumerate(zip(step.counts, step.lens)):
        first = n - c
        for blk in range(max(first, 0) // BLOCK, (n + BLOCK - 1) // BLOCK if c else 0):
            lo, hi = max(first, blk * BLOCK, 0), min(n, blk * BLOCK + BLOCK)
            page, at = step.where(b, blk * BLOCK)
            s = at // BLOCK
            rows = slice(step.q_start[b] + lo - first, step.q_start[b] + hi - first)
            touched[page, at:at + BLOCK] = touched_scale[page, s] = True
            for h in range(nkv):
                yy, tt = y[rows, h], tol[rows, h]
                ok = torch.isfinite(yy)
                top = yy.abs()[ok].max().item() if ok.any() else 0.0
                off = tt[ok].max().item() if ok.any() else 0.0
                e = int(e1[page, s, h])
                fresh = lo == blk * BLOCK and first <= blk * BLOCK
                least, most = needed(top - off), needed(top + off)
                if not fresh:
                    least, most = max(least, int(e0[page, s, h])), max(most, int(e0[page, s, h]))
                assert least <= e <= most, (what, b, blk, h, e, least, most)
                got = c1[page, at + lo - blk * BLOCK:at + hi - blk * BLOCK, h] * 2.0 ** e
                yc = yy.clamp(-448 * 2.0 ** e, 448 * 2.0 ** e)
                bad = ~((got - yc).abs() <= torch.maximum(2.0 ** -4 * yc.abs(), torch.tensor(2.0 ** (e - 10))) + tt)
                assert torch.equal(torch.isnan(got), ~ok), (what, b, blk, h)
                assert not bad[ok].any(), (what, b, blk, h, float((got - yc).abs()[ok].max()))
                if float(tt[ok].max() if ok.any() else 0) == 0:
                    assert same(got, torch.where(ok, e4m3(yy / 2.0 ** e) * 2.0 ** e, math.nan)), (what, b, blk, h)
                others = [i for i in range(BLOCK) if not lo <= blk * BLOCK + i < hi]
                if others:
                    was, now = c0[page, [at + i for i in others], h], c1[page, [at + i for i in others], h]
                    want = was if fresh else rescaled(was, e - int(e0[page, s, h]))
                    assert same(now, want), (what, "others", b, blk, h)
    assert same(c0[~touched], c1[~touched]), (what, "codes elsewhere")
    assert torch.equal(before[1].cpu()[~touched_scale], after[1].cpu()[~touched_scale]), (what, "scales elsewhere")


def attention(step, q, pk, pv, cache, scale, parent=None):
    """(out, weights times |v|, largest sum |q k| scale, bounds of the tensor-core kernels), the bounds being
      - what is left out of q, of a score: 2^-25 of a row's largest |q| in each element (binary16 after a scaling to
        [1, 2)), and 2^-17 where sequences have more than 64 rows (token, head of a group) on average: parts of four
        bits in e4m3, whose steps are 2^-9, so that half of one is left, of a largest element of 2^7 or more
      - what weights are rounded by: to bf16 with a bf16 prefix, or bf16 queries in sequences of many rows, to
        binary16 otherwise
      - what is left of a term below binary16's normal numbers: 2^-25 where the row's largest weight times scale stands
        at 2^7 or more, 2^-32 of that for each key, and of codes up to 448
      - the largest |v|."""
    kp, vp = values(cache.k, cache.k_scale), values(cache.v, cache.v_scale)
    out, mag, size = R.attention(step, q, pk, pv, kp, vp, scale, parent)
    slots = [step.where(b, s) for b, n in enumerate(step.lens) if step.counts[b] for s in range(max(n, 0))]
    many = step.n * (q.shape[1] // cache.k.shape[-2]) > 64 * len(step.counts)
    most = max([float(kp[s].abs().sum(-1).max()) for s in slots] or [0.0])
    fine = float(q[:step.n].double().abs().max()) if step.n else 0.0
    weights = torch.bfloat16 if pk.dtype is torch.bfloat16 or (many and q.dtype is torch.bfloat16) else torch.float16
    es = exps(cache.v_scale)
    unit = max([float(es[p, s // BLOCK].max()) for p, s in slots] or [LOW])
    v = [float(vp[s].abs().max()) for s in slots] + ([float(pv.double().abs().max())] if pv.numel() else [])
    return out, mag, size, (fine * most * scale * 2.0 ** (-17 if many else -25), R.U[weights], 2.0 ** (unit - 32) * 448, max(v or [0.0]))


def check_attention(got, ref, mag, size, bounds, keys, what=""):
    """The bound of batch_ref.check_attention -- half a step of the output; a score's (d + 3) half steps of fp32 of
    sum |q k| and the exponential's 4, each twice; the sums' half steps per key -- and, for the 16-bit types: the
    weights' rounding, the tensor cores' truncated sums, what is left out of q, of a score and so twice of a weight, and
    of small terms.  All but the last are relative to a weight.  One below 2^-126 of the row's largest is no normal fp32
    number and counts as 0, so that its own error is all of it: 2^-126 |v| for each key at most, which shows where v is 0
    at every key of weight.  An output of binary16 whose bound reaches past the type's largest number may be infinite."""
    got, t, (left, weights, term, v) = got.double().cpu(), got.dtype, bounds
    d = got.shape[-1]
    rel = 2 * ((d + 3) * R.F32 * size + 4 * R.F32) + (4 * keys + 64) * R.F32
    off = 2.0 ** -126 * keys * v
    if t is not torch.float32:
        rel += weights + d * R.F32 * 2 * size + 2 * left
        off += keys * term
    tol = R.U[t] * ref.abs().clamp(min=torch.finfo(t).tiny) + rel * mag + off
    past = torch.isinf(got) & (got.sign() * ref + tol > 65504) if t is torch.float16 else torch.zeros_like(got, dtype=torch.bool)
    bad = ~((got - ref).abs() <= tol) & ~past
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), float((got - ref).abs().max()))


def compacted(step, paths, side):
    """One side (codes, scale) of a layer's 8-bit pages, or values alone, after the paths' move; float64."""
    x, scale = side
    x = x.cpu().double().clone()
    e = None if scale is None else exps(scale)
    for b, path in enumerate(paths):
        first = step.lens[b] - step.counts[b]
        frm, to = [step.where(b, first + i) for i in path], [step.where(b, first + j) for j in range(len(path))]
        rows = [x[f].clone() for f in frm]
        if e is None:
            for r, t in zip(rows, to):
                x[t] = r
            continue
        came = [e[p, s // BLOCK].clone() for p, s in frm]
        for page, blk in dict.fromkeys((p, s // BLOCK) for p, s in to):
            here = [j for j, (p, s) in enumerate(to) if (p, s // BLOCK) == (page, blk)]
            new = torch.stack([e[page, blk]] + [came[j] for j in here]).amax(0)
            part = x[page, blk * BLOCK:(blk + 1) * BLOCK]
            part.copy_(e4m3(part * torch.exp2((e[page, blk] - new).double())[None, :, None]))
            for j in here:
                x[to[j]] = e4m3(rows[j] * torch.exp2((came[j] - new).double())[:, None])
            e[page, blk] = new
    return x, e
