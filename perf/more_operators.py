"""Performance cases of the operators around an 8-bit paged cache: what a server calls that keeps the
requests' own positions in e4m3 codes, with a power-of-two scale for each block of 16 positions and kv
head, and what happens to pages between two steps.

  append8     the step's K (normed, rotated) and V into 8-bit pages
  attention8  the step's queries over the shared prefix (16 bits or fp32) and the own 8-bit pages
  compact     the accepted nodes of every request's tree to their committed places, in all layers
  copy        pages of forked requests, in all layers

A case's sizes follow from its fields alone ("ragged" seeds the lengths, the page order, the trees and
the accepted paths); the values of the tensors follow from the seed.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}
E4M3 = torch.float8_e4m3fn
BLOCK = 16                      # positions that share a scale
LOW, HIGH = -117, 119           # exponents of the scales
BIAS = 127                      # a scale's byte is its exponent and this


def listed():
    return [
        # one decoding token of each of 64 requests: lookups, one row a block
        dict(name="append8-decode", op="append8", batch=64, mode="decode", q=1, suffix=700, nkv=8, d=128, dtype="bf16",
             page=16, norm=True, ragged=31),
        # the requests' own prompts behind the shared one, rescaled rates, no norms
        dict(name="append8-prompts", op="append8", batch=24, mode="ragged", q=700, suffix=40, nkv=8, d=128, dtype="bf16",
             page=64, norm=False, ragged=32),
        # one request, one token, short context: latency
        dict(name="attn8-one-0.6b", op="attention8", batch=1, mode="decode", q=1, prefix=1024, suffix=17, nq=16, nkv=8,
             d=128, dtype="bf16", prefix_dtype="bf16", page=16, ragged=41),
        # the ordinary decoding step of a server: 64 requests of an 8B-class target in long sessions
        dict(name="attn8-decode-8b", op="attention8", batch=64, mode="decode", q=1, prefix=2048, suffix=4000, nq=32, nkv=8,
             d=128, dtype="bf16", prefix_dtype="bf16", page=16, ragged=42),
        # few requests of very long contexts, nothing shared
        dict(name="attn8-decode-far", op="attention8", batch=6, mode="decode", q=1, prefix=0, suffix=64000, nq=64, nkv=8,
             d=128, dtype="bf16", prefix_dtype="bf16", page=64, ragged=43),
        # a tree of up to 64 candidates for each of 16 requests
        dict(name="attn8-trees-8b", op="attention8", batch=16, mode="tree", q=64, prefix=2048, suffix=400, nq=32, nkv=8,
             d=128, dtype="bf16", prefix_dtype="bf16", page=32, ragged=44),
        # ragged prompts of 40-head requests behind a binary16 prefix, earlier turns held in 8 bits
        dict(name="attn8-prompts-f16", op="attention8", batch=13, mode="ragged", q=300, prefix=1000, suffix=1500, nq=40,
             nkv=8, d=128, dtype="f16", prefix_dtype="f16", page=64, ragged=45),
        # fp32 toy decoder
        dict(name="attn8-f32", op="attention8", batch=9, mode="ragged", q=8, prefix=501, suffix=120, nq=4, nkv=2, d=64,
             dtype="f32", prefix_dtype="f32", page=48, ragged=46),
        # the accepted paths of 32 requests' trees, all layers of an 8B-class target
        dict(name="compact-trees-8b", op="compact", batch=32, mode="tree", q=64, suffix=200, nkv=8, d=128, dtype="bf16",
             layers=36, page=32, ragged=51),
        dict(name="compact8-trees-8b", op="compact", batch=32, mode="tree", q=64, suffix=200, nkv=8, d=128, dtype="e4m3",
             layers=36, page=32, ragged=52),
        # 96 forks of an 8B-class target: each copies the page it goes on in
        dict(name="copy-forks-8b", op="copy", pairs=96, nkv=8, d=128, dtype="bf16", layers=36, page=16, ragged=61),
        # 3 forks on the small target: latency
        dict(name="copy8-forks-0.6b", op="copy", pairs=3, nkv=8, d=128, dtype="e4m3", layers=28, page=64, ragged=62),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append8", "attention8", "attention8", "attention8", "compact", "copy"])
    ragged = rng.randint(1, 1 << 30)
    page = rng.choice([16, 16, 32, 48, 64, 128, 256])
    if op in ("compact", "copy"):
        nkv, d = rng.choice([(8, 128), (8, 128), (2, 64), (3, 80), (1, 128)])
        common = dict(op=op, nkv=nkv, d=d, dtype=rng.choice(["bf16", "e4m3", "e4m3", "f16", "f32"]),
                      layers=_log(rng, 1, 36), ragged=ragged)
        if op == "copy":
            return dict(common, pairs=min(_log(rng, 1, 96), max(1, 1536 // page)), page=page)
        return dict(common, batch=_log(rng, 1, 32), mode="tree", q=_log(rng, 2, 64), suffix=_log(rng, 1, 200), page=page)
    f32 = rng.random() < 0.2
    if f32:
        heads, d = rng.choice([(4, 2), (6, 6), (9, 3), (8, 1)]), rng.choice([32, 64, 80, 128])
        dtype = prefix_dtype = "f32"
    else:
        heads, d = rng.choice([(16, 8), (32, 8), (40, 8), (64, 8), (4, 2), (12, 12)]), 128
        dtype, prefix_dtype = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f16"), ("f16", "f16")])
    nq, nkv = heads
    mode = rng.choice(["decode", "decode", "tree", "ragged"])
    batch = _log(rng, 1, 256)
    common = dict(op=op, batch=batch, mode=mode, nkv=nkv, d=d, dtype=dtype, page=page, ragged=ragged)
    if op == "append8":
        q = 1 if mode == "decode" else min(128 if mode == "tree" else 2048, _log(rng, 1, max(1, 16000 // batch)))
        return dict(common, q=q, suffix=_log(rng, 1, 1500), norm=rng.random() < 0.5)
    most = 256 if f32 else 2048
    q = 1 if mode == "decode" else min(128 if mode == "tree" else 400, _log(rng, 1, max(1, most // batch)))
    suffix = _log(rng, 1, max(2, min(1500 if f32 else 16000, 100000 // batch // q)))
    far = min(16384, int(1.5e10 / (128 * nq * batch * q)) if not f32 else 1024)   # bounds the work of the prefix
    prefix = _log(rng, 1, max(1, far)) if rng.random() < 0.8 else 0
    return dict(common, prefix_dtype=prefix_dtype, q=q, suffix=suffix, nq=nq, prefix=prefix)


# ------------------------------------------------------------------ sizes

def _lengths(case):
    """Tokens of the step and positions held behind the prefix, of every request."""
    rng = random.Random(case["ragged"])
    B, mode = case["batch"], case["mode"]
    counts = [1 if mode == "decode" else rng.randint(max(1, case["q"] // 2), case["q"]) for _ in range(B)]
    if mode == "ragged" and B > 3:
        counts[rng.randrange(B)] = 0       # a request that waits
    lens = [c + rng.randint(0, case["suffix"]) for c in counts]
    return counts, lens


def _accepted(case):
    """The accepted path of every tree: node numbers among the request's rows, the root first."""
    rng = random.Random(case["ragged"] + 2)
    paths = []
    for c in _lengths(case)[0]:
        n = min(c, rng.randint(2, 9))
        paths.append([0] + sorted(rng.sample(range(1, c), n - 1)))
    return paths


def _pages(lens, page):
    return [(n + page - 1) // page for n in lens]


def _layout(case):
    """The plan a server keeps for a step: offsets, lengths, the page table."""
    rng = random.Random(case["ragged"] + 1)
    counts, lens = _lengths(case)
    need = _pages(lens, case["page"])
    total = sum(need) + 3
    order = list(range(total))
    rng.shuffle(order)
    width = max(1, max(need))
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [0] * (width - n))
        at += n
    start = [0]
    for c in counts:
        start.append(start[-1] + c)
    pad = 2 if case["mode"] != "decode" else 0      # rows behind the last request
    i32 = dict(dtype=torch.int32, device="cuda")
    s = dict(counts=counts, lens=lens, total=total, n=start[-1], rows=start[-1] + pad,
             q_start=torch.tensor(start, **i32), seq_len=torch.tensor(lens, **i32),
             block_table=torch.tensor(table, **i32), status=torch.zeros(1, **i32),
             positions=torch.tensor([1000 + n - c + j for c, n in zip(counts, lens) for j in range(c)] + [0] * pad, **i32),
             parent=None)
    if case["mode"] == "tree":
        par = []
        for c in counts:
            par += [-1] + [rng.randint(max(0, j - 6), j - 1) for j in range(1, c)]
        s["parent"] = torch.tensor(par + [-1] * pad, **i32)
    return s


def _pairs(case):
    rng = random.Random(case["ragged"])
    n = case["pairs"]
    order = list(range(2 * n + 3))
    rng.shuffle(order)
    return [rng.choice(order[:n]) for _ in range(n)], order[n:2 * n], 2 * n + 3


def work(case):
    es = ESIZE[case["dtype"]]
    d, nkv = case["d"], case["nkv"]
    if case["op"] == "copy":
        row = nkv * d * es + (nkv / BLOCK if es == 1 else 0)
        src, dst, _ = _pairs(case)
        return {"bytes": 2 * case["layers"] * case["page"] * row * (len(set(src)) + len(dst)) + 8 * len(src), "flops": 0}
    counts, lens = _lengths(case)
    n = sum(counts)
    if case["op"] == "compact":
        moved = sum(j != i for p in _accepted(case) for j, i in enumerate(p))
        return {"bytes": 4 * case["layers"] * moved * (nkv * d * es + (nkv / BLOCK if es == 1 else 0)) + 12 * case["batch"] +
                4 * sum(map(len, _accepted(case))), "flops": 0}
    if case["op"] == "append8":
        return {"bytes": 2 * n * nkv * (d * (es + 1) + 1 / BLOCK) + 8 * n + 8 * case["batch"], "flops": 12 * n * nkv * d}
    seen = sum(c * (m - c) + (c * (c + 1) // 2 if case["mode"] != "tree" else 4 * c) for c, m in zip(counts, lens))
    keys = sum(m for c, m in zip(counts, lens) if c)
    return {"bytes": 2 * nkv * (case["prefix"] * d * ESIZE[case["prefix_dtype"]] + keys * (d + 1 / BLOCK)) +
            2 * n * case["nq"] * d * es + 8 * case["batch"] + 4 * sum(_pages(lens, case["page"])),
            "flops": 4 * d * case["nq"] * (n * case["prefix"] + seen)}


# ------------------------------------------------------------------ inputs

def _rates(case):
    """Rotation rates, radians per position, in 64 bits; rescaled where no norms are."""
    d, rescale = case["d"], not case["norm"]
    f = (5e5 if rescale else 1e6) ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    if rescale:       # long wavelengths turn slower, a band between blends
        w = ((8192 * f / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        f = (1 - w) * f / 8.0 + w * f
    return f


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    d, nkv, page = case["d"], case["nkv"], case["page"]
    dt = DTYPES.get(case["dtype"])
    layers = case.get("layers", 0)

    def randn(*shape, std=1.0, to=dt):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(to)

    def codes(*shape):            # of values whose blocks have their largest ones anywhere in the last octave
        x = torch.empty(*shape, dtype=E4M3, device="cuda")
        for part in x.view(-1, *shape[-3:]).split(4096):
            part.copy_((torch.randn(part.shape, generator=g, device="cuda") * 90).clamp(-448, 448))
        return x

    def scales(*shape):
        return torch.randint(BIAS - 8, BIAS - 4, shape, generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)

    s = dict(case=dict(case), eps=1e-6)
    if case["op"] == "copy":
        src, dst, total = _pairs(case)
        s["src"], s["dst"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (src, dst))
        s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        s.update(_layout(case))
        total = s["total"]
    lead = (layers,) if layers else ()
    pool, blocks = lead + (total, page, nkv, d), lead + (total, page // BLOCK, nkv)
    if case["dtype"] == "e4m3" or not layers:
        s["k"], s["v"] = codes(*pool), codes(*pool)
        s["k_scale"], s["v_scale"] = scales(*blocks), scales(*blocks)
    else:
        s["k"], s["v"] = randn(*pool), randn(*pool)
    if case["op"] == "compact":
        paths = _accepted(case)
        nodes = [p + [-1] * (c - len(p)) for p, c in zip(paths, s["counts"])]
        i32 = dict(dtype=torch.int32, device="cuda")
        s["accepted"] = torch.tensor(sum(nodes, []) + [-1] * (s["rows"] - s["n"]), **i32)
        s["accepted_len"] = torch.tensor([len(p) for p in paths], **i32)
        s["new_len"] = torch.zeros(case["batch"], **i32)
    elif case["op"] == "append8":
        s["rates"] = _rates(case)
        s["k_norm"] = 1.35 + randn(d, std=0.1)
        s["k_in"], s["v_in"] = randn(s["rows"], nkv, d, std=1.4), randn(s["rows"], nkv, d)
    elif case["op"] == "attention8":
        s["q"] = randn(s["rows"], case["nq"], d, std=1.5 * 0.6)
        to = DTYPES[case["prefix_dtype"]]
        s["prefix_k"] = randn(case["prefix"] + 5, nkv, d, to=to)      # a cache with room behind the prefix
        s["prefix_v"] = randn(case["prefix"] + 5, nkv, d, to=to)
        s["out"] = torch.zeros(s["rows"], case["nq"], d, dtype=dt, device="cuda")
    if own:
        from paper_2608_00814_gb300 import binding as B
        if layers and case["dtype"] == "e4m3":
            s["layers"] = B.PagedLayers([B.PagedCache8(*x) for x in zip(s["k"], s["v"], s["k_scale"], s["v_scale"])])
        elif layers:
            s["layers"] = B.PagedLayers([B.PagedCache(*x) for x in zip(s["k"], s["v"])])
        else:
            s["cache"] = B.PagedCache8(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if case["op"] != "copy":
            s["step"] = B.Batch(s["q_start"], s["seq_len"], s["block_table"], s["rows"])
        if case["op"] == "append8":
            s["rope"] = B.OosRopeConfig(1e6) if case["norm"] else B.OosRopeConfig(5e5, 8.0, 1.0, 4.0, 8192)
        if case["op"] == "attention8":
            s["ws"] = torch.empty(B.oos_shared_prefix_attention8_workspace_bytes(
                s["q"], case["prefix"], s["cache"], s["step"]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if own:
        from paper_2608_00814_gb300 import binding as B
        if case["op"] == "append8":
            B.oos_paged_append8(s["cache"], s["step"], s["k_in"], s["v_in"], s["k_norm"] if case["norm"] else None,
                                s["eps"], s["rope"], s["positions"], s["status"])
            return _pool(s)
        if case["op"] == "attention8":
            B.oos_shared_prefix_attention8(s["q"], s["prefix_k"], s["prefix_v"], case["prefix"], s["cache"], s["step"],
                                           s["parent"], 1.0 / math.sqrt(case["d"]), s["out"], s["ws"], s["status"])
            return s["out"]
        if case["op"] == "compact":
            f = B.oos_paged_compact8 if case["dtype"] == "e4m3" else B.oos_paged_compact
            f(s["layers"], s["step"], s["accepted"], s["accepted_len"], s["new_len"], s["status"])
            return dict(_pool(s), new_len=s["new_len"])
        f = B.oos_pages_copy8 if case["dtype"] == "e4m3" else B.oos_pages_copy
        f(s["layers"], s["src"], s["dst"], s["status"])
        return _pool(s)
    return {"append8": _plain_append8, "attention8": _plain_attention8, "compact": _plain_compact, "copy": _plain_copy}[case["op"]](s)


def _pool(s):
    """The pages: e4m3 codes and their scales as the powers of two that the bytes stand for, or the values themselves."""
    return {x: s[x].view(torch.float8_e8m0fnu) if x.endswith("scale") else s[x] for x in ("k", "v", "k_scale", "v_scale") if x in s}


def _power(byte):
    return torch.exp2(byte.float() - BIAS)


def _needed(amax):
    """Byte of the least scale that holds the largest magnitude: amax <= 448 2^e, 448 = 0.875 2^9."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(amax > 0, e, LOW).clamp(LOW, HIGH) + BIAS


def _sequence_of(s):
    """Request and place within the step of every token, and its slot behind the prefix."""
    i = torch.arange(s["n"], device="cuda")
    b = torch.searchsorted(s["q_start"][1:].contiguous(), i, right=True)
    j = i - s["q_start"][b]
    first = s["seq_len"] - (s["q_start"][1:] - s["q_start"][:-1])
    return b, j, first[b] + j


def _plain_append8(s):
    case, n = s["case"], s["n"]
    page, nkv, d = case["page"], case["nkv"], case["d"]
    b, j, slot = _sequence_of(s)
    first = slot - j
    at = s["block_table"][b, slot // page].long() * page + slot % page      # position in the pool
    k = s["k_in"][:n].float()
    if case["norm"]:
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + s["eps"]) * s["k_norm"].float()
    a = s["positions"][:n].double()[:, None] * s["rates"]                   # far positions need 64 bits
    cs, sn = a.cos().float()[:, None], a.sin().float()[:, None]
    lo, hi = k[..., :d // 2], k[..., d // 2:]
    k = torch.cat((lo * cs - hi * sn, hi * cs + lo * sn), -1)
    # the blocks that the step writes into, each once, and their place in the pool
    blocks, of = torch.unique(at // BLOCK, return_inverse=True)
    begun = torch.zeros(blocks.numel(), dtype=torch.bool, device="cuda")
    begun[of] = first > slot // BLOCK * BLOCK                               # holds positions from before
    for name, x in (("k", k), ("v", s["v_in"][:n].float())):
        pool, scale = s[name].view(-1, BLOCK, nkv, d), s[name + "_scale"].view(-1, nkv)
        amax = torch.zeros(blocks.numel(), nkv, device="cuda")
        amax.scatter_reduce_(0, of[:, None].expand(n, nkv), x.abs().amax(-1), "amax")
        old = scale[blocks].int()
        new = torch.where(begun[:, None], torch.maximum(old, _needed(amax)), _needed(amax))
        ratio = torch.where(begun[:, None], torch.exp2((old - new).float()), 1.0)
        codes = pool[blocks].float() * ratio[:, None, :, None]
        codes[of, at % BLOCK] = x / _power(new)[of][..., None]
        pool[blocks] = codes.clamp(-448, 448).to(E4M3)
        scale[blocks] = new.to(torch.uint8)
    return _pool(s)


def _plain_attention8(s):
    case, n = s["case"], s["n"]
    B, P, page, nkv, d = case["batch"], case["prefix"], case["page"], case["nkv"], case["d"]
    G = case["nq"] // nkv
    Q, L = max(max(s["counts"]), 1), max(s["lens"])
    b, j, slot = _sequence_of(s)
    q = (s["q"][:n].float() / math.sqrt(d)).view(n, nkv, G, d)
    # the prefix: one product for all tokens
    pk, pv = s["prefix_k"][:P].float(), s["prefix_v"][:P].float()
    sp = (q.permute(1, 0, 2, 3).reshape(nkv, n * G, d) @ pk.permute(1, 2, 0)).view(nkv, n, G, P)
    # the requests' own positions, gathered, scaled and padded to the longest
    at = torch.arange(L, device="cuda")
    pages = s["block_table"][:, at // page].long()
    own_k, own_v = (s[x][pages, at % page].float() * _power(s[x + "_scale"][pages, at % page // BLOCK])[..., None]
                    for x in ("k", "v"))                                        # [B, L, nkv, d]
    qp = torch.zeros(B, Q, nkv, G, d, device="cuda")
    qp[b, j] = q
    ss = (qp.permute(0, 2, 1, 3, 4).reshape(B, nkv, Q * G, d) @ own_k.permute(0, 2, 3, 1)).view(B, nkv, Q, G, L)
    first = (s["seq_len"] - (s["q_start"][1:] - s["q_start"][:-1]))[:, None]
    own_slot = first + torch.arange(Q, device="cuda")
    if s["parent"] is None:
        seen = at[None, None] <= own_slot[..., None]        # [B, Q, L]
    else:
        # ancestors: powers of (identity + parent relation), 2^7 = 128 steps
        up = torch.zeros(B, Q, Q + 1, device="cuda")
        par = s["parent"][:n].long()
        up[b, j, torch.where(par < 0, Q, par)] = 1
        up = up[..., :Q] + torch.eye(Q, device="cuda")
        for _ in range(7):
            up = (up @ up).clamp(max=1)
        k = at[None, None] - first[..., None]               # the slot's node, negative for committed ones
        anc = torch.gather(up, 2, k.clamp(0, Q - 1).expand(B, Q, L)) > 0
        seen = (k < 0) | (anc & (k < Q) & (at[None, None] < s["seq_len"][:, None, None]))
    ss = ss.masked_fill(~seen[:, None, :, None], -math.inf)
    ss = ss.permute(0, 2, 1, 3, 4)[b, j]                    # [n, nkv, G, L]
    sp = sp.permute(1, 0, 2, 3)                             # [n, nkv, G, P]
    m = ss.amax(-1, keepdim=True)
    if P:
        m = torch.maximum(m, sp.amax(-1, keepdim=True))
    m = m.masked_fill(m == -math.inf, 0.0)
    ep, es = (sp - m).exp(), (ss - m).exp()
    z = ep.sum(-1, keepdim=True) + es.sum(-1, keepdim=True)
    op = (ep.permute(1, 0, 2, 3).reshape(nkv, n * G, P) @ pv.permute(1, 0, 2)).view(nkv, n, G, d).permute(1, 0, 2, 3)
    w = torch.zeros(B, Q, nkv, G, L, device="cuda")
    w[b, j] = es
    os_ = (w.permute(0, 2, 1, 3, 4).reshape(B, nkv, Q * G, L) @ own_v.permute(0, 2, 1, 3)).view(B, nkv, Q, G, d)
    o = (op + os_.permute(0, 2, 1, 3, 4)[b, j]) / z.clamp(min=1e-38)
    s["out"][:n] = o.reshape(n, nkv * G, d).to(s["out"].dtype)
    return s["out"]


def _plain_compact(s):
    case, n = s["case"], s["n"]
    page, nkv, d, layers = case["page"], case["nkv"], case["d"], case["layers"]
    b, j, slot = _sequence_of(s)
    taken = j < s["accepted_len"][b]
    node = torch.where(taken, s["accepted"][:n], j)         # the others move onto themselves
    source = slot - j + node

    def place(x):
        return s["block_table"][b, x // page].long() * page + x % page

    to, frm = place(slot), place(source)
    if case["dtype"] != "e4m3":
        for name in ("k", "v"):
            pool = s[name].view(layers, -1, nkv, d)
            pool[:, to] = pool[:, frm]
    else:
        # blocks with a place that is taken: the largest of the scales that meet there
        blocks, of = torch.unique((to // BLOCK)[taken], return_inverse=True)
        for name in ("k", "v"):
            pool, scale = s[name].view(layers, -1, nkv, d), s[name + "_scale"].view(layers, -1, nkv)
            old = scale[:, blocks].int()
            new = old.scatter_reduce(1, of[None, :, None].expand(layers, -1, nkv), scale[:, (frm // BLOCK)[taken]].int(), "amax")
            codes = pool.view(layers, -1, BLOCK, nkv, d)[:, blocks].float() * torch.exp2((old - new).float())[:, :, None, :, None]
            value = pool[:, frm[taken]].float() * torch.exp2((scale[:, (frm // BLOCK)[taken]].int() - new[:, of]).float())[..., None]
            codes[:, of, (to % BLOCK)[taken]] = value
            pool.view(layers, -1, BLOCK, nkv, d)[:, blocks] = codes.to(E4M3)
            scale[:, blocks] = new.to(torch.uint8)
    s["new_len"].copy_(s["seq_len"] - (s["q_start"][1:] - s["q_start"][:-1]) + s["accepted_len"])
    return dict(_pool(s), new_len=s["new_len"])


def _plain_copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    for x in ("k", "v", "k_scale", "v_scale"):
        if x in s:
            s[x][:, dst] = s[x][:, src]
    return _pool(s)


# ------------------------------------------------------------------ the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "copy":
        out = {x: t.double() for x, t in _pool(s).items()}
        was = {x: t.clone() for x, t in out.items()}
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            for x in out:
                out[x][:, b] = was[x][:, a]
        return out
    page, nkv, d = case["page"], case["nkv"], case["d"]
    table, starts = s["block_table"].tolist(), s["q_start"].tolist()

    def where(b, p):
        return table[b][p // page] * page + p % page

    def power(byte):
        return torch.ldexp(torch.ones_like(byte, dtype=torch.float64), byte.long() - BIAS)

    def rounded(x):
        """To four significant bits and steps of 2^-9 at least, half to even."""
        step = torch.ldexp(torch.ones_like(x), torch.frexp(x.abs().clamp(min=2.0 ** -6))[1] - 4)
        return (x / step).round() * step

    def least(top):
        e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 448.0))
        e = torch.where(448.0 * torch.exp2(e - 1) >= top, e - 1, e)
        return e.clamp(LOW, HIGH).long() + BIAS

    if case["op"] == "append8":
        k = s["k_in"].double()
        if case["norm"]:
            k = k / (k.pow(2).mean(-1, keepdim=True) + s["eps"]).sqrt() * s["k_norm"].double()
        z = torch.complex(k[..., :d // 2], k[..., d // 2:])
        a = torch.outer(s["positions"].double(), s["rates"])
        z = z * torch.polar(torch.ones_like(a), a).unsqueeze(1)
        new = {"k": torch.cat((z.real, z.imag), -1), "v": s["v_in"].double()}
        out = {}
        for x in ("k", "v"):
            pool, scale = s[x].double().view(-1, nkv, d), s[x + "_scale"].long().view(-1, nkv)
            for b, (c, n) in enumerate(zip(s["counts"], s["lens"])):
                p = n - c
                while p < n:
                    end = min(n, p // BLOCK * BLOCK + BLOCK)
                    rows = new[x][starts[b] + p - (n - c):starts[b] + end - (n - c)]
                    at = where(b, p)
                    block = at // BLOCK
                    byte = least(rows.abs().amax((0, 2)))
                    if p % BLOCK:       # shared with positions from before
                        byte = torch.maximum(byte, scale[block])
                        whole = pool[block * BLOCK:(block + 1) * BLOCK]
                        whole.copy_(rounded(whole * (power(scale[block]) / power(byte))[:, None]))
                    pool[at:at + end - p] = rounded(rows / power(byte)[:, None])
                    scale[block] = byte
                    p = end
            out[x], out[x + "_scale"] = pool.view(s[x].shape), power(scale).view(s[x + "_scale"].shape)
        return out
    if case["op"] == "compact":
        layers, paths = case["layers"], _accepted(case)
        out = {}
        for x in ("k", "v"):
            pool = s[x].double().view(layers, -1, nkv, d)
            scale = s[x + "_scale"].long().view(layers, -1, nkv) if case["dtype"] == "e4m3" else None
            for b, (c, n) in enumerate(zip(s["counts"], s["lens"])):
                frm = [where(b, n - c + i) for i in paths[b]]
                to = [where(b, n - c + j) for j in range(len(paths[b]))]
                if scale is None:
                    pool[:, to] = pool[:, frm]
                    continue
                moved = pool[:, frm] * power(scale[:, [i // BLOCK for i in frm]])[..., None]
                came = [scale[:, i // BLOCK].clone() for i in frm]
                for block in sorted(set(t // BLOCK for t in to)):
                    byte = torch.stack([scale[:, block]] + [e for e, t in zip(came, to) if t // BLOCK == block]).amax(0)
                    whole = pool[:, block * BLOCK:(block + 1) * BLOCK]
                    whole.copy_(rounded(whole * (power(scale[:, block]) / power(byte))[:, None, :, None]))
                    for j, t in enumerate(to):
                        if t // BLOCK == block:
                            pool[:, t] = rounded(moved[:, j] / power(byte)[..., None])
                    scale[:, block] = byte
            out[x] = pool.view(s[x].shape)
            if scale is not None:
                out[x + "_scale"] = power(scale).view(s[x + "_scale"].shape)
        out["new_len"] = torch.tensor([n - c + len(p) for c, n, p in zip(s["counts"], s["lens"], paths)], dtype=torch.int32,
                                      device="cuda")
        return out
    G = case["nq"] // nkv
    out = s["out"].double()
    pk, pv = s["prefix_k"][:case["prefix"]].double(), s["prefix_v"][:case["prefix"]].double()
    flat = {x: s[x].view(-1, nkv, d) for x in ("k", "v")}
    byte = {x: s[x + "_scale"].view(-1, nkv) for x in ("k", "v")}
    for b in range(case["batch"]):
        lo, hi, n = starts[b], starts[b + 1], s["lens"][b]
        if lo == hi:
            continue
        at = torch.tensor([where(b, p) for p in range(n)], device="cuda")
        k, v = (torch.cat((x, flat[y][at].double() * power(byte[y][at // BLOCK])[..., None])) for x, y in ((pk, "k"), (pv, "v")))
        c = hi - lo
        keep = torch.ones(c, k.shape[0], dtype=torch.bool)
        if s["parent"] is None:
            keep[:, k.shape[0] - c:] = torch.ones(c, c).tril() > 0
        else:
            par = s["parent"][lo:hi].tolist()
            keep[:, k.shape[0] - c:] = False
            for i in range(c):
                a = i
                while a >= 0:
                    keep[i, k.shape[0] - c + a] = True
                    a = par[a]
        keep = keep.cuda()
        for h in range(case["nq"]):
            t = s["q"][lo:hi, h].double() @ k[:, h // G].T / math.sqrt(d)
            t = torch.softmax(t.masked_fill(~keep, -math.inf), -1)
            out[lo:hi, h] = t @ v[:, h // G]
    return out
