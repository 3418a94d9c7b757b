"""Performance cases of the batch operators: what a program calls that serves many
requests whose prompts begin alike (a system prompt and tool schemas, prefilled
once) and go on in pages of their own.

  qk_norm_rope   the norms of the heads of q and k and the position rotation
  append         the step's K (normed, rotated) and V into the requests' pages
  attention      the step's queries over the shared prefix and the own pages

A case's sizes follow from its fields alone ("ragged" seeds the lengths, the
page order and the trees); the values of the tensors follow from the seed.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # one token of one request on the small target: launch latency
        dict(name="rope-one-0.6b", op="qk_norm_rope", n=1, nq=16, nkv=8, d=128, dtype="bf16", norm=True, rescale=False,
             fused=True, far=False),
        # a prefill chunk of the 8B-class target, q and k slices of one projection's rows
        dict(name="rope-chunk-8b", op="qk_norm_rope", n=2048, nq=32, nkv=8, d=128, dtype="bf16", norm=True,
             rescale=False, fused=True, far=False),
        # a long batch of prompts, rotation only, rescaled rates, far positions
        dict(name="rope-long-f16", op="qk_norm_rope", n=15001, nq=32, nkv=8, d=128, dtype="f16", norm=False,
             rescale=True, fused=False, far=True),
        # one decoding token of each of 64 requests
        dict(name="append-decode", op="append", batch=64, mode="decode", q=1, suffix=700, nkv=8, d=128, dtype="bf16",
             kv="bf16", page=16, norm=True, ragged=11),
        # the requests' own prompts after the shared one, binary16 pages, rescaled rates
        dict(name="append-prompts-f16", op="append", batch=24, mode="ragged", q=700, suffix=40, nkv=8, d=128,
             dtype="bf16", kv="f16", page=64, norm=False, ragged=12),
        # an fp32 toy decoder of odd sizes
        dict(name="append-f32", op="append", batch=5, mode="ragged", q=9, suffix=33, nkv=2, d=64, dtype="f32", kv="f32",
             page=7, norm=True, ragged=13),
        # one request, one token, short context: latency
        dict(name="attn-one-0.6b", op="attention", batch=1, mode="decode", q=1, prefix=1024, suffix=17, nq=16, nkv=8,
             d=128, dtype="bf16", kv="bf16", page=16, ragged=21),
        # the ordinary decoding step of a server: 64 requests of an 8B-class target
        dict(name="attn-decode-8b", op="attention", batch=64, mode="decode", q=1, prefix=8192, suffix=1000, nq=32, nkv=8,
             d=128, dtype="bf16", kv="bf16", page=16, ragged=22),
        # many requests behind a long prefix
        dict(name="attn-decode-long", op="attention", batch=256, mode="decode", q=1, prefix=32768, suffix=300, nq=32,
             nkv=8, d=128, dtype="bf16", kv="bf16", page=64, ragged=23),
        # a tree of up to 64 candidates for each of 16 requests, the verification step in a batch
        dict(name="attn-trees-8b", op="attention", batch=16, mode="tree", q=64, prefix=2048, suffix=400, nq=32, nkv=8,
             d=128, dtype="bf16", kv="bf16", page=32, ragged=24),
        # ragged prompts of 40-head requests after the shared one, binary16 pages
        dict(name="attn-prompts-f16", op="attention", batch=13, mode="ragged", q=300, prefix=4095, suffix=100, nq=40,
             nkv=8, d=128, dtype="bf16", kv="f16", page=64, ragged=25),
        # fp32 toy decoder
        dict(name="attn-f32", op="attention", batch=9, mode="ragged", q=8, prefix=501, suffix=120, nq=4, nkv=2, d=64,
             dtype="f32", kv="f32", page=10, ragged=26),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["qk_norm_rope", "append", "attention", "attention", "attention"])
    f32 = rng.random() < 0.2
    if f32:
        heads, d = rng.choice([(4, 2), (6, 6), (9, 3), (8, 1)]), rng.choice([32, 64, 80, 128])
        dtype, kv = "f32", "f32"
    else:
        heads, d = rng.choice([(16, 8), (32, 8), (40, 8), (64, 8), (4, 2), (12, 12)]), 128
        dtype, kv = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f16"), ("f16", "f16")])
    nq, nkv = heads
    if op == "qk_norm_rope":
        return dict(op=op, n=_log(rng, 1, 15000), nq=nq, nkv=nkv, d=d, dtype=dtype, norm=rng.random() < 0.6,
                    rescale=rng.random() < 0.4, fused=rng.random() < 0.5, far=rng.random() < 0.3)
    mode = rng.choice(["decode", "decode", "tree", "ragged"])
    batch = _log(rng, 1, 256)
    page = rng.choice([1, 7, 16, 16, 32, 64, 100, 128, 256])
    common = dict(op=op, batch=batch, mode=mode, nkv=nkv, d=d, dtype=dtype, kv=kv, page=page,
                  ragged=rng.randint(1, 1 << 30))
    if op == "append":
        q = 1 if mode == "decode" else min(128 if mode == "tree" else 2048, _log(rng, 1, max(1, 16000 // batch)))
        return dict(common, q=q, suffix=_log(rng, 1, 1500), norm=rng.random() < 0.5)
    most = 256 if f32 else 2048
    q = 1 if mode == "decode" else min(128 if mode == "tree" else 400, _log(rng, 1, max(1, most // batch)))
    suffix = _log(rng, 1, max(2, min(2000, 100000 // batch)))
    tokens = batch * q
    far = min(32768, int(3.0e10 / (128 * nq * tokens)) if not f32 else 2048)   # bounds the work of the prefix
    prefix = _log(rng, 1, max(1, far)) if rng.random() < 0.93 else 0
    return dict(common, q=q, suffix=suffix, nq=nq, prefix=prefix)


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


def _pages(lens, page):
    return [(n + page - 1) // page for n in lens]


def _layout(case, g):
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
    pos0 = 1000
    s = dict(counts=counts, lens=lens, total=total, n=start[-1], rows=start[-1] + pad,
             q_start=torch.tensor(start, **i32), seq_len=torch.tensor(lens, **i32),
             block_table=torch.tensor(table, **i32), status=torch.zeros(1, **i32),
             positions=torch.tensor([pos0 + n - c + j for c, n in zip(counts, lens) for j in range(c)] + [0] * pad,
                                    **i32), parent=None)
    if case["mode"] == "tree":
        par = []
        for c in counts:
            par += [-1] + [rng.randint(max(0, j - 6), j - 1) for j in range(1, c)]
        s["parent"] = torch.tensor(par + [-1] * pad, **i32)
    return s


def work(case):
    es = ESIZE[case["dtype"]]
    d, nkv = case["d"], case["nkv"]
    if case["op"] == "qk_norm_rope":
        elems = case["n"] * (case["nq"] + nkv) * d
        return {"bytes": 2 * elems * es + 4 * case["n"], "flops": (10 if case["norm"] else 6) * elems}
    counts, lens = _lengths(case)
    n, ks = sum(counts), ESIZE[case["kv"]]
    if case["op"] == "append":
        return {"bytes": 2 * n * nkv * d * (es + ks) + 8 * n + 8 * case["batch"], "flops": 10 * n * nkv * d}
    seen = sum(c * (m - c) + (c * (c + 1) // 2 if case["mode"] != "tree" else 4 * c) for c, m in zip(counts, lens))
    keys = case["prefix"] + sum(m for c, m in zip(counts, lens) if c)
    return {"bytes": 2 * keys * nkv * d * ks + 2 * n * case["nq"] * d * es + 8 * case["batch"] +
            4 * sum(_pages(lens, case["page"])),
            "flops": 4 * d * case["nq"] * (n * case["prefix"] + seen)}


# ------------------------------------------------------------------ inputs

def _rates(case):
    """Rotation rates, radians per position, in 64 bits."""
    d, theta = case["d"], 5e5 if case.get("rescale") else 1e6
    f = theta ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    if case.get("rescale"):       # long wavelengths turn slower, a band between blends
        wave = 2 * math.pi / f
        w = ((8192 / wave - 1.0) / 3.0).clamp(0.0, 1.0)
        f = (1 - w) * f / 8.0 + w * f
    return f


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    d, nkv = case["d"], case["nkv"]

    def randn(*shape, std=1.0, to=dt):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(to)

    s = dict(case=dict(case), rates=_rates(case), eps=1e-6)
    s["q_norm"], s["k_norm"] = 1 + randn(d, std=0.1), 1 + randn(d, std=0.1)
    if case["op"] == "qk_norm_rope":
        n, nq = case["n"], case["nq"]
        if case["fused"]:       # rows of one projection: q heads, k heads, v heads
            rows = randn(n, nq + 2 * nkv, d, std=2.0)
            s["q"], s["k"] = rows[:, :nq], rows[:, nq:nq + nkv]
        else:
            s["q"], s["k"] = randn(n, nq, d, std=2.0), randn(n, nkv, d, std=2.0)
        most = 1000000 if case["far"] else 16384
        s["positions"] = torch.randint(0, most, (n,), generator=g, device="cuda", dtype=torch.int32)
        s["q_out"], s["k_out"] = torch.empty(n, nq, d, dtype=dt, device="cuda"), torch.empty(n, nkv, d, dtype=dt, device="cuda")
    else:
        s.update(_layout(case, g))
        kdt = DTYPES[case["kv"]]
        pool = (s["total"], case["page"], nkv, d)
        s["k_pages"], s["v_pages"] = randn(*pool, to=kdt), randn(*pool, to=kdt)
        if case["op"] == "append":
            s["k"], s["v"] = randn(s["rows"], nkv, d, std=2.0), randn(s["rows"], nkv, d)
        else:
            s["q"] = randn(s["rows"], case["nq"], d, std=1.5)
            s["prefix_k"] = randn(case["prefix"] + 5, nkv, d, to=kdt)      # a cache with room behind the prefix
            s["prefix_v"] = randn(case["prefix"] + 5, nkv, d, to=kdt)
            s["out"] = torch.zeros(s["rows"], case["nq"], d, dtype=dt, device="cuda")
    if own:
        from paper_2608_00814_gb300 import binding as B
        s["rope"] = B.OosRopeConfig(5e5, 8.0, 1.0, 4.0, 8192) if case.get("rescale") else B.OosRopeConfig(1e6)
        if case["op"] != "qk_norm_rope":
            s["cache"] = B.PagedCache(s["k_pages"], s["v_pages"])
            s["step"] = B.Batch(s["q_start"], s["seq_len"], s["block_table"], s["rows"])
        if case["op"] == "attention":
            s["ws"] = torch.empty(B.oos_shared_prefix_attention_workspace_bytes(
                s["q"], case["prefix"], s["cache"], s["step"]), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if own:
        from paper_2608_00814_gb300 import binding as B
        norm = case.get("norm", False)
        if case["op"] == "qk_norm_rope":
            B.oos_qk_norm_rope(s["q"], s["k"], s["q_norm"] if norm else None, s["k_norm"] if norm else None, s["eps"],
                               s["rope"], s["positions"], s["q_out"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        if case["op"] == "append":
            B.oos_paged_append(s["cache"], s["step"], s["k"], s["v"], s["k_norm"] if norm else None, s["eps"],
                               s["rope"], s["positions"], s["status"])
            return {"k": s["k_pages"], "v": s["v_pages"]}
        B.oos_shared_prefix_attention(s["q"], s["prefix_k"], s["prefix_v"], case["prefix"], s["cache"], s["step"],
                                      s["parent"], 1.0 / math.sqrt(case["d"]), s["out"], s["ws"], s["status"])
        return s["out"]
    return {"qk_norm_rope": _plain_qk_norm_rope, "append": _plain_append, "attention": _plain_attention}[case["op"]](s)


def _norm_rotate(x, gain, eps, positions, rates):
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * gain.float()
    a = positions.double()[:, None] * rates        # far positions need 64 bits
    c, s = a.cos().float()[:, None], a.sin().float()[:, None]
    h = x.shape[-1] // 2
    lo, hi = x[..., :h], x[..., h:]
    return torch.cat((lo * c - hi * s, hi * c + lo * s), -1)


def _plain_qk_norm_rope(s):
    norm = s["case"]["norm"]
    for name in ("q", "k"):
        y = _norm_rotate(s[name], s[name + "_norm"] if norm else None, s["eps"], s["positions"], s["rates"])
        s[name + "_out"].copy_(y)
    return {"q": s["q_out"], "k": s["k_out"]}


def _sequence_of(s):
    """Request and place within the step of every token, and its slot behind the prefix."""
    i = torch.arange(s["n"], device="cuda")
    b = torch.searchsorted(s["q_start"][1:].contiguous(), i, right=True)
    j = i - s["q_start"][b]
    first = s["seq_len"] - (s["q_start"][1:] - s["q_start"][:-1])
    return b, j, first[b] + j


def _plain_append(s):
    case, n = s["case"], s["n"]
    b, _, slot = _sequence_of(s)
    page = s["block_table"][b, slot // case["page"]].long()
    k = _norm_rotate(s["k"][:n], s["k_norm"] if case["norm"] else None, s["eps"], s["positions"][:n], s["rates"])
    s["k_pages"][page, slot % case["page"]] = k.to(s["k_pages"].dtype)
    s["v_pages"][page, slot % case["page"]] = s["v"][:n].float().to(s["v_pages"].dtype)
    return {"k": s["k_pages"], "v": s["v_pages"]}


def _plain_attention(s):
    case, n = s["case"], s["n"]
    B, P, page, nkv, d = case["batch"], case["prefix"], case["page"], case["nkv"], case["d"]
    G = case["nq"] // nkv
    Q, L = max(max(s["counts"]), 1), max(s["lens"])
    b, j, slot = _sequence_of(s)
    q = (s["q"][:n].float() / math.sqrt(d)).view(n, nkv, G, d)
    # the prefix: one product for all tokens
    pk, pv = s["prefix_k"][:P].float(), s["prefix_v"][:P].float()
    sp = (q.permute(1, 0, 2, 3).reshape(nkv, n * G, d) @ pk.permute(1, 2, 0)).view(nkv, n, G, P)
    # the requests' own positions, gathered and padded to the longest
    at = torch.arange(L, device="cuda")
    pages = s["block_table"][:, at // page].long()
    own_k = s["k_pages"][pages, at % page].float()          # [B, L, nkv, d]
    own_v = s["v_pages"][pages, at % page].float()
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


# ------------------------------------------------------------------ the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)

    def turned(x, gain, positions):
        x = x.double()
        if gain is not None:
            x = x / (x.pow(2).mean(-1, keepdim=True) + s["eps"]).sqrt() * gain.double()
        half = case["d"] // 2
        z = torch.complex(x[..., :half], x[..., half:])
        a = torch.outer(positions.double(), s["rates"])
        z = z * torch.polar(torch.ones_like(a), a).unsqueeze(1)
        return torch.cat((z.real, z.imag), -1)

    if case["op"] == "qk_norm_rope":
        return {x: turned(s[x], s[x + "_norm"] if case["norm"] else None, s["positions"]) for x in ("q", "k")}
    page = case["page"]
    table = s["block_table"].tolist()
    starts = s["q_start"].tolist()
    if case["op"] == "append":
        k = turned(s["k"], s["k_norm"] if case["norm"] else None, s["positions"])
        out = {"k": s["k_pages"].double(), "v": s["v_pages"].double()}
        flat = {x: out[x].view(-1, case["nkv"], case["d"]) for x in out}
        rows, to = [], []
        for b in range(case["batch"]):
            for i in range(starts[b], starts[b + 1]):
                p = s["lens"][b] - (starts[b + 1] - i)
                rows.append(i)
                to.append(table[b][p // page] * page + p % page)
        rows, to = torch.tensor(rows, device="cuda"), torch.tensor(to, device="cuda")
        flat["k"][to] = k[rows]
        flat["v"][to] = s["v"].double()[rows]
        return out
    G = case["nq"] // case["nkv"]
    out = s["out"].double()
    pk, pv = s["prefix_k"][:case["prefix"]].double(), s["prefix_v"][:case["prefix"]].double()
    for b in range(case["batch"]):
        lo, hi, n = starts[b], starts[b + 1], s["lens"][b]
        if lo == hi:
            continue
        where = [table[b][p // page] * page + p % page for p in range(n)]
        where = torch.tensor(where, device="cuda")
        k = torch.cat((pk, s["k_pages"].view(-1, case["nkv"], case["d"])[where].double()))
        v = torch.cat((pv, s["v_pages"].view(-1, case["nkv"], case["d"])[where].double()))
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
            t = s["q"][lo:hi, h].double() @ k[:, h // G].T / math.sqrt(case["d"])
            t = torch.softmax(t.masked_fill(~keep, -math.inf), -1)
            out[lo:hi, h] = t @ v[:, h // G]
    return out
