"""Performance cases of the operators around the prefill: rotary positions,
the quantised key/value cache, and attention of drafted tokens over it.

Every operator stands here in its plain form (elementary torch operations in
32 bits, angles in 64) beside the library's call, on the same inputs; `exact`
states it once more from the definition in 64 bits.

Cache values: a row of 128 channels is four groups of 32, each with one
power-of-two scale 2^e, e the smallest integer >= -126 that brings the
group's largest magnitude to at most the type's largest code; every code is
the nearest one (ties to even). Codes times scale are exact in bfloat16.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
D, GROUP = 128, 32
TOP = {"fp8": 448.0, "int8": 127.0, "fp4": 6.0}
ROW = {"bf16": 256, "fp8": 128, "int8": 128, "fp4": 64}
FP4 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
HEADS = [(28, 4), (28, 4), (32, 8), (16, 2), (8, 8), (2, 1)]


# ------------------------------------------------------------------ the cases
def listed():
    def rope(name, S, Hq, Hkv, **kw):
        return {"name": name, "what": "rope", "S": S, "Hq": Hq, "Hkv": Hkv, "layout": "half", "rot": 128,
                "scaling": "none", "factor": 1.0, "axes": 1, "inverse": False, "fused": False, "first": 0, **kw}

    def rows(name, what, n, kind, Hkv, page, **kw):
        return {"name": name, "what": what, "rows": n, "type": kind, "Hkv": Hkv, "page": page, "skip": 0.0, **kw}

    def tree(name, B, T, L, Hq, Hkv, kind, page, **kw):
        return {"name": name, "what": "tree", "seqs": B, "drafts": T, "len": L, "Hq": Hq, "Hkv": Hkv, "type": kind,
                "page": page, "ragged": False, "masked": T > 1, "lse": False, "behind": 0, **kw}

    return [
        # one decoded token far into a long context: launches and latency only
        rope("rope_one", 1, 28, 4, scaling="parts", factor=8.0, first=1048575),
        # a short video prompt: (t, h, w) position triples, Q and K as views of one fused projection
        rope("rope_clip", 20240, 28, 4, axes=3, fused=True),
        # the gradient of a long prompt's rotation, half of each head rotated, neighbouring pairs, scaled positions
        rope("rope_grad_256k", 262144, 32, 8, layout="interleaved", rot=64, scaling="linear", factor=4.0, inverse=True),
        # one decoded token of each of 32 sequences goes into the cache and comes back as it is held
        rows("store_32", "store", 32, "fp8", 8, 64),
        # a long prompt's keys and values go into the cache, padding rows among them, and come back as they are held
        rows("store_256k", "store", 262144, "int8", 8, 64, skip=0.01),
        # a short cached prefix read back for a further prefill
        rows("read_4k", "read", 4097, "fp4", 4, 16),
        # a long cached prefix read back
        rows("read_128k", "read", 131072, "fp8", 4, 64),
        # one token of one sequence over a short cache: latency
        tree("tree_one", 1, 1, 4096, 28, 4, "bf16", 64),
        # one token of each of 32 sequences of different lengths: ordinary batched decoding
        tree("decode_32", 32, 1, 32768, 32, 8, "fp8", 64, ragged=True),
        # 64 drafted tokens of one long sequence: the verification of a wide tree, LSE asked for
        tree("tree_128k", 1, 64, 131072, 28, 4, "bf16", 64, lse=True),
        # trees of different sizes over caches from empty to long, padding rows behind the last one
        tree("trees_ragged", 6, 64, 262144, 28, 4, "int8", 16, ragged=True, lse=True, behind=13),
        # the benchmark's length in four bits, a small tree
        tree("tree_1m", 1, 16, 1048576, 28, 4, "fp4", 256),
    ]


def draw(rng: random.Random):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    what = rng.choice(["rope", "store", "read", "tree", "tree", "tree"])
    Hq, Hkv = rng.choice(HEADS)
    if what == "rope":
        layout, rot = rng.choice(["half", "interleaved"]), rng.choice([32, 64, 96, 128, 128])
        scaling = rng.choice(["none", "linear", "ntk", "parts"])
        return {"what": what, "S": size(1, 200000), "Hq": Hq, "Hkv": Hkv, "layout": layout, "rot": rot,
                "scaling": scaling, "factor": 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                "axes": rng.choice([1, 1, 3]), "inverse": rng.random() < 0.3, "fused": rng.random() < 0.5,
                "first": rng.choice([0, rng.randint(1, 1 << 20)])}
    kind, page = rng.choice(["bf16", "fp8", "int8", "fp4"]), rng.choice([16, 32, 64, 128, 256])
    if what != "tree":
        return {"what": what, "rows": size(1, 200000), "type": kind, "Hkv": Hkv, "page": page,
                "skip": rng.choice([0.0, 0.02])}
    B, T = size(1, 64), rng.choice([1, 1, size(2, 64), size(2, 256)])
    most = min(1000000 // (B * Hkv) * 4, 200000000 // (B * Hq * T), 262144)
    return {"what": what, "seqs": B, "drafts": T, "len": size(1, max(2, most)), "Hq": Hq, "Hkv": Hkv, "type": kind,
            "page": page, "ragged": rng.random() < 0.6, "masked": rng.random() < 0.7, "lse": rng.random() < 0.5,
            "behind": rng.choice([0, rng.randint(1, 9)])}


def counts(c):
    """(cached tokens, drafted tokens) of every sequence of a tree case."""
    B, T, L = c["seqs"], c["drafts"], c["len"]
    if not c["ragged"]:
        return np.full(B, L), np.full(B, T)
    rng = np.random.default_rng([B, T, L])
    n = np.exp(rng.uniform(0, np.log(L + 1), B)).astype(np.int64)
    t = rng.integers(1, T + 1, B)
    n[0], t[0] = L, T
    if B > 2:
        n[1], t[2] = 0, max(1, T // 2)
    return n, t


def work(c):
    if c["what"] == "rope":
        heads = c["S"] * (c["Hq"] + c["Hkv"])
        return {"bytes": 4.0 * D * heads + 4.0 * c["S"] * c["axes"], "flops": 3.0 * c["rot"] * heads}
    held = 2.0 * (ROW[c["type"]] + (0 if c["type"] == "bf16" else 4))
    if c["what"] != "tree":
        once = c["rows"] * (c["Hkv"] * (4.0 * D + held) + 8)
        return {"bytes": once * (2 if c["what"] == "store" else 1), "flops": 4.0 * D * c["rows"] * c["Hkv"]}
    n, t = counts(c)
    pairs = float((t * n).sum() + (t * (t + 1) / 2).sum())
    return {"bytes": float(n.sum()) * c["Hkv"] * held + 4.0 * D * float(t.sum()) * (c["Hq"] + c["Hkv"]),
            "flops": 4.0 * D * c["Hq"] * pairs}


# ------------------------------------------------------------------ inputs
def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def keys_values(g, n, Hkv):
    """K and V [n, Hkv, 128] as a layer makes them: a few channels of K many times larger than the rest."""
    big = torch.where(torch.rand(Hkv, D, generator=g, device=DEV) < 0.03, 8.0, 1.0).to(torch.bfloat16)
    return normal(g, n, Hkv, D) * big, normal(g, n, Hkv, D)


def frequencies(c):
    """Radians a position of every pair."""
    r = c["rot"]
    theta = 1e6 if c["scaling"] != "ntk" else 1e6 * c["factor"] ** (r / (r - 2))
    f = theta ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "parts":                   # fast pairs as they are, slow ones interpolated
        g = np.clip((32768 * f / (2 * np.pi) - 1.0) / (32.0 - 1.0), 0, 1)
        f = ((1 - g) / c["factor"] + g) * f
    return f


def sections(c):
    """Pairs that take their position from t, h and w."""
    half = c["rot"] // 2
    return (half - 2 * (half * 3 // 8), half * 3 // 8, half * 3 // 8) if c["axes"] == 3 else (0, 0, 0)


def attention_factor(c):
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "parts" else 1.0


_ctx = None


def context():
    """The one handle that a program keeps."""
    global _ctx
    if _ctx is None:
        from paper_2504_16083_amd import mmi
        _ctx = mmi.Ctx(0)
    return _ctx


def prepare(c, seed):
    g = gen(seed)
    s = {"case": c}
    if c["what"] == "rope":
        S, Hq, Hkv = c["S"], c["Hq"], c["Hkv"]
        H = Hq + (2 if c["fused"] else 1) * Hkv
        if c["fused"]:
            a, b = normal(g, S, H, D), torch.zeros(S, H, D, device=DEV, dtype=torch.bfloat16)
            s["q"], s["k"], s["q_out"], s["k_out"] = a[:, :Hq], a[:, Hq:Hq + Hkv], b[:, :Hq], b[:, Hq:Hq + Hkv]
        else:
            s["q"], s["k"] = normal(g, S, Hq, D), normal(g, S, Hkv, D)
            s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
        p = torch.arange(S, device=DEV) + c["first"]
        if c["axes"] == 3:                        # frames of 14 x 14 tokens
            p = torch.stack([c["first"] + p // 196, c["first"] + p % 196 // 14, c["first"] + p % 14])
        s["pos"] = p.to(torch.int32)
        return s
    Hkv, page, kind = c["Hkv"], c["page"], c["type"]
    if c["what"] != "tree":
        n = c["rows"]
        n_pages = -(-n // page) + 3
        at = torch.randperm(n_pages, generator=g, device=DEV)
        i = torch.arange(n, device=DEV)
        s["slot"] = at[i // page] * page + i % page
        if n <= 64:                               # one token of each of several sequences
            s["slot"] = torch.randperm(n_pages * page, generator=g, device=DEV)[:n]
        s["slot"] = torch.where(torch.rand(n, generator=g, device=DEV) < c["skip"], -1, s["slot"])
        s["k"], s["v"] = keys_values(g, n, Hkv)
        s["k_out"], s["v_out"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        s["cache"] = pools(kind, n_pages, Hkv, page)
        if c["what"] == "read":
            for name in "kv":
                put(s["cache"], name, s["slot"], s.pop(name), kind, page)
        return s
    n, t = counts(c)
    need = -(-n // page)
    n_pages, most = int(need.sum()) + 2, max(1, int(need.max()))
    order = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32).cpu().numpy()
    table = np.full((len(n), most), -1, np.int32)
    first = np.concatenate([[0], np.cumsum(need)])
    for b in range(len(n)):
        table[b, :need[b]] = order[first[b]:first[b + 1]]
    s["pages"] = torch.from_numpy(table).to(DEV)
    s["cache"] = pools(kind, n_pages, Hkv, page)
    step = max(page, 262144 // page * page)
    for a in range(0, n_pages * page, step):
        slot = torch.arange(a, min(a + step, n_pages * page), device=DEV)
        k, v = keys_values(g, len(slot), Hkv)
        put(s["cache"], "k", slot, k, kind, page)
        put(s["cache"], "v", slot, v, kind, page)
    rows = int(t.sum()) + c["behind"]
    s["q"] = normal(g, rows, c["Hq"], D)
    s["k"], s["v"] = keys_values(g, rows, Hkv)
    s["o"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(c["Hq"], rows, device=DEV) if c["lse"] else None
    s["row_start"] = torch.from_numpy(np.concatenate([[0], np.cumsum(t)]).astype(np.int32)).to(DEV)
    s["length"] = torch.from_numpy(n.astype(np.int32)).to(DEV)
    s["mask"] = None
    if c["masked"]:                               # every drafted token: itself and its ancestors
        words = -(-c["drafts"] // 64)
        m = np.zeros((rows, words * 64), np.uint8)
        pick, r = np.random.default_rng(seed), 0
        for tb in t:
            for i in range(tb):
                m[r + i, i] = 1
                up = int(pick.integers(max(-1, i - 9), i)) if i else -1
                if up >= 0:
                    m[r + i] |= m[r + up]
            r += int(tb)
        s["mask"] = torch.from_numpy(np.packbits(m, axis=1, bitorder="little").view(np.int64)).to(DEV)
    return s


def pools(kind, n_pages, Hkv, page):
    """The cache's memory: codes of K and V, and their scale bytes."""
    made = {}
    for x in "kv":
        if kind == "bf16":
            made[x] = torch.zeros(n_pages, Hkv, page, D, device=DEV, dtype=torch.bfloat16)
            made[x + "_scale"] = None
        else:
            made[x] = torch.zeros(n_pages, Hkv, page, ROW[kind], device=DEV, dtype=torch.uint8)
            made[x + "_scale"] = torch.zeros(n_pages, Hkv, page, D // GROUP, device=DEV, dtype=torch.uint8)
    return made


# ------------------------------------------------------------------ plain forms
def power(e):
    """2^e in 32 bits, exactly (-126 <= e <= 127)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def encode(x, kind):
    """Codes and scale bytes of rows x [..., 128]."""
    x = x.float().unflatten(-1, (D // GROUP, GROUP))
    m, e = torch.frexp(x.abs().amax(-1))
    tm, te = math.frexp(TOP[kind])
    e = torch.where(m == 0, -126, e - te + (m > tm).to(torch.int32)).clamp(min=-126)
    y = (x * power(-e)[..., None]).flatten(-2)
    scale = (e + 127).to(torch.uint8)
    if kind == "fp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8), scale
    if kind == "int8":
        return torch.round(y).to(torch.int8).view(torch.uint8), scale
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
    a = y.abs()
    low, up = torch.bucketize(a, edges, right=False), torch.bucketize(a, edges, right=True)
    code = torch.where(low % 2 == 0, low, up).to(torch.uint8)      # between two codes: the even one
    code = code | (torch.signbit(y).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def decode(code, scale, kind):
    """Values [..., 128] of codes and scale bytes, in 32 bits."""
    if kind == "bf16":
        return code.float()
    if kind == "fp8":
        y = code.view(torch.float8_e4m3fn).float()
    elif kind == "int8":
        y = code.view(torch.int8).float()
    else:
        table = torch.tensor(FP4 + [-x for x in FP4], device=code.device)
        y = torch.stack([table[(code & 15).long()], table[(code >> 4).long()]], -1).flatten(-2)
    return y * power(scale.to(torch.int32) - 127).repeat_interleave(GROUP, -1)


def put(cache, name, slot, rows, kind, page):
    """rows [n, Hkv, 128] into the pool `name` at the slots (-1: nowhere)."""
    here = slot >= 0
    p, r = (slot // page)[here], (slot % page)[here]
    if kind == "bf16":
        cache[name][p, :, r] = rows[here]
    else:
        cache[name][p, :, r], cache[name + "_scale"][p, :, r] = encode(rows[here], kind)


def take(cache, name, slot, kind, page):
    """What the pool `name` holds at the slots (-1: zeros), [n, Hkv, 128] bfloat16."""
    at = slot.clamp(min=0)
    p, r = at // page, at % page
    scale = cache[name + "_scale"]
    rows = decode(cache[name][p, :, r], None if scale is None else scale[p, :, r], kind)
    return (rows * (slot >= 0)[:, None, None]).to(torch.bfloat16)


def rotate(x, cos, sin, c):
    r = c["rot"]
    y = x.float()
    if c["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
    u, v = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([u, v], -1) if c["layout"] == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1).to(torch.bfloat16)


def plain_rope(s):
    c = s["case"]
    pos = s["pos"].double()
    if c["axes"] == 3:
        pos = pos.repeat_interleave(torch.tensor(sections(c), device=DEV), 0).T
    else:
        pos = pos[:, None]
    angle = pos * torch.from_numpy(frequencies(c)).to(DEV)
    m = attention_factor(c)
    cos, sin = (torch.cos(angle) * m).float()[:, None], (torch.sin(angle) * (-m if c["inverse"] else m)).float()[:, None]
    return {"q": rotate(s["q"], cos, sin, c), "k": rotate(s["k"], cos, sin, c)}


def plain_tree(s):
    c = s["case"]
    kind, page, Hq, Hkv = c["type"], c["page"], c["Hq"], c["Hkv"]
    B, T, g = c["seqs"], c["drafts"], Hq // Hkv
    cache, table = s["cache"], s["pages"].clamp(min=0).long()
    L = table.shape[1] * page

    def cached(name):                             # [B, Hkv, L, 128]
        scale = cache[name + "_scale"]
        x = decode(cache[name][table], None if scale is None else scale[table], kind)
        return x.transpose(1, 2).flatten(2, 3)

    start, stop = s["row_start"][:-1].long(), s["row_start"][1:].long()
    t = torch.arange(T, device=DEV)
    row = start[:, None] + t
    live = row < stop[:, None]                    # [B, T]
    row = torch.where(live, row, 0)
    k = torch.cat([cached("k"), s["k"][row].float().transpose(1, 2)], 2)
    v = torch.cat([cached("v"), s["v"][row].float().transpose(1, 2)], 2)
    q = s["q"][row].float().unflatten(2, (Hkv, g)).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [B, Hkv, g T, 128]
    seen = (torch.arange(L, device=DEV) < s["length"][:, None])[:, None].expand(B, T, L)
    if s["mask"] is None:
        among = (t <= t[:, None]).expand(B, T, T)
    else:
        among = (s["mask"][row][..., t // 64] >> (t % 64) & 1).bool()
    seen = torch.cat([seen, among & live[:, None]], 2)[:, None]                           # [B, 1, T, L + T]
    score = (q @ k.transpose(2, 3)) / math.sqrt(D)
    score = score.unflatten(2, (g, T)).masked_fill(~seen[:, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    o = p.flatten(2, 3) @ v
    o = o.unflatten(2, (g, T)) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)                                            # [B, T, Hq, 128]
    out = {"o": s["o"].clone()}
    out["o"][row[live]] = o[live].to(torch.bfloat16)
    if s["lse"] is not None:
        lse = (top + torch.log(total)).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3)      # [B, T, Hq]
        out["lse"] = s["lse"].clone()
        out["lse"][:, row[live]] = lse[live].T
    return out


# ------------------------------------------------------------------ one pass
def handles(s):
    """What a program keeps of the library for this state: its configuration, cache and batch."""
    from paper_2504_16083_amd import cache as KV

    c = s["case"]
    if c["what"] == "rope":
        s["cfg"] = KV.RopeCfg(rot_dim=c["rot"], layout=c["layout"], theta=1e6, scaling=c["scaling"],
                              factor=c["factor"], orig_len=32768, beta_fast=32.0, beta_slow=1.0, sections=sections(c))
        return
    p = s["cache"]
    s["pool"] = KV.Cache(c["type"], p["k"], p["v"], p["k_scale"], p["v_scale"])
    if c["what"] == "tree":
        s["tree"] = KV.Tree(s["row_start"], s["length"], s["pages"], mask=s["mask"], max_rows=c["drafts"],
                            max_len=c["len"])
        s["ws"] = torch.empty(KV.mmi_tree_workspace(context(), s["pool"], s["tree"], c["Hq"], len(s["q"])),
                              device=DEV, dtype=torch.uint8)


def run(s):
    c = s["case"]
    what = c["what"]
    if own:
        from paper_2504_16083_amd import cache as KV

        if "cfg" not in s and "pool" not in s:
            handles(s)
        ctx = context()
        if what == "rope":
            KV.mmi_rope(ctx, s["cfg"], s["q"], s["k"], pos=s["pos"], q_out=s["q_out"], k_out=s["k_out"],
                        inverse=c["inverse"])
            return {"q": s["q_out"], "k": s["k_out"]}
        if what == "tree":
            KV.mmi_tree_attention(ctx, s["pool"], s["tree"], s["q"], s["k"], s["v"], s["o"], lse=s["lse"],
                                  workspace=s["ws"])
            return {"o": s["o"], **({} if s["lse"] is None else {"lse": s["lse"]})}
        if what == "store":
            KV.mmi_cache_write(ctx, s["pool"], s["k"], s["v"], s["slot"])
        KV.mmi_cache_read(ctx, s["pool"], s["slot"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if what == "rope":
        return plain_rope(s)
    if what == "tree":
        return plain_tree(s)
    if what == "store":
        put(s["cache"], "k", s["slot"], s["k"], c["type"], c["page"])
        put(s["cache"], "v", s["slot"], s["v"], c["type"], c["page"])
    return {x: take(s["cache"], x, s["slot"], c["type"], c["page"]) for x in "kv"}


# ------------------------------------------------------------------ the definition in 64 bits
def two_to(e):
    """2^e in 64 bits for whole e, from a table (a device's power function may be off by a rounding)."""
    table = torch.tensor([2.0 ** i for i in range(-160, 161)], dtype=torch.float64, device=e.device)
    return table[e.long() + 160]


def held(x, kind):
    """What a cache of this type holds for rows x, from the grid of the type's codes."""
    if kind == "bf16":
        return x.double()
    y = x.double().reshape(*x.shape[:-1], D // GROUP, GROUP)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / TOP[kind])).clamp(min=-126)
    e = torch.where(top > TOP[kind] * two_to(e), e + 1, e)         # the logarithm may be off by a rounding
    e = torch.where((top <= TOP[kind] * two_to(e - 1)) & (e > -126), e - 1, e)
    y = y / two_to(e)
    if kind == "int8":
        step = torch.ones_like(y)
    else:                                         # spacing of the codes around y: 3 or 1 bits behind the leading one
        bits, low = (3, -6) if kind == "fp8" else (1, 0)
        step = two_to(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** low))) - bits)
    return (torch.round(y / step) * step * two_to(e)).reshape(x.shape)


def values(code, scale, kind):
    """What codes and scale bytes stand for, from their bits."""
    if kind == "bf16":
        return code.double()
    u = code.long()
    if kind == "int8":
        y = torch.where(u > 127, u - 256, u).double()
    else:
        if kind == "fp4":
            u = torch.stack([u % 16, u // 16], -1).reshape(*u.shape[:-1], D)
        m, bias = (3, 7) if kind == "fp8" else (1, 1)
        sign = torch.where(u >= (128 if kind == "fp8" else 8), -1.0, 1.0).double()
        u = u % (128 if kind == "fp8" else 8)
        ex, frac = u >> m, (u % (1 << m)).double() / (1 << m)
        y = sign * torch.where(ex > 0, (1 + frac) * two_to(ex - bias), frac * 2.0 ** (1 - bias))
    return y * two_to(scale.long() - 127).repeat_interleave(GROUP, -1)


def exact(c, seed):
    s = prepare(c, seed)
    if c["what"] == "rope":
        f = frequencies(c)
        sec = sections(c)
        axis = [0] * len(f) if c["axes"] == 1 else [0] * sec[0] + [1] * sec[1] + [2] * sec[2]
        pos = s["pos"].double().reshape(c["axes"], -1)
        turn = torch.stack([pos[a] * float(x) for a, x in zip(axis, f)], 1)
        if c["inverse"]:
            turn = -turn
        w = torch.polar(torch.full_like(turn, attention_factor(c)), turn)[:, None]

        def turned(x):
            y = x.double()
            h = c["rot"] // 2
            i = torch.arange(h, device=DEV)
            i, j = (i, i + h) if c["layout"] == "half" else (2 * i, 2 * i + 1)
            z = torch.complex(y[..., i], y[..., j]) * w
            y[..., i], y[..., j] = z.real, z.imag
            return y

        return {"q": turned(s["q"]), "k": turned(s["k"])}
    kind, page = c["type"], c["page"]
    if c["what"] == "store":
        keep = (s["slot"] >= 0).double()[:, None, None]
        return {x: held(s[x], kind) * keep for x in "kv"}
    p = s["cache"]

    def rows(name, slot, heads):
        scale = p[name + "_scale"]
        a, r = slot // page, slot % page
        return values(p[name][a, heads, r], None if scale is None else scale[a, heads, r], kind)

    if c["what"] == "read":
        every = torch.arange(c["Hkv"], device=DEV)[None]
        got = {}
        for x in "kv":
            v = rows(x, s["slot"].clamp(min=0)[:, None], every)
            got[x] = v * (s["slot"] >= 0).double()[:, None, None]
        return got
    n, t = counts(c)
    g = c["Hq"] // c["Hkv"]
    if float((n * t).sum()) * c["Hq"] > 4e9:
        return None
    o = s["o"].double()
    lse = None if s["lse"] is None else s["lse"].double()
    r0 = 0
    for b in range(len(n)):
        nb, tb = int(n[b]), int(t[b])
        i = torch.arange(nb, device=DEV)
        slot = s["pages"][b].long()[i // page] * page + i % page
        mask = torch.tril(torch.ones(tb, tb, device=DEV, dtype=torch.bool))
        if s["mask"] is not None:
            bits = np.unpackbits(s["mask"][r0:r0 + tb].cpu().numpy().view(np.uint8), axis=1, bitorder="little")
            mask = torch.from_numpy(bits[:, :tb].astype(bool)).to(DEV)
        for h in range(c["Hkv"]):
            k = torch.cat([rows("k", slot, h), s["k"][r0:r0 + tb, h].double()])
            v = torch.cat([rows("v", slot, h), s["v"][r0:r0 + tb, h].double()])
            for x in range(h * g, (h + 1) * g):
                z = s["q"][r0:r0 + tb, x].double() @ k.T * D ** -0.5
                z[:, nb:][~mask] = -math.inf
                o[r0:r0 + tb, x] = torch.softmax(z, 1) @ v
                if lse is not None:
                    lse[x, r0:r0 + tb] = torch.logsumexp(z, 1)
        r0 += tb
    return {"o": o} if lse is None else {"o": o, "lse": lse}
