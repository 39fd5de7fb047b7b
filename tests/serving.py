"""Shared by the tests of the operators around the prefill: caches made and
read on the host, batches of sequences, and the comparison with the oracle."""
import numpy as np
import torch

from oracle import serving as OS
from paper_2504_16083_amd import cache as KV

D = 128
HALF_STEP = 2.0 ** -8            # rounding to bfloat16, relative to the value


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def fill(kind, n_pages, Hkv, page, seed, device="cuda"):
    """A cache whose every row holds something: random codes with random scales, so that reading it needs no
    write to have worked. Returns (Cache, K, V values [slots, Hkv, 128] in fp64)."""
    g = torch.Generator().manual_seed(seed)
    shape = (n_pages, Hkv, page)
    vals, mem = [], []
    for _ in "kv":
        if kind == "bf16":
            t = torch.randn(*shape, D, generator=g).to(torch.bfloat16)
            vals.append(f64(t))
            mem.append((t, None))
            continue
        if kind == "fp4":
            code = torch.randint(0, 16, (*shape, D), generator=g)
            packed = (code[..., 0::2] | code[..., 1::2] << 4).to(torch.uint8)
        else:
            code = torch.randint(0, 256, (*shape, D), generator=g)
            code = torch.where(code & 127 == 127, 0, code) if kind == "fp8" else torch.where(code == 128, 0, code)
            packed = code.to(torch.uint8)
        low = {"fp8": -9, "int8": -6, "fp4": -2}[kind]          # values of about one
        scale = torch.randint(127 + low, 130 + low, (*shape, 4), generator=g)
        vals.append(OS.value(code.numpy(), scale.numpy(), kind))
        mem.append((packed, scale.to(torch.uint8)))
    (k, ks), (v, vs) = mem
    up = lambda t: None if t is None else t.to(device)  # noqa: E731
    cache = KV.Cache(kind, up(k), up(v), up(ks), up(vs))
    rows = [x.transpose(0, 2, 1, 3).reshape(n_pages * page, Hkv, D) for x in vals]
    return cache, rows[0], rows[1]


class Batch:
    """Sequences of `lens` cached and `drafts` drafted tokens over a filled cache, as the call takes them and
    as the oracle does. mask: None (chain), "tree", or a function (sequence, i, j) -> bool."""

    def __init__(self, kind, lens, drafts, Hq, Hkv, page, seed=0, mask=None, behind=0, words=None, max_len=None,
                 max_rows=None, spare=3):
        rng = np.random.default_rng(seed)
        self.lens, self.drafts, self.Hq, self.Hkv = lens, drafts, Hq, Hkv
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + spare
        self.cache, self.K, self.V = fill(kind, n_pages, Hkv, page, seed)
        order = rng.permutation(n_pages)
        cols = max(1, max(need, default=0))
        self.max_len = max(lens, default=0) if max_len is None else max_len
        cols = max(cols, -(-self.max_len // page))
        table = np.full((len(lens), cols), -1, np.int32)
        self.slots, at = [], 0
        for b, n in enumerate(lens):
            table[b, :need[b]] = order[at:at + need[b]]
            at += need[b]
            i = np.arange(n)
            self.slots.append(table[b][i // page].astype(np.int64) * page + i % page)
        self.n = sum(drafts) + behind
        g = torch.Generator().manual_seed(seed + 1)
        mk = lambda h: torch.randn(self.n, h, D, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
        self.q, self.k, self.v = mk(Hq), mk(Hkv), mk(Hkv)
        self.max_rows = max(1, max(drafts, default=1)) if max_rows is None else max_rows
        self.start = np.concatenate([[0], np.cumsum(drafts)]).astype(np.int64)
        self.sees = []                                  # [T, T] of every sequence
        for b, t in enumerate(drafts):
            m = np.tril(np.ones((t, t), bool))
            if mask == "tree":
                m = np.zeros((t, t), bool)
                for i in range(t):
                    up = int(rng.integers(-1, i)) if i else -1
                    if up >= 0:
                        m[i] = m[up]
                    m[i, i] = True
            elif callable(mask):
                m = np.array([[mask(b, i, j) for j in range(t)] for i in range(t)], bool).reshape(t, t)
            self.sees.append(m)
        bits = None
        if mask is not None:
            words = -(-self.max_rows // 64) if words is None else words
            all_bits = np.zeros((self.n, words * 64), np.uint8)
            for b, t in enumerate(drafts):
                all_bits[self.start[b]:self.start[b] + t, :t] = self.sees[b]
            bits = torch.from_numpy(np.packbits(all_bits, axis=1, bitorder="little").view(np.int64)).cuda()
        self.table = table
        self.tree = KV.Tree(torch.from_numpy(self.start.astype(np.int32)).cuda(),
                            torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.from_numpy(table).cuda(),
                            mask=bits, max_rows=self.max_rows, max_len=self.max_len)
        self.scale = D ** -0.5

    def outputs(self):
        return (torch.full((self.n, self.Hq, D), 7.0, dtype=torch.bfloat16, device="cuda"),
                torch.full((self.Hq, self.n), 7.0, device="cuda"))

    def workspace(self, ctx):
        return torch.empty(KV.mmi_tree_workspace(ctx, self.cache, self.tree, self.Hq, self.n), dtype=torch.uint8,
                           device="cuda")

    def run(self, ctx, lse=True, stream=None):
        o, l = self.outputs()
        KV.mmi_tree_attention(ctx, self.cache, self.tree, self.q, self.k, self.v, o, self.workspace(ctx),
                              lse=l if lse else None, stream=stream)
        torch.cuda.synchronize()
        return o, l

    def check(self, o, lse=None, rows=None, visible=None):
        """Every row (or those (sequence, token) of `rows`) against the oracle; visible(b) -> which cached
        tokens of b exist."""
        q, k, v, o = f64(self.q), f64(self.k), f64(self.v), f64(o)
        g = self.Hq // self.Hkv
        for b, t in enumerate(self.drafts):
            cached = np.ones(self.lens[b], bool) if visible is None else visible(b)
            r0 = self.start[b]
            for h in range(self.Hkv):
                kk = np.concatenate([self.K[self.slots[b], h], k[r0:r0 + t, h]])
                vv = np.concatenate([self.V[self.slots[b], h], v[r0:r0 + t, h]])
                for i in range(t):
                    if rows is not None and (b, i) not in rows:
                        continue
                    sees = np.concatenate([cached, self.sees[b][i]])
                    for x in range(h * g, (h + 1) * g):
                        want, l, spread, bound = OS.attend(q[r0 + i, x], kk, vv, sees, self.scale)
                        compare(o[r0 + i, x], want, spread, bound, f"sequence {b} row {i} head {x}")
                        if lse is not None:
                            got = float(lse[x, r0 + i])
                            if not np.isfinite(l):
                                assert got == l or (np.isnan(got) and np.isnan(l)), (b, i, x, got, l)
                            else:
                                # the scores' own error, and sums of n fp32 terms in short chains
                                tol = score_error(bound) + 2.0 ** -20 + 2.0 ** -24 * (abs(l) + len(sees) / 32 + 64)
                                assert abs(got - l) <= tol, (b, i, x, got, l, tol)


def score_error(bound):
    """Error of a score in fp32: 128 products added one after another, the scale's two roundings."""
    return bound * 132 * 2.0 ** -24


def compare(got, want, spread, bound, what):
    """|o - oracle|: the weights are off by their rounding to bfloat16 (half a step), twice the scores' error
    and 2^-20 for the exponentials and sums, which moves o by that times the spread of V around it (and, as the
    weights are normalised after rounding, 1% more of that); the output's own rounding is half a step of it."""
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    assert np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)]), what
    got, want, spread = got[finite], want[finite], spread[finite]
    tol = spread * 1.01 * (HALF_STEP + 2 * score_error(bound) + 2.0 ** -20) + np.abs(want) * HALF_STEP + 1e-30
    off = np.abs(got - want) - tol * (1 + HALF_STEP)
    assert off.max(initial=-1.0) <= 0, f"{what}: off by {np.abs(got - want).max()} at most {tol[off.argmax()]} allowed"
