"""Attention of drafted tokens where the row count or the place of a key picks
other code: more than 32 rows a head (both tiles), chunks' first keys."""
import numpy as np
import pytest
import torch

from serving import Batch, D, f64

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "fp8", "int8", "fp4"]
WIDE = [(16, 3), (16, 7), (43, 7)]                       # drafts, heads a KV head: 48, 112, 301 rows
ROWS = [(1, 4), (3, 7)] + WIDE                           # and 4, 21


@pytest.fixture(scope="module")
def ctx():
    from paper_2504_16083_amd import mmi
    return mmi.Ctx(0)


@pytest.mark.parametrize("T,g", ROWS)
@pytest.mark.parametrize("L", [20, 64, 300, 9000])
def test_infinities_in_cached_values(ctx, T, g, L):
    """Every row sees a cached token: an infinity in its V makes that channel infinite, wherever the token lies in
    its chunk, and both infinities in one channel a NaN. The other channels are as they were."""
    b = Batch("bf16", [L], [T], g, 1, 16, seed=L)
    for token, d, value in [(0, 5, np.inf), (19, 6, -np.inf), (L - 1, 7, np.inf), (L // 2, 8, np.inf), (0, 90, np.inf),
                            (L - 1, 90, -np.inf)] + [(c, d, -np.inf) for d, c in enumerate(range(128, min(L, 4000), 128), 20)]:
        s = int(b.slots[0][token])
        b.V[s, 0, d] = value
        b.cache.v[s // 16, 0, s % 16, d] = value
    with np.errstate(all="ignore"):
        b.check(*b.run(ctx), rows={(0, 0), (0, T - 1)})


def both(ctx, b):
    """o and lse of a batch; without the lse o is the same."""
    o, lse = b.run(ctx)
    assert torch.equal(b.run(ctx, lse=False)[0].view(torch.int16), o.view(torch.int16))      # NaN too
    return o, lse


def some(b, s=0):
    t = b.drafts[s]
    return {(s, i) for i in {0, t // 2, t - 1} if t}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,g", WIDE)
@pytest.mark.parametrize("L", [1, 37, 300, 9000])
def test_memory_behind_the_last_token(ctx, kind, T, g, L):
    """What lies behind a sequence's last token in its page, and in pages of others, is NaN in every group."""
    b = Batch(kind, [L, 18], [T, 2], g, 1, 64, seed=L)
    used = np.zeros(b.cache.n_pages * 64, bool)
    for s in b.slots:
        used[s] = True
    free = torch.from_numpy(np.flatnonzero(~used)).cuda()
    for t in (b.cache.k, b.cache.v) if kind == "bf16" else (b.cache.k_scale, b.cache.v_scale):
        t[free // 64, :, free % 64] = float("nan") if kind == "bf16" else 255
    b.check(*both(ctx, b), rows=some(b) | some(b, 1))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,g", WIDE)
@pytest.mark.parametrize("L,page,bad", [(300, 16, (0, 7, 18)), (300, 16, range(19)), (300, 64, (4,)), (9000, 64, (0, 1, 2, 77, 140)),
                                        (9000, 16, tuple(range(3, 562, 9)))])
def test_bad_pages(ctx, kind, T, g, L, page, bad):
    """Page numbers outside the cache, at the ends of it and in the middle: their tokens do not exist."""
    b = Batch(kind, [L], [T], g, 1, page, seed=L)
    there = np.ones(L, bool)
    for i, p in enumerate(bad):
        b.tree.pages[0, p] = (b.cache.n_pages, -1, 2 ** 31 - 1, -(2 ** 31))[i % 4]
        there[p * page:(p + 1) * page] = False
    b.check(*both(ctx, b), rows=some(b), visible=lambda s: there)


@pytest.mark.parametrize("T,g", WIDE)
def test_lengths_and_rows_out_of_range(ctx, T, g):
    """Lengths are cut to [0, max_len], rows to n_rows and max_rows; what is behind them is left alone."""
    b = Batch("int8", [500, 40, 64], [T, 2, T], g, 1, 16, seed=5, behind=2)
    good = [x.clone() for x in both(ctx, b)]
    b.tree.length.copy_(torch.tensor([10 ** 9, 40, -5], dtype=torch.int32))
    o, lse = both(ctx, b)
    assert torch.equal(o[:T + 2], good[0][:T + 2]) and torch.equal(lse[:, :T + 2], good[1][:, :T + 2])
    b.lens[2], b.slots[2] = 0, b.slots[2][:0]
    b.check(o, lse, rows=some(b, 2))
    b.tree.length.copy_(torch.tensor([500, 40, 0], dtype=torch.int32))
    b.tree.row_start.copy_(torch.tensor([-3, T, T + 2, 10 ** 6], dtype=torch.int32))
    o, lse = both(ctx, b)
    assert torch.equal(o[:T], good[0][:T])
    assert (o[T + 2:T + 2 + T] != 7).any() and (o[T + 2 + T:] == 7).all() and (lse[:, T + 2 + T:] == 7).all()


@pytest.mark.parametrize("T,g", WIDE)
def test_rows_that_see_nothing(ctx, T, g):
    b = Batch("bf16", [0, 5], [T, 3], g, 1, 16, mask=lambda s, i, j: i % 3 != 2 and j < i)
    o, lse = both(ctx, b)
    b.check(o, lse)
    assert (o[0] == 0).all() and (lse[:, 0] == -np.inf).all() and (o[2] == 0).all() and (o[5] == 0).all()


@pytest.mark.parametrize("T,g", [(16, 7), (43, 7)])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_not_finite_drafts(ctx, T, g, value):
    """With other chunks beside the one that has the drafted tokens."""
    b = Batch("fp8", [700], [T], g, 1, 16, seed=4, mask="tree")
    for j, d in ((3, 0), (T // 2, 127), (T - 1, 64)):
        b.v[j, 0, d] = value
    with np.errstate(all="ignore"):
        b.check(*both(ctx, b))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,g", WIDE)
def test_scores_that_grow(ctx, kind, T, g):
    """Within every chunk (640 tokens here) scores rise 17 times by more than the running maximum is let fall behind,
    at places that go through the halves of the stages, and as high in every chunk. Rows follow it by different
    steps, so that it moves in some rows of a tile and not in others."""
    from paper_2504_16083_amd import cache as KV
    L, page, H = 20000 if g == 7 and T == 43 else 40000, 64, 4
    b = Batch(kind, [L], [T], g * H, H, page, seed=T + g)
    rng = np.random.default_rng(1)
    u = torch.from_numpy(rng.choice([-1.0, 1.0], D)).to(torch.bfloat16).cuda()
    at = np.arange(5, L, 37)
    height = torch.from_numpy(0.8 * (at % 640 // 37)).to(torch.bfloat16).cuda()
    slot = torch.from_numpy(b.slots[0][at]).cuda()
    k, v = (torch.empty(len(at), H, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    KV.mmi_cache_read(ctx, b.cache, slot, k, v)
    k.copy_(k * 0.1 + height[:, None, None] * u)
    KV.mmi_cache_write(ctx, b.cache, k, v, slot)
    KV.mmi_cache_read(ctx, b.cache, slot, k, v)              # as it is held
    b.K[b.slots[0][at]], b.V[b.slots[0][at]] = f64(k), f64(v)
    step = torch.tensor([1.0, 0.4, 0.05, -1.0], device="cuda").to(torch.bfloat16)
    b.q.copy_(b.q * 0.1 + step[torch.arange(T, device="cuda") % 4][:, None, None] * u)
    b.check(*both(ctx, b), rows={(0, i) for i in (0, 1, 2, 3, T - 1)})


def test_strides(ctx):
    """q, k, v as views of a fused projection, o as a view of a wider buffer, pages among those of other layers."""
    from paper_2504_16083_amd import cache as KV
    for T, g in WIDE:
        b = Batch("fp8", [700, 200], [T, 3], 2 * g, 2, 32, seed=10, mask="tree", words=3)
        want, _ = b.run(ctx)
        b.check(want, rows=some(b) | some(b, 1))
        H = 2 * g
        fused = torch.zeros(b.n, H + 8, D, dtype=torch.bfloat16, device="cuda")
        fused[:, 1:H + 1], fused[:, H + 2:H + 4], fused[:, H + 6:] = b.q, b.k, b.v
        wide = torch.full((b.n, H + 3, D), 7.0, dtype=torch.bfloat16, device="cuda")
        c = b.cache
        mem = torch.zeros(c.n_pages, 3, 2, 2, 32, 128, dtype=torch.uint8, device="cuda")
        sc = torch.zeros(c.n_pages, 3, 2, 2, 32, 4, dtype=torch.uint8, device="cuda")
        mem[:, 1, 0], mem[:, 1, 1], sc[:, 1, 0], sc[:, 1, 1] = c.k, c.v, c.k_scale, c.v_scale
        c = KV.Cache("fp8", mem[:, 1, 0], mem[:, 1, 1], sc[:, 1, 0], sc[:, 1, 1])
        KV.mmi_tree_attention(ctx, c, b.tree, fused[:, 1:H + 1], fused[:, H + 2:H + 4], fused[:, H + 6:], wide[:, 2:H + 2],
                              b.workspace(ctx))
        assert torch.equal(wide[:, 2:H + 2], want) and (wide[:, :2] == 7).all() and (wide[:, H + 2:] == 7).all()


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_offsets_past_32_bits(ctx, kind):
    """Pages whose place in memory lies beyond 2^32 bytes, for codes and, with a stride of their own, scales."""
    from paper_2504_16083_amd import cache as KV
    b = Batch(kind, [600], [16], 14, 2, 256, seed=12)
    want = b.run(ctx)[0]
    c, n, many = b.cache, b.cache.n_pages, 40000
    def far(t, stride):                                          # the last pages of `many`, `stride` apart
        room = torch.empty(many * stride, dtype=t.dtype, device="cuda")
        view = room.as_strided((many, *t.shape[1:]), (stride, *t.stride()[1:]))
        view[-n:] = t
        return view
    page = 2 * 256 * D
    pools = [far(c.k, page), far(c.v, page)] if kind == "bf16" else [far(t, 120000) for t in (c.k, c.v, c.k_scale, c.v_scale)]
    pages = torch.where(b.tree.pages >= 0, b.tree.pages + many - n, -1)
    tree = KV.Tree(b.tree.row_start, b.tree.length, pages, max_rows=b.max_rows, max_len=b.max_len)
    o, _ = b.outputs()
    KV.mmi_tree_attention(ctx, KV.Cache(kind, *pools), tree, b.q, b.k, b.v, o, b.workspace(ctx))
    assert torch.equal(o, want)


@pytest.mark.parametrize("T,g", WIDE)
def test_replays_and_repeats(ctx, T, g):
    """A captured call replayed with other lengths and rows within its bounds, between eager ones."""
    from paper_2504_16083_amd import cache as KV
    b = Batch("fp4", [9000, 900], [T, 5], 2 * g, 2, 64, seed=1)
    first = b.run(ctx)
    graph, o, ws = torch.cuda.CUDAGraph(), torch.zeros_like(first[0]), b.workspace(ctx)
    with torch.cuda.graph(graph):
        KV.mmi_tree_attention(ctx, b.cache, b.tree, b.q, b.k, b.v, o, ws)
    for lens, start in (([9000, 900], [0, T, T + 5]), ([17, 0], [0, 1, T]), ([0, 900], [0, 3, T]), ([8999, 64], [0, T, T]),
                        ([9000, 900], [0, T, T + 5])):
        b.tree.length.copy_(torch.tensor(lens, dtype=torch.int32))
        b.tree.row_start.copy_(torch.tensor(start, dtype=torch.int32))
        o.fill_(7.0)
        graph.replay()
        eager = b.run(ctx)
        torch.cuda.synchronize()
        assert torch.equal(o, eager[0])
    assert torch.equal(eager[0], first[0]) and torch.equal(eager[1], first[1])
