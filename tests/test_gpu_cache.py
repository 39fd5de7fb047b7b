"""Writing the paged cache and reading it back on the GPU: codes, scales and
values are those of the oracle, exactly."""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from serving import D, f64, fill

pytestmark = pytest.mark.gpu
KINDS = ["bf16", "fp8", "int8", "fp4"]


@pytest.fixture(scope="module")
def ctx():
    from paper_2504_16083_amd import mmi
    return mmi.Ctx(0)


def empty(kind, n_pages, Hkv, page, value=0x5a):
    """A cache with a pattern in every byte."""
    from paper_2504_16083_amd import cache as KV
    c = KV.Cache.empty(kind, n_pages, Hkv, page)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(value)
    return c


def codes(cache, name, slot, h):
    """(codes [128], scale bytes [4]) at a slot, as whole numbers."""
    p, r = divmod(int(slot), cache.page)
    row = getattr(cache, name)[p, h, r].cpu()
    if cache.type == "fp4":
        row = torch.stack([row & 15, row >> 4], -1).flatten()
    return row.numpy().astype(np.int64), getattr(cache, name + "_scale")[p, h, r].cpu().numpy().astype(np.int64)


def rows(n, H, seed):
    """Rows with the values that matter: wide ranges, ties, zeros of both signs, powers of two and the largest
    codes themselves."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, H, D, generator=g) * torch.exp(torch.randn(n, H, 1, generator=g) * 4)
    x[0] = torch.arange(-64, 64) * 0.25
    if n > 1:
        x[1, :, ::2] = 0.0
        x[1, :, 1::4] = -0.0
    if n > 2:
        x[2] = torch.exp2(torch.randint(-12, 12, (H, D), generator=g).float())
    if n > 3:
        x[3] = torch.randint(-127, 128, (H, D), generator=g).float() / 2
    if n > 4:
        x[4] = torch.tensor([448.0, 127.0, 6.0, 0.25, 0.75, 1.75, 2.5, 5.0] * 16)
    return x.to(torch.bfloat16).cuda()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page,Hkv,n", [(16, 1, 1), (32, 3, 7), (64, 8, 33), (256, 4, 130)])
def test_write_and_read(ctx, kind, page, Hkv, n):
    from paper_2504_16083_amd import cache as KV
    n_pages = -(-n // page) + 2
    c = empty(kind, n_pages, Hkv, page)
    before = [None if t is None else t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)]
    k, v = rows(n, Hkv, 1), rows(n, Hkv, 2)
    slot = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(3))[:n]
    if n > 3:
        slot[3] = -1
    if n > 6:
        slot[5], slot[6] = n_pages * page, -(2 ** 62)          # behind the last page, far before the first
    KV.mmi_cache_write(ctx, c, k, v, slot.cuda())
    ko, vo = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    KV.mmi_cache_read(ctx, c, slot.cuda(), ko, vo)
    torch.cuda.synchronize()
    written = np.zeros(n_pages * page, bool)
    for i in range(n):
        s = int(slot[i])
        if not 0 <= s < n_pages * page:
            assert (ko[i] == 0).all() and (vo[i] == 0).all()
            continue
        written[s] = True
        for name, x, out in (("k", k, ko), ("v", v, vo)):
            if kind == "bf16":
                assert torch.equal(out[i].view(torch.int16), x[i].view(torch.int16))
                continue
            for h in range(Hkv):
                want, scale = OS.quantise(f64(x[i, h]), kind)
                got, got_scale = codes(c, name, s, h)
                assert np.array_equal(got_scale, scale), (i, h, got_scale, scale)
                if kind == "fp4" or kind == "fp8":      # a zero of either sign is zero
                    g = OS.grid(kind)
                    assert np.array_equal(g[got], g[want]), (i, h, got, want)
                else:
                    assert np.array_equal(got & 255, want & 255), (i, h)
                assert np.array_equal(f64(out[i, h]), OS.value(want, scale, kind))
    # nothing but the named slots has changed
    for t, b in zip((c.k, c.v, c.k_scale, c.v_scale), before):
        if t is not None:
            a, b = (x.view(torch.uint8).transpose(1, 2).reshape(n_pages * page, -1).cpu() for x in (t, b))
            assert torch.equal(a[~torch.from_numpy(written)], b[~torch.from_numpy(written)])


@pytest.mark.parametrize("kind", KINDS)
def test_every_code_and_scale_reads_back(ctx, kind):
    """Random codes with random scales (written by the host): what is read is what they stand for."""
    from paper_2504_16083_amd import cache as KV
    c, K, V = fill(kind, 20, 2, 32, 5)
    slot = torch.randperm(640, generator=torch.Generator().manual_seed(1))
    slot[7] = slot[8]                                            # a slot may repeat
    ko, vo = (torch.empty(640, 2, D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    KV.mmi_cache_read(ctx, c, slot.cuda(), ko, vo)
    assert np.array_equal(f64(ko), K[slot.numpy()]) and np.array_equal(f64(vo), V[slot.numpy()])


@pytest.mark.parametrize("kind", ["fp8", "int8", "fp4"])
def test_not_finite(ctx, kind):
    from paper_2504_16083_amd import cache as KV
    c = empty(kind, 1, 1, 16)
    k = rows(4, 1, 9)
    k[1, 0, 37] = float("inf")
    k[2, 0, 3], k[2, 0, 100] = float("nan"), float("-inf")
    v = k.flip(0).contiguous()
    slot = torch.arange(4, device="cuda")
    KV.mmi_cache_write(ctx, c, k, v, slot)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    KV.mmi_cache_read(ctx, c, slot, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        for i in range(4):
            want = OS.value(*OS.quantise(f64(x[i, 0]), kind), kind)
            assert np.array_equal(f64(y[i, 0]), want, equal_nan=True)


@pytest.mark.parametrize("kind", ["fp8", "int8", "fp4"])
def test_ends_of_the_range(ctx, kind):
    """Groups at the type's largest bfloat16 values, and down to where values are no longer normal."""
    from paper_2504_16083_amd import cache as KV
    g = torch.Generator().manual_seed(4)
    e = torch.tensor([127, 126, 120, 0, -80, -100])
    x = ((torch.rand(6, 1, D, generator=g) * 0.99 + 1) * torch.exp2(e.float())[:, None, None]).to(torch.bfloat16)
    x[0, 0, 0] = torch.finfo(torch.bfloat16).max
    x = torch.where(torch.rand(6, 1, D, generator=g) < 0.5, -x, x).cuda()
    c = empty(kind, 1, 1, 16)
    slot = torch.arange(6, device="cuda")
    KV.mmi_cache_write(ctx, c, x, x, slot)
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    KV.mmi_cache_read(ctx, c, slot, ko, vo)
    for i in range(6):
        assert np.array_equal(f64(ko[i, 0]), OS.value(*OS.quantise(f64(x[i, 0]), kind), kind)), i
    assert torch.equal(ko, vo)


@pytest.mark.parametrize("kind", ["bf16", "fp4"])
def test_strides(ctx, kind):
    """Rows as views of a fused projection; pages of one layer among those of others."""
    from paper_2504_16083_amd import cache as KV
    n, H, page, layers = 40, 2, 16, 3
    fused = rows(n, 8, 3)
    k, v = fused[:, 2:4], fused[:, 6:8]
    row = D if kind == "bf16" else 64
    mem = torch.zeros(4, layers, 2, H, page, row, dtype=torch.bfloat16 if kind == "bf16" else torch.uint8, device="cuda")
    sc = torch.zeros(4, layers, 2, H, page, 4, dtype=torch.uint8, device="cuda")
    caches = [KV.Cache(kind, mem[:, i, 0], mem[:, i, 1], sc[:, i, 0], sc[:, i, 1]) for i in range(layers)]
    slot = torch.randperm(64, generator=torch.Generator().manual_seed(2))[:n].cuda()
    KV.mmi_cache_write(ctx, caches[1], k, v, slot)
    assert not mem[:, 0].any() and not mem[:, 2].any()
    out = torch.zeros(n, 8, D, dtype=torch.bfloat16, device="cuda")
    KV.mmi_cache_read(ctx, caches[1], slot, out[:, 1:3], out[:, 5:7])
    plain = KV.Cache.empty(kind, 4, H, page)
    KV.mmi_cache_write(ctx, plain, k.contiguous(), v.contiguous(), slot)
    ko, vo = torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(n, H, D, dtype=torch.bfloat16, device="cuda")
    KV.mmi_cache_read(ctx, plain, slot, ko, vo)
    assert torch.equal(out[:, 1:3], ko) and torch.equal(out[:, 5:7], vo)
    assert not out[:, 0].any() and not out[:, 3:5].any() and not out[:, 7].any()


def test_offsets_past_32_bits(ctx):
    """Slots whose place in memory lies beyond 2^32 bytes."""
    from paper_2504_16083_amd import cache as KV
    page, H, n_pages = 256, 8, 9000                               # 4.7 GB each of K and V
    c = KV.Cache("bf16", *(torch.empty(n_pages, H, page, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"))
    k, v = rows(50, H, 5), rows(50, H, 6)
    slot = torch.cat([torch.arange(25), n_pages * page - 25 + torch.arange(25)])
    KV.mmi_cache_write(ctx, c, k, v, slot.cuda())
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    KV.mmi_cache_read(ctx, c, slot.cuda(), ko, vo)
    bits = lambda t: t.view(torch.int16)  # noqa: E731
    assert torch.equal(bits(ko), bits(k)) and torch.equal(bits(vo), bits(v))
    assert torch.equal(bits(c.k[n_pages - 1, :, page - 25:].transpose(0, 1).contiguous()), bits(k[25:]))


def test_empty_and_stream_and_graph(ctx):
    from paper_2504_16083_amd import cache as KV
    c = empty("fp8", 4, 2, 16)
    none = torch.empty(0, 2, D, dtype=torch.bfloat16, device="cuda")
    KV.mmi_cache_write(ctx, c, none, none, torch.empty(0, dtype=torch.int64, device="cuda"))
    KV.mmi_cache_read(ctx, c, torch.empty(0, dtype=torch.int64, device="cuda"), none, none)
    k, v, slot = rows(20, 2, 1), rows(20, 2, 2), torch.arange(20, device="cuda") + 3
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        KV.mmi_cache_write(ctx, c, k, v, slot)
        KV.mmi_cache_read(ctx, c, slot, ko, vo)
    st = torch.cuda.Stream()
    for seed in range(3):
        k.copy_(rows(20, 2, 30 + seed))
        slot.copy_((torch.arange(20, device="cuda") * 3 + seed) % 64)
        graph.replay()
        torch.cuda.synchronize()
        other = empty("fp8", 4, 2, 16)
        a, b = torch.zeros_like(k), torch.zeros_like(v)
        st.wait_stream(torch.cuda.current_stream())
        KV.mmi_cache_write(ctx, other, k, v, slot, stream=st)
        KV.mmi_cache_read(ctx, other, slot, a, b, stream=st)
        torch.cuda.synchronize()
        assert torch.equal(a, ko) and torch.equal(b, vo)
