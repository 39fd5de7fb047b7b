"""Rotary positions on the GPU against the oracle in fp64."""
import numpy as np
import pytest
import torch

from oracle import serving as OS
from serving import D, HALF_STEP, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2504_16083_amd import mmi
    return mmi.Ctx(0)


def rand(shape, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()


def check(got, x, want, m, freq, layout):
    """Angles are off by 2^-25 of a turn (1.9e-7) and the rounding of its number in fp32 (as much), sine and
    cosine by an ulp or two, the two products and the factor by a rounding each: under 2^-20 of m (|x| + |y|);
    then half a step of the result."""
    a, b = OS.pairs(2 * len(freq), layout)
    size = np.abs(f64(x))
    reach = size.copy()
    reach[..., a] = reach[..., b] = size[..., a] + size[..., b]
    tol = 2.0 ** -20 * m * reach
    tol[..., 2 * len(freq):] = 0
    tol += HALF_STEP * (np.abs(want) + tol)
    off = np.abs(f64(got) - want) - tol
    assert off.max() <= 0, off.max()
    assert np.array_equal(f64(got)[..., 2 * len(freq):], f64(x)[..., 2 * len(freq):])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [16, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("S,Hq,Hkv", [(1, 28, 4), (3, 2, 1), (67, 8, 8), (300, 5, 1)])
def test_layouts_and_shapes(ctx, layout, rot, S, Hq, Hkv):
    from paper_2504_16083_amd import cache as KV
    q, k = rand((S, Hq, D), 1), rand((S, Hkv, D), 2)
    pos = torch.randint(0, 1 << 21, (S,), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    KV.mmi_rope(ctx, KV.RopeCfg(rot_dim=rot, layout=layout, theta=1e6), q, k, pos=pos.cuda(), q_out=qo, k_out=ko)
    f = OS.frequencies(rot, 1e6)
    for x, y in ((q, qo), (k, ko)):
        check(y, x, OS.rope(f64(x), pos.numpy(), f, layout), 1.0, f, layout)
    q0 = q.clone()
    KV.mmi_rope(ctx, KV.RopeCfg(rot_dim=rot, layout=layout, theta=1e6), q=q, pos=pos.cuda())     # in place, q alone
    assert torch.equal(q, qo)
    KV.mmi_rope(ctx, KV.RopeCfg(rot_dim=rot, layout=layout, theta=1e6), k=k, pos=pos.cuda())
    assert torch.equal(k, ko)
    assert not torch.equal(q0, qo)


@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("parts", 16.0)])
def test_scalings_and_far_positions(ctx, scaling, factor):
    from paper_2504_16083_amd import cache as KV
    kw = dict(theta=5e5, scaling=scaling, factor=factor, orig_len=8192.0, beta_fast=32.0, beta_slow=1.0)
    pos = np.array([0, 1, 8191, 131072, 1048576, 2097151, 2 ** 31 - 1, -1, -(2 ** 31)])
    q = rand((len(pos), 4, D), 5)
    out = torch.empty_like(q)
    KV.mmi_rope(ctx, KV.RopeCfg(**kw), q=q, q_out=out, pos=torch.tensor(pos, dtype=torch.int32).cuda())
    f = OS.frequencies(128, **kw)
    m = 0.1 * np.log(factor) + 1 if scaling == "parts" else 1.0
    # far positions in fp64 lose 2^31 * 2^-53 of an angle: far below the bound
    check(out, q, OS.rope(f64(q), pos, f, m=m), m, f, "half")
    table = KV.RopeCfg(inv_freq=f, attn_factor=m)
    again = torch.empty_like(q)
    KV.mmi_rope(ctx, table, q=q, q_out=again, pos=torch.tensor(pos, dtype=torch.int32).cuda())
    check(again, q, OS.rope(f64(q), pos, f, m=m), m, f, "half")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_position_triples_and_fused_views(ctx, layout):
    from paper_2504_16083_amd import cache as KV
    S, Hq, Hkv, sec = 200, 6, 2, (10, 19, 19)
    fused = rand((S, Hq + 2 * Hkv, D), 7)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:].clone()
    q0, k0 = q.clone(), k.clone()
    pos = torch.randint(0, 5000, (3, S), generator=torch.Generator().manual_seed(8)).to(torch.int32)
    KV.mmi_rope(ctx, KV.RopeCfg(rot_dim=96, layout=layout, sections=sec), q, k, pos=pos.cuda())     # in place
    f = OS.frequencies(96)
    for x, y in ((q0, q), (k0, k)):
        check(y, x, OS.rope(f64(x), pos.numpy(), f, layout, sections=sec), 1.0, f, layout)
    assert torch.equal(fused[:, Hq + Hkv:], v)                       # the rest of the buffer is untouched


def test_default_positions(ctx):
    from paper_2504_16083_amd import cache as KV
    q = rand((130, 2, D), 9)
    a, b, c = (torch.empty_like(q) for _ in range(3))
    KV.mmi_rope(ctx, KV.RopeCfg(), q=q, q_out=a)
    KV.mmi_rope(ctx, KV.RopeCfg(), q=q, q_out=b, pos=torch.arange(130, dtype=torch.int32, device="cuda"))
    KV.mmi_rope(ctx, KV.RopeCfg(sections=(20, 22, 22)), q=q, q_out=c)
    assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("layout,rot,sections", [("half", 128, (0, 0, 0)), ("interleaved", 64, (8, 12, 12))])
def test_gradient(ctx, layout, rot, sections):
    """The inverse rotation is the gradient: against the transposed map of the definition, and against
    differences of it."""
    from paper_2504_16083_amd import cache as KV
    S, H, m = 5, 3, 1.25
    f = OS.frequencies(rot, 100.0)
    axes = 3 if any(sections) else 1
    pos = np.random.default_rng(4).integers(0, 1000, (axes, S))
    g = rand((S, H, D), 11)
    out = torch.empty_like(g)
    cfg = KV.RopeCfg(rot_dim=rot, layout=layout, theta=100.0, sections=sections, attn_factor=m)
    KV.mmi_rope(ctx, cfg, q=g, q_out=out, pos=torch.tensor(pos if axes == 3 else pos[0], dtype=torch.int32).cuda(),
                inverse=True)
    fwd = lambda x: OS.rope(x, pos, f, layout, m=m, sections=sections)  # noqa: E731
    # sum(g * fwd(x)) has the gradient fwd^T g: column by column through unit inputs
    G = f64(g)
    want = np.zeros((S, H, D))
    for d in range(D):
        unit = np.zeros((S, H, D))
        unit[..., d] = 1.0
        want[..., d] = (G * fwd(unit)).sum(-1)
    check(out, g, want, m, f, layout)
    x = np.random.default_rng(5).standard_normal((S, H, D))
    for s, h, d in [(0, 0, 0), (1, 2, 5), (4, 1, rot - 1), (3, 0, rot // 2), (2, 2, 127)]:
        up, down = x.copy(), x.copy()
        up[s, h, d] += 1e-3
        down[s, h, d] -= 1e-3
        diff = ((G * fwd(up)).sum() - (G * fwd(down)).sum()) / 2e-3
        assert abs(diff - want[s, h, d]) < 1e-8 * max(1.0, abs(diff))


def test_stream_and_graph(ctx):
    from paper_2504_16083_amd import cache as KV
    q, k = rand((64, 4, D), 12), rand((64, 2, D), 13)
    cfg = KV.RopeCfg()
    want_q, want_k = torch.empty_like(q), torch.empty_like(k)
    KV.mmi_rope(ctx, cfg, q, k, q_out=want_q, k_out=want_k)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    a, b = torch.zeros_like(q), torch.zeros_like(k)
    st.wait_stream(torch.cuda.current_stream())
    KV.mmi_rope(ctx, cfg, q, k, q_out=a, k_out=b, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(a, want_q) and torch.equal(b, want_k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        KV.mmi_rope(ctx, cfg, q, k, q_out=a, k_out=b)
    for seed in range(3):
        q.copy_(rand(q.shape, 20 + seed))
        a.zero_()
        graph.replay()
        KV.mmi_rope(ctx, cfg, q, k, q_out=want_q, k_out=want_k)
        torch.cuda.synchronize()
        assert torch.equal(a, want_q) and torch.equal(b, want_k)


def exact_turns(pos, f):
    """position * f / (2 pi) modulo one, of whole numbers and doubles, by whole-number arithmetic."""
    from fractions import Fraction
    pi = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862, 10 ** 76)
    out = np.zeros((len(pos), len(f)))
    for j, y in enumerate(f):
        step = Fraction(float(y)) / (2 * pi)
        for i, p in enumerate(pos):
            t = int(p) * step
            out[i, j] = float(t - round(t))
    return out


@pytest.mark.parametrize("top", [1.0, 100.0, 1e5, 2.0 ** 40])
def test_angles_of_far_positions_and_high_frequencies(ctx, top):
    """A caller's frequencies up to `top` radians a position, at positions up to the ends of 32 bits: the number of
    turns is held to 2^-63 a position, 2^-32 at 2^31, and the fraction that is left rounded to fp32, half a step of
    a number below 1/2: 2^-26 of a turn and less, inside what check() allows."""
    from paper_2504_16083_amd import cache as KV
    rng = np.random.default_rng(int(top))
    f = np.sort(np.exp(rng.uniform(np.log(1e-7), np.log(top), 64)))[::-1].copy()
    f[0] = top
    pos = np.concatenate([[0, 1, -1, 2 ** 31 - 1, -(2 ** 31)], rng.integers(-(2 ** 31), 2 ** 31, 120),
                          rng.integers(0, 1 << 21, 120)])
    q = rand((len(pos), 2, D), 31)
    out = torch.empty_like(q)
    KV.mmi_rope(ctx, KV.RopeCfg(inv_freq=f), q=q, q_out=out, pos=torch.tensor(pos, dtype=torch.int32).cuda())
    x, angle = f64(q), 2 * np.pi * exact_turns(pos, f)[:, None]
    a, b = x[..., :64], x[..., 64:]
    want = np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1)
    check(out, q, want, 1.0, f, "half")


def test_long_prompt_in_a_fused_projection(ctx):
    """Q and K of 524289 tokens as views of one projection, rotated in place: K's token stride times the length
    passes 2^31 elements. As the same rows in tensors of their own."""
    from paper_2504_16083_amd import cache as KV
    S, Hq, Hkv = (1 << 19) + 1, 28, 4
    fused = torch.empty(S, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    fused.random_(-8, 8, generator=torch.Generator(device="cuda").manual_seed(1))
    q, k = fused[:, :Hq], fused[:, Hq:Hq + Hkv]
    qc, kc, v = q.contiguous(), k.contiguous(), fused[:, Hq + Hkv:].clone()
    cfg = KV.RopeCfg(theta=1e6)
    KV.mmi_rope(ctx, cfg, qc, kc)
    KV.mmi_rope(ctx, cfg, q, k)
    assert torch.equal(q, qc) and torch.equal(k, kc) and torch.equal(fused[:, Hq + Hkv:], v)
