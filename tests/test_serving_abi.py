"""include/mmi_cache.h without a device: the library exports what the header
declares, the structures agree, and bad arguments are refused with the
documented codes before anything is launched."""
import ctypes as ct
import os
import re
import subprocess

import pytest
import torch

from paper_2504_16083_amd import cache as KV
from paper_2504_16083_amd import mmi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = 1 << 20                    # an address; no call here comes as far as using it
INVALID, UNSUPPORTED, BAD_CONFIG = -1, -2, -3


def test_symbols_and_structures():
    src = open(os.path.join(ROOT, "include", "mmi_cache.h")).read()
    names = set(re.findall(r"^int\s+(mmi_\w+)\s*\(", src, re.M))
    assert names == set(KV.SYMBOLS)
    L = KV.lib()
    assert all(hasattr(L, n) for n in names)
    assert KV.mmi_rope_cfg.theta.offset == 32 and ct.sizeof(KV.mmi_rope_cfg) == 88
    assert KV.mmi_cache.page_stride.offset == 56 and ct.sizeof(KV.mmi_cache) == 72
    assert KV.mmi_tree.scale.offset == 128 and ct.sizeof(KV.mmi_tree) == 136


def test_header_is_c(tmp_path):
    """The header compiles as C99, and the compiler's structure sizes are the binding's."""
    c = tmp_path / "sizes.c"
    c.write_text('#include "mmi_cache.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu", '
                 'sizeof(mmi_rope_cfg), sizeof(mmi_cache), sizeof(mmi_tree)); return 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(c), "-o",
                    str(tmp_path / "sizes")], check=True, capture_output=True)
    out = subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in out] == [ct.sizeof(s) for s in (KV.mmi_rope_cfg, KV.mmi_cache, KV.mmi_tree)]


def test_rope_frequencies():
    """mmi_rope_freq against the oracle, for every scaling."""
    from oracle import serving as OS
    for scaling, factor in (("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("parts", 16.0)):
        for rot in (16, 96, 128):
            kw = dict(theta=5e5, scaling=scaling, factor=factor, orig_len=8192.0, beta_fast=32.0, beta_slow=1.0)
            cfg = KV.RopeCfg(rot_dim=rot, **kw)
            got = [cfg.c[0].inv_freq[i] for i in range(rot // 2)]
            assert all(abs(a - b) <= 2e-15 * b for a, b in zip(got, OS.frequencies(rot, **kw)))
    L = KV.lib()
    assert L.mmi_rope_freq(None, None) == INVALID
    c = KV.mmi_rope_cfg(128, 0, 0, 0, (ct.c_int32 * 3)(0, 0, 0), 0, 10000.0, 1.0, 0.0, 32.0, 1.0, 0.0, None)
    assert L.mmi_rope_freq(ct.byref(c), None) == INVALID
    c.theta = -1.0
    assert L.mmi_rope_freq(ct.byref(c), (ct.c_double * 64)()) == BAD_CONFIG
    with pytest.raises(mmi.MMIError):
        KV.RopeCfg(rot_dim=20)


def rope(prob=None, cfg=None, q=DEV, k=DEV, qo=DEV, ko=DEV, pos=None, **kw):
    c = KV.mmi_rope_cfg(128, 0, 0, 0, (ct.c_int32 * 3)(0, 0, 0), 0, 10000.0, 1.0, 0.0, 32.0, 1.0, 0.0, None)
    for name, value in kw.items():
        setattr(c, name, value)
    p = prob or mmi.Problem(100, 4, 2)
    return KV.lib().mmi_rope(None, ct.byref(p.c), None if cfg == 0 else ct.byref(c), pos, q, k, qo, ko, None)


def test_rope_refusals():
    assert rope() == INVALID and "ctx" in mmi.mmi_last_error()       # all but the context is right
    assert KV.lib().mmi_rope(None, None, None, None, None, None, None, None, None) == INVALID
    assert rope(cfg=0) == INVALID
    for r in (0, 8, 24, 144, -16):
        assert rope(rot_dim=r) == UNSUPPORTED
    for kw in ({"layout": 2}, {"scaling": 4}, {"scaling": -1}, {"inverse": 2}, {"theta": 0.0}, {"theta": float("nan")},
               {"scaling": 1, "factor": 0.5}, {"scaling": 3, "factor": 2.0, "orig_len": 0.0},
               {"scaling": 3, "factor": 2.0, "orig_len": 10.0, "beta_fast": 1.0}, {"attn_factor": -1.0},
               {"sections": (ct.c_int32 * 3)(16, 24, 25)}, {"sections": (ct.c_int32 * 3)(-1, 40, 25)}):
        assert rope(**kw) == BAD_CONFIG, kw
    assert rope(reserved=1) == INVALID
    table = (ct.c_double * 64)(*([1.0] * 63 + [float("inf")]))
    assert rope(inv_freq=table) == BAD_CONFIG
    table[63] = -1.0
    assert rope(inv_freq=table) == BAD_CONFIG
    table[63] = 100.0
    assert rope(inv_freq=table, theta=0.0) == INVALID and "ctx" in mmi.mmi_last_error()
    assert rope(q=None, qo=None) == INVALID and "ctx" in mmi.mmi_last_error()
    assert rope(q=None, qo=None, k=None, ko=None) == INVALID and "NULL" in mmi.mmi_last_error()
    assert rope(q=None) == INVALID and rope(ko=None) == INVALID
    assert rope(q=DEV + 8) == INVALID and rope(ko=DEV + 2) == INVALID and rope(pos=DEV + 2) == INVALID
    assert rope(mmi.Problem(0, 4, 2)) == INVALID and rope(mmi.Problem(100, 3, 2)) == UNSUPPORTED
    assert rope(mmi.Problem(100, 4, 2, strides={"q": (516, 128)})) == INVALID
    assert rope(mmi.Problem(100, 4, 2, strides={"q": (0, 128)})) == INVALID


def pool(**kw):
    c = KV.mmi_cache(1, 64, 2, 128, 10, DEV, DEV, DEV, DEV, 0, 0)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def rows(c, n=5, k=DEV, v=DEV, slot=DEV, ks=(0, 0), vs=(0, 0)):
    p = None if c is None else ct.byref(c)
    a = KV.lib().mmi_cache_write(None, p, k, *ks, v, *vs, slot, n, None)
    assert a == KV.lib().mmi_cache_read(None, p, slot, n, k, *ks, v, *vs, None)
    return a


def test_cache_refusals():
    assert rows(pool()) == INVALID and "ctx" in mmi.mmi_last_error()
    assert rows(None) == INVALID
    assert rows(pool(type=4)) == BAD_CONFIG and rows(pool(type=-1)) == BAD_CONFIG
    assert rows(pool(D=64)) == UNSUPPORTED
    for page in (0, 8, 48, 512, -16):
        assert rows(pool(page=page)) == UNSUPPORTED
    assert rows(pool(Hkv=0)) == INVALID and rows(pool(Hkv=2000)) == UNSUPPORTED
    assert rows(pool(n_pages=0)) == INVALID and rows(pool(n_pages=1 << 31)) == UNSUPPORTED
    assert rows(pool(k=None)) == INVALID and rows(pool(v=DEV + 8)) == INVALID
    assert rows(pool(k_scale=None)) == INVALID and rows(pool(v_scale=DEV + 2)) == INVALID
    assert rows(pool(type=0, k_scale=None, v_scale=None)) == INVALID and "ctx" in mmi.mmi_last_error()
    packed = 64 * 2 * 128
    assert rows(pool(page_stride=packed - 16)) == INVALID and rows(pool(page_stride=packed + 8)) == INVALID
    assert rows(pool(scale_stride=64 * 2 * 4 - 4)) == INVALID and rows(pool(scale_stride=64 * 2 * 4 + 2)) == INVALID
    assert rows(pool(page_stride=packed + 16, scale_stride=64 * 2 * 4 + 4)) == INVALID
    assert "ctx" in mmi.mmi_last_error()
    assert rows(pool(page_stride=1 << 41)) == UNSUPPORTED
    assert rows(pool(), n=-1) == INVALID and rows(pool(), n=(1 << 25) + 1) == UNSUPPORTED
    assert rows(pool(), k=None) == INVALID and rows(pool(), v=DEV + 4) == INVALID and rows(pool(), slot=DEV + 4) == INVALID
    assert rows(pool(), ks=(252, 128)) == INVALID and rows(pool(), vs=(-256, 128)) == INVALID
    assert rows(pool(), n=0, k=None, v=None, slot=None) == INVALID and "ctx" in mmi.mmi_last_error()


def tree(c=None, q=DEV, o=DEV, ws=DEV, bytes=1 << 40, lse=None, **kw):
    t = KV.mmi_tree(n_seq=3, n_rows=9, Hq=8, max_rows=3, max_len=100, max_pages=2, mask_words=1, row_start=DEV,
                    length=DEV, pages=DEV, mask=DEV)
    for name, value in kw.items():
        setattr(t, name, value)
    c = c or pool()
    need = ct.c_size_t()
    L = KV.lib()
    a = L.mmi_tree_attention(None, ct.byref(c), ct.byref(t), q, DEV, DEV, o, lse, ws, bytes, None)
    b = L.mmi_tree_workspace(None, ct.byref(c), ct.byref(t), ct.byref(need))
    return a, b


def test_tree_refusals():
    both = lambda code: (code, code)  # noqa: E731
    assert tree() == both(INVALID) and "ctx" in mmi.mmi_last_error()
    assert KV.lib().mmi_tree_attention(None, ct.byref(pool()), None, DEV, DEV, DEV, DEV, None, DEV, 1, None) == INVALID
    assert KV.lib().mmi_tree_workspace(None, None, None, None) == INVALID
    for kw in ({"n_seq": -1}, {"n_rows": -1}, {"Hq": 0}, {"max_rows": 0}, {"max_len": -1}, {"max_pages": 1},
               {"max_pages": -1}, {"mask_words": 0}, {"max_rows": 65}, {"scale": -1.0}, {"scale": float("nan")},
               {"reserved": 1}, {"q_stride_s": 12, "q_stride_h": 128}, {"o_stride_s": 1024}):
        assert tree(**kw) == both(INVALID), kw
    for kw in ({"n_seq": 5000}, {"n_rows": (1 << 20) + 1}, {"Hq": 7}, {"Hq": 2048}, {"max_rows": 257},
               {"max_len": (1 << 30) + 1, "max_pages": 1 << 25}, {"k_stride_s": 1 << 41, "k_stride_h": 128}):
        assert tree(**kw) == both(UNSUPPORTED), kw
    assert tree(pool(type=9)) == both(BAD_CONFIG)
    # only the attention call takes these
    for kw in ({"q": None}, {"o": DEV + 8}, {"lse": DEV + 2}, {"row_start": None}, {"length": DEV + 1}, {"pages": None},
               {"mask": DEV + 4}):
        assert tree(**kw)[0] == INVALID, kw
        assert KV.lib().mmi_tree_workspace is not None
    assert tree(pages=None, max_len=0)[0] == INVALID and "ctx" in mmi.mmi_last_error()


class _Ctx:
    device, h = 0, None


def test_binding_refusals():
    """What the C side cannot see: types, shapes and devices of the tensors."""
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(ValueError, match="bfloat16"):
        KV.mmi_rope(_Ctx, KV.RopeCfg(), q=torch.zeros(4, 2, 128))
    with pytest.raises(ValueError, match="context"):
        KV.mmi_rope(_Ctx, KV.RopeCfg(), q=bf(4, 2, 128))
    with pytest.raises(ValueError, match="neither"):
        KV.mmi_rope(_Ctx, KV.RopeCfg())
    with pytest.raises(ValueError):
        KV.RopeCfg(layout="other")
    with pytest.raises(ValueError):
        KV.RopeCfg(rot_dim=64, inv_freq=[1.0] * 31)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError, match="scales"):
        KV.Cache("fp8", u8(3, 2, 16, 128), u8(3, 2, 16, 128))
    with pytest.raises(ValueError, match="shape"):
        KV.Cache("fp4", u8(3, 2, 16, 128), u8(3, 2, 16, 128), u8(3, 2, 16, 4), u8(3, 2, 16, 4))
    with pytest.raises(ValueError, match="contiguous"):
        KV.Cache("bf16", bf(3, 16, 2, 128).transpose(1, 2), bf(3, 16, 2, 128).transpose(1, 2))
    with pytest.raises(ValueError, match="overlap"):
        KV.Cache("bf16", bf(1, 2, 16, 128).expand(3, 2, 16, 128), bf(1, 2, 16, 128).expand(3, 2, 16, 128))
    with pytest.raises(ValueError, match="unknown"):
        KV.Cache("fp16", bf(3, 2, 16, 128), bf(3, 2, 16, 128))
    c = KV.Cache("bf16", bf(3, 2, 16, 128), bf(3, 2, 16, 128))
    with pytest.raises(ValueError, match="context"):
        KV.mmi_cache_write(_Ctx, c, bf(4, 2, 128), bf(4, 2, 128), torch.zeros(4, dtype=torch.int64))


def test_tree_binding_refusals():
    """A batch's tensors are checked when it is made, its device and rows with every call."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    mask = torch.zeros(5, 1, dtype=torch.int64)
    for args in [(i32(2), i32(2), i32(2, 3)), (i32(3), i32(2).long(), i32(2, 3)), (i32(3), i32(2), i32(3, 3)),
                 (i32(3), i32(2), i32(6)), (i32(3), i32(2), i32(3, 2).t()), (i32(6)[::2], i32(2), i32(2, 3)),
                 (i32(3), i32(2), i32(2, 3), mask.int()), (i32(3), i32(2), i32(2, 3), mask[0])]:
        with pytest.raises(ValueError, match="must be"):
            KV.Tree(*args)
    tree = KV.Tree(i32(3), i32(2), i32(2, 3), mask)
    with pytest.raises(AttributeError):                      # another tensor is another batch
        tree.length = i32(2)
    tree.length += 1                                         # its contents are the caller's
    assert tree.length.tolist() == [1, 1]
    with pytest.raises(ValueError, match="context"):
        tree._struct(_Ctx, 4, 5)
    host = type("", (), {"device": -1})
    with pytest.raises(ValueError, match="5 rows for 4"):
        tree._struct(host, 4, 4)
    tree.max_rows, tree.max_len, tree.scale = 3, 48, 0.5
    t = tree._struct(host, 4, 5, *range(8, 72, 8))
    assert (t.n_seq, t.n_rows, t.Hq, t.max_rows, t.max_len, t.max_pages, t.mask_words) == (2, 5, 4, 3, 48, 3, 1)
    assert (t.row_start, t.length, t.pages, t.mask) == tuple(x.data_ptr() for x in (tree.row_start, tree.length, tree.pages, mask))
    assert [getattr(t, f"{x}_stride_{y}") for x in "qkvo" for y in "sh"] == list(range(8, 72, 8))
    assert t.scale == 0.5 and t.reserved == 0


class _Host:
    """A context whose tensors are the host's: the binding takes them, the library refuses the missing context."""
    device, h = -1, None


def _calls(n, q, k, v):
    """Every entry point that takes rows, on tensors [n, heads, 128] given in each place in turn."""
    new = lambda t: torch.zeros(*t.shape, dtype=torch.bfloat16)  # noqa: E731
    cache = KV.Cache("bf16", *(torch.zeros(3, k.shape[1], 16, 128, dtype=torch.bfloat16) for _ in "kv"))
    slot = torch.zeros(n, dtype=torch.int64)
    tree = KV.Tree(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                   torch.zeros(1, 3, dtype=torch.int32), max_rows=n)
    ws = torch.zeros(16, dtype=torch.uint8)
    return [lambda: KV.mmi_rope(_Host, KV.RopeCfg(), q=q, stream=0), lambda: KV.mmi_rope(_Host, KV.RopeCfg(), k=k, stream=0),
            lambda: KV.mmi_rope(_Host, KV.RopeCfg(), q=new(q), q_out=q, stream=0),
            lambda: KV.mmi_rope(_Host, KV.RopeCfg(), k=new(k), k_out=k, stream=0),
            lambda: KV.mmi_cache_write(_Host, cache, k, new(v), slot, stream=0),
            lambda: KV.mmi_cache_write(_Host, cache, new(k), v, slot, stream=0),
            lambda: KV.mmi_cache_read(_Host, cache, slot, k, new(v), stream=0),
            lambda: KV.mmi_cache_read(_Host, cache, slot, new(k), v, stream=0),
            lambda: KV.mmi_tree_attention(_Host, cache, tree, q, new(k), new(v), new(q), ws, stream=0),
            lambda: KV.mmi_tree_attention(_Host, cache, tree, new(q), k, new(v), new(q), ws, stream=0),
            lambda: KV.mmi_tree_attention(_Host, cache, tree, new(q), new(k), v, new(q), ws, stream=0),
            lambda: KV.mmi_tree_attention(_Host, cache, tree, new(q), new(k), new(v), q, ws, stream=0)]


@pytest.mark.parametrize("n,Hq,Hkv", [(64, 8, 2), (1, 8, 2), (64, 1, 1)])
def test_broadcast_rows_are_refused(n, Hq, Hkv):
    """A row repeated over tokens and heads has the strides 0, 0, which the library takes for packed: 128 channels
    would be read, or written, as n * heads rows of them."""
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    for call in _calls(n, bf(n, Hq, 128), bf(n, Hkv, 128), bf(n, Hkv, 128)):
        with pytest.raises(mmi.MMIError, match="ctx"):       # all but the context is right
            call()
    every = [lambda H: bf(1, 1, 128).expand(n, H, 128)]
    if n > 1:
        every.append(lambda H: bf(1, H, 128).expand(n, H, 128))
    if Hkv > 1:
        every.append(lambda H: bf(n, 1, 128).expand(n, H, 128))
    for wide in every:
        for call in _calls(n, wide(Hq), wide(Hkv), wide(Hkv)):
            with pytest.raises(ValueError, match="broadcast|strides"):
                call()


@pytest.mark.parametrize("theta", [100.0, 1e4, 1e6, 3e7])
@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 3.0), ("ntk", 8.0), ("parts", 40.0)])
def test_rope_frequencies_to_the_last_places(theta, scaling, factor):
    """mmi_rope_freq against the formula in 50 digits: off by (ln theta + 8) 2^-53 of itself at most."""
    from decimal import Decimal, getcontext
    getcontext().prec = 50
    pi = Decimal("3.1415926535897932384626433832795028841971693993751")
    for rot in (16, 48, 96, 128):
        cfg = KV.RopeCfg(rot_dim=rot, theta=theta, scaling=scaling, factor=factor, orig_len=32768.0)
        base, F = Decimal(theta), Decimal(factor)
        if scaling == "ntk":
            base = base * F ** (Decimal(rot) / (rot - 2))
        for i in range(rot // 2):
            f = base ** (Decimal(-2 * i) / rot)
            if scaling == "linear":
                f /= F
            if scaling == "parts":
                g = min(max((32768 * f / (2 * pi) - 1) / 31, Decimal(0)), Decimal(1))
                f *= g + (1 - g) / F
            off = abs(Decimal(cfg.c[0].inv_freq[i]) / f - 1)
            assert off <= (base.ln() + 8) * Decimal(2) ** -53, (rot, i, off)


def test_rope_frequencies_end_at_2_to_40():
    table = (ct.c_double * 64)(*[2.0 ** 40] * 64)
    assert rope(inv_freq=table) == INVALID and "ctx" in mmi.mmi_last_error()
    table[5] = 2.0 ** 40 * (1 + 2.0 ** -52)
    assert rope(inv_freq=table) == BAD_CONFIG
    assert rope(theta=1e-20) == BAD_CONFIG and rope(theta=1e-12) == INVALID


@pytest.mark.parametrize("S", [524288, 1048576, 1 << 21])
def test_rope_takes_long_fused_projections(S):
    """Views of a [S, 36, 128] projection: K's token stride times S passes 2^31 elements, a limit of the attention
    kernel's and not of the rotation."""
    wide = {"q": (36 * 128, 128), "k": (36 * 128, 128)}
    assert rope(mmi.Problem(S, 28, 4, strides=wide)) == INVALID and "ctx" in mmi.mmi_last_error()
    assert rope(mmi.Problem(S, 28, 4, strides={"k": (1 << 30, 1 << 24)})) == INVALID and "ctx" in mmi.mmi_last_error()
    assert rope(mmi.Problem(S, 28, 4, strides={"k": (1 << 41, 128)})) == UNSUPPORTED
    assert rope(mmi.Problem((1 << 21) + 1, 28, 4)) == UNSUPPORTED


def _moved(how, t):
    """t with its memory replaced by a longer tensor's."""
    other = torch.zeros(4, *t.shape, dtype=t.dtype)
    if how == "set":
        t.set_(other[1])
    elif how == "data":
        t.data = other[1]
    else:
        t.resize_(64 * t.numel() + 4096)
        assert t.numel() > 4096


@pytest.mark.parametrize("how", ["set", "data", "resize"])
@pytest.mark.parametrize("which", ["k", "v", "k_scale", "v_scale", "row_start", "length", "pages", "mask"])
def test_tensors_with_other_memory_are_refused(how, which):
    """A cache and a batch hand addresses on that they took when they were made: a tensor that has been given other
    memory since must not be read or written at the old one. Another tensor in its place is no assignment."""
    cache = KV.Cache("fp8", *(torch.zeros(3, 2, 16, w, dtype=torch.uint8) for w in (128, 128, 4, 4)))
    tree = KV.Tree(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                   torch.zeros(1, 3, dtype=torch.int32), mask=torch.zeros(5, 1, dtype=torch.int64), max_rows=5)
    bf = lambda h: torch.zeros(5, h, 128, dtype=torch.bfloat16)  # noqa: E731
    slot, ws = torch.zeros(5, dtype=torch.int64), torch.zeros(16, dtype=torch.uint8)
    calls = [lambda: KV.mmi_tree_attention(_Host, cache, tree, bf(4), bf(2), bf(2), bf(4), ws, stream=0)]
    if which in ("k", "v", "k_scale", "v_scale"):
        calls += [lambda: KV.mmi_cache_write(_Host, cache, bf(2), bf(2), slot, stream=0),
                  lambda: KV.mmi_cache_read(_Host, cache, slot, bf(2), bf(2), stream=0)]
    owner = tree if len(calls) == 1 else cache
    t = getattr(owner, which)
    t += 1                                                   # the contents are the caller's
    for call in calls:
        with pytest.raises(mmi.MMIError, match="ctx"):
            call()
    with pytest.raises(AttributeError):
        setattr(owner, which, t.clone())
    _moved(how, t)
    for call in calls:
        with pytest.raises(ValueError, match="other memory"):
            call()


def test_mask_without_words_is_refused():
    """Such a tensor has no address: the call would go on without a mask, every token seeing those before it."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="words"):
        KV.Tree(i32(2), i32(1), i32(1, 3), mask=torch.zeros(5, 0, dtype=torch.int64), max_rows=5)


def test_scale_that_overflows_is_refused():
    """Scores are taken times scale * log2(e): an infinity there makes a score of zero a NaN."""
    assert tree(scale=3e38) == (INVALID, INVALID) and "scale" in mmi.mmi_last_error()
    for scale in (2.0 ** 127, 1.0, 1e-45):
        assert tree(scale=scale) == (INVALID, INVALID) and "ctx" in mmi.mmi_last_error()
