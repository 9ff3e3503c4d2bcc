"""CPU tests of the C ABI of the rotary positions and the 8-bit cache: every
refusal comes before any HIP call, the host functions are right, and the Python
checks name their reason."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2402_02082_amd as glide
from oracle import rope as OR
from paper_2402_02082_amd import _lib

FAKE = 0x1000  # never dereferenced: every call below fails validation
EINVAL = glide.GLIDE_EINVAL


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _cache(blocks=FAKE, scales=FAKE, tail=FAKE):
    return _lib._Q8Pointers(blocks, scales, tail)


BAD_CACHES = [dict(blocks=None), dict(scales=None), dict(tail=None), dict(blocks=FAKE + 8), dict(scales=FAKE + 4),
              dict(tail=FAKE + 2)]
BAD_SIZES = [dict(B=0), dict(B=65536), dict(Hkv=0), dict(Hkv=65536), dict(D=64), dict(L_cap=0), dict(L_cap=16),
             dict(L_cap=100), dict(L_cap=(1 << 22) + 32), dict(B=1 << 15, Hkv=128), dict(kind=0), dict(kind=1), dict(kind=4)]


def _rope(lib, **kw):
    a = dict(q=FAKE, qo=FAKE, qs=(0, 4096, 128), qos=(0, 4096, 128), H=32, k=FAKE, ko=FAKE, ks=(0, 1024, 128), Hkv=8,
             freqs=FAKE, rot=128, m=1.0, pos=None, lens=FAKE, par=FAKE, B=1, T=16, D=128, dtype=0, flags=0)
    a.update(kw)
    S = ctypes.c_int64 * 3
    q = _lib._RopeRows(a["q"], a["qo"], S(*a["qs"]), S(*a["qos"]), a["H"])
    k = _lib._RopeRows(a["k"], a["ko"], S(*a["ks"]), S(*a["ks"]), a["Hkv"])
    return lib.glide_rope(ctypes.byref(q), ctypes.byref(k), a["freqs"], a["rot"], a["m"], a["pos"], a["lens"],
                          a["par"], a["B"], a["T"], a["D"], a["dtype"], a["flags"], None)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(freqs=None), dict(q=FAKE + 2), dict(ko=FAKE + 4),
    dict(qs=(0, 4100, 128)), dict(qos=(0, 4096, 130)), dict(ks=(-8, 1024, 128)), dict(qs=(0, 4096, 2), dtype=1),
    dict(H=0), dict(Hkv=0), dict(rot=0), dict(rot=3), dict(rot=130), dict(m=float("nan")), dict(m=float("inf")),
    dict(pos=FAKE), dict(pos=FAKE, lens=None), dict(pos=FAKE, par=None), dict(B=0), dict(B=65536), dict(T=0),
    dict(T=65), dict(par=None, T=(1 << 22) + 1), dict(D=64), dict(dtype=2), dict(dtype=-1), dict(flags=4), dict(par=None, T=1 << 21, B=64),
])
def test_rope_rejects(lib, bad):
    assert _rope(lib, **bad) == EINVAL


def test_rope_rejects_no_queries(lib):
    assert lib.glide_rope(None, None, FAKE, 128, 1.0, None, None, None, 1, 1, 128, 0, 0, None) == EINVAL


@pytest.mark.parametrize("rot", [2, 50, 64, 128])
@pytest.mark.parametrize("scaling,kw", [(None, {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
                                        ("yarn", dict(factor=8.0, original_len=4096)),
                                        ("yarn", dict(factor=1.0, original_len=100))])
def test_rope_frequencies(rot, scaling, kw):
    if scaling == "ntk" and rot == 2:
        with pytest.raises(glide.GlideError):
            glide.rope_frequencies(rot, scaling=scaling, device="cpu", **kw)
        return
    f, m = glide.rope_frequencies(rot, base=500000.0, scaling=scaling, device="cpu", **kw)
    want, want_m = OR.frequencies(rot, 500000.0, scaling, **kw)
    assert f.dtype == torch.float64 and f.shape == (rot // 2,)
    assert np.allclose(f.numpy(), want, rtol=1e-13) and abs(m - want_m) <= 2.0 ** -24 * 2


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=130), dict(rot_dim=7), dict(scaling="other")])
def test_rope_frequencies_rejects(bad):
    with pytest.raises(ValueError):
        glide.rope_frequencies(**{**dict(rot_dim=128, device="cpu"), **bad})


@pytest.mark.parametrize("bad", [dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                                 dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("nan")),
                                 dict(scaling="yarn", factor=2.0, original_len=0),
                                 dict(scaling="ntk", base=1e300, factor=1e300)])
def test_rope_frequencies_refuses(bad):
    with pytest.raises(glide.GlideError):
        glide.rope_frequencies(128, device="cpu", **bad)


def _append(lib, cache=None, **kw):
    a = dict(k=FAKE, v=FAKE, sb=8, st=4096, sh=128, lens=FAKE, counts=None, hold=0, B=1, T=16, Hkv=32, D=128,
             L_cap=2048, kind=glide.GLIDE_E4M3)
    a.update(kw)
    c = _cache(**(cache or {}))
    return lib.glide_q8_append(a["k"], a["v"], a["sb"], a["st"], a["sh"], a["lens"], a["counts"], a["hold"],
                               ctypes.byref(c), a["B"], a["T"], a["Hkv"], a["D"], a["L_cap"], a["kind"], None)


@pytest.mark.parametrize("bad", BAD_SIZES + [
    dict(k=None), dict(v=None), dict(lens=None), dict(k=FAKE + 2), dict(v=FAKE + 8), dict(T=0), dict(T=65, hold=1),
    dict(T=(1 << 22) + 1), dict(sb=4), dict(st=-8), dict(sh=130)])
def test_append_rejects(lib, bad):
    assert _append(lib, **bad) == EINVAL


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_append_rejects_caches(lib, bad):
    assert _append(lib, cache=bad) == EINVAL


def _read(lib, cache=None, **kw):
    a = dict(lens=FAKE, k=FAKE, v=FAKE, dtype=0, B=1, Hkv=32, D=128, L_cap=2048, kind=glide.GLIDE_INT8, start=0, T=64)
    a.update(kw)
    c = _cache(**(cache or {}))
    return lib.glide_q8_read(ctypes.byref(c), a["lens"], a["k"], a["v"], a["dtype"], a["B"], a["Hkv"], a["D"],
                             a["L_cap"], a["kind"], a["start"], a["T"], None)


@pytest.mark.parametrize("bad", BAD_SIZES + [
    dict(lens=None), dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(dtype=2), dict(start=-1), dict(T=0),
    dict(start=2048, T=32), dict(start=1, T=2047 + 32), dict(start=2147483647, T=2147483647)])
def test_read_rejects(lib, bad):
    assert _read(lib, **bad) == EINVAL


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_read_rejects_caches(lib, bad):
    assert _read(lib, cache=bad) == EINVAL


def _attn(lib, cache=None, **kw):
    a = dict(q=FAKE, lens=FAKE, par=FAKE, out=FAKE, B=1, N=16, H=32, Hkv=8, D=128, L_cap=2048, kind=glide.GLIDE_INT8,
             scale=0.0, splits=0, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    c = _cache(**(cache or {}))
    return lib.glide_q8_tree_attn(a["q"], ctypes.byref(c), a["lens"], a["par"], a["out"], a["B"], a["N"], a["H"],
                                  a["Hkv"], a["D"], a["L_cap"], a["kind"], a["scale"], a["splits"], a["ws"],
                                  a["ws_bytes"], None)


@pytest.mark.parametrize("bad", BAD_SIZES + [
    dict(q=None), dict(lens=None), dict(out=None), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(N=0), dict(N=65),
    dict(H=0), dict(H=4), dict(H=12), dict(B=4096, N=64, H=1024, Hkv=1), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(splits=-1), dict(splits=65), dict(ws=None), dict(ws_bytes=16), dict(ws=FAKE + 4)])
def test_attn_rejects(lib, bad):
    assert _attn(lib, **bad) == EINVAL


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_attn_rejects_caches(lib, bad):
    assert _attn(lib, cache=bad) == EINVAL


def test_attn_workspace(lib):
    ws = lib.glide_q8_tree_attn_workspace
    assert ws(1, 16, 32, 32, 128, 2048, 0) > glide.ATTN_COUNTER_BYTES
    assert ws(1, 16, 32, 32, 128, 2048, 1) == 0 and ws(1, 16, 32, 32, 128, 32, 0) == 0
    for bad in ((0, 16, 32, 32, 128, 2048, 0), (1, 65, 32, 32, 128, 2048, 0), (1, 16, 32, 5, 128, 2048, 0),
                (1, 16, 32, 32, 64, 2048, 0), (1, 16, 32, 32, 128, 2040, 0), (1, 16, 32, 32, 128, 2048, 65)):
        assert ws(*bad) == 0
    sizes = [ws(4, 32, 40, 40, 128, 4096, s) for s in (2, 4, 8, 16, 32)]
    assert sizes == sorted(sizes)


def _commit(lib, cache=None, **kw):
    a = dict(layers=2, lens=FAKE, acc=FAKE, path=FAKE, out=FAKE + 64, B=1, N=16, Hkv=32, D=128, L_cap=2048,
             kind=glide.GLIDE_INT8)
    a.update(kw)
    c = (_lib._Q8Pointers * 130)(*[_cache(tail=FAKE + 32 * i) for i in range(130)])
    c[1] = _cache(**{**dict(tail=FAKE + 32), **(cache or {})})
    return lib.glide_q8_commit(c, a["layers"], a["lens"], a["acc"], a["path"], a["out"], a["B"], a["N"], a["Hkv"],
                               a["D"], a["L_cap"], a["kind"], None)


@pytest.mark.parametrize("bad", BAD_SIZES + [dict(lens=None), dict(acc=None), dict(out=None), dict(out=FAKE),
                                             dict(layers=0), dict(layers=129), dict(N=0), dict(N=65)])
def test_commit_rejects(lib, bad):
    assert _commit(lib, **bad) == EINVAL


def test_commit_rejects_a_layer_given_twice(lib):
    for layers, same in ((2, dict(tail=FAKE)), (5, dict(tail=FAKE + 3 * 32)), (128, dict(tail=FAKE + 127 * 32))):
        assert _commit(lib, cache=same, layers=layers) == EINVAL


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_commit_rejects_caches(lib, bad):
    assert _commit(lib, cache=bad) == EINVAL


def test_binding_rejects_host_tensors():
    c = glide.q8_cache(1, 2, 64, device="cpu")
    assert c.blocks.shape == (1, 2, 2, 8192) and c.scales.shape == (1, 2, 2, 2) and c.tail.shape == (1, 2, 2, 128, 128)
    assert glide.q8_cache(1, 2, 65, "int8", "cpu").blocks.shape[2] == 3
    q, lens = torch.zeros((1, 4, 2, 128), dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    f = torch.ones(64, dtype=torch.float64)
    for call in (lambda: glide.glide_rope(q, None, f, q, None),
                 lambda: glide.glide_q8_append(q, q, c, lens),
                 lambda: glide.glide_q8_read(c, lens, q, q),
                 lambda: glide.glide_q8_tree_attn(q, c, lens, None, q),
                 lambda: glide.glide_q8_commit([c], lens, lens, None, lens.clone())):
        with pytest.raises(ValueError):
            call()
    for bad in (dict(kind="fp8"), dict(B=0), dict(H_kv=0), dict(L_cap=0)):
        with pytest.raises(ValueError):
            glide.q8_cache(**{**dict(B=1, H_kv=1, L_cap=32, device="cpu"), **bad})


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("H,Hkv", [(1 << 27, 1), (1 << 28, 1), (1, 1 << 27), ((1 << 26), 1), (1, 1 << 26),
                                   ((1 << 31) - 2, 1)])
def test_rope_rejects_heads_whose_pieces_pass_an_int(lib, dtype, H, Hkv):
    """A row is 8 or 16 pieces for the threads of its token, counted in 32 bits."""
    assert _rope(lib, H=H, Hkv=Hkv, B=1, T=1, dtype=dtype) == EINVAL


@pytest.mark.parametrize("bad", [dict(acc=FAKE + 64), dict(path=FAKE + 64), dict(lens=FAKE + 68), dict(lens=FAKE + 60),
                                 dict(acc=FAKE + 68), dict(acc=FAKE + 60), dict(path=FAKE + 68),
                                 dict(path=FAKE + 64 - 4 * 32 + 4), dict(path=FAKE)])
def test_commit_rejects_lengths_out_that_overlap_what_is_read(lib, bad):
    """Workgroups read lengths, counts and paths while one of them writes the new
    lengths: of two sequences and 16 nodes here."""
    apart = dict(lens=FAKE + 1024, acc=FAKE + 2048, path=FAKE + 4096, out=FAKE + 64, B=2)
    assert _commit(lib, **{**apart, **bad}) == EINVAL
