"""Rotary positions on the GPU against the float64 oracle.

Tolerance.  The angle is reduced in float64 and its sine and cosine taken in
float32: the reduced turn is off by at most 2^-26 (2 pi 2^-26 < 1e-7 of angle),
the two functions by about two units of 2^-24, their product with m, the two
products and the sum by 2^-24 each: below 6e-7 of m (|x1| + |x2|) in all, taken
as 1e-6; and the result is rounded once, by at most eps / 2 of its size."""

import numpy as np
import pytest
import torch

import paper_2402_02082_amd as glide
from oracle import rope as OR
from tests.gpu_common import cpu_normal, require_gpu, say

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def f64(t):
    return t.detach().double().cpu().numpy()


def _tree(T, rng):
    return [int(rng.integers(-1, n)) if n else -1 for n in range(T)]


def _check(got, x, pos, freqs, m, inter, back):
    x64 = f64(x)
    want = OR.rope(x64, pos, freqs, m, inter, back)
    both = np.zeros_like(x64)
    half = len(freqs)
    a, b = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if inter else (np.arange(half),
                                                                                 np.arange(half, 2 * half))
    both[..., a] = both[..., b] = np.abs(x64[..., a]) + np.abs(x64[..., b])
    tol = torch.finfo(x.dtype).eps / 2 * np.abs(want) + 1e-6 * m * both
    err = np.abs(f64(got) - want)
    assert np.all(err <= tol), (err - tol).max()
    assert np.array_equal(f64(got)[..., 2 * half:], x64[..., 2 * half:])  # the other dims are copied


def _positions(where, B, T, rng):
    """(keyword arguments, positions [B, T])"""
    if where == "given":
        pos = rng.integers(0, 1 << 22, (B, T)).astype(np.int32)
        return dict(positions=torch.from_numpy(pos).cuda()), pos
    if where == "zero":
        return {}, np.tile(np.arange(T), (B, 1))
    lens = rng.integers(0, 100000, B).astype(np.int32)
    kw = dict(seq_lens=torch.from_numpy(lens).cuda())
    if where == "start":
        return kw, lens[:, None] + np.arange(T)
    par = np.array([_tree(T, rng) for _ in range(B)], dtype=np.int32)
    kw["tree_parents"] = torch.from_numpy(par).cuda()
    if where == "tree0":
        del kw["seq_lens"]
        lens = lens * 0
    return kw, np.array([OR.tree_positions(lens[b], par[b]) for b in range(B)])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True], ids=["half", "inter"])
@pytest.mark.parametrize("rot", [128, 64, 112, 50, 2, 126])
@pytest.mark.parametrize("where", ["given", "zero", "start", "tree", "tree0"])
def test_rope(dtype, inter, rot, where):
    require_gpu()
    rng = np.random.default_rng(rot)
    for B, T, H, Hk, back in ((1, 1, 1, 1, False), (2, 5, 3, 1, True), (1, 37, 20, 4, False), (3, 64, 5, 5, True)):
        say("rope", str(dtype), inter, rot, where, B, T, H, Hk, back)
        kw, pos = _positions(where, B, T, rng)
        freqs, m = glide.rope_frequencies(rot, scaling="yarn", factor=8.0, original_len=2048)
        q, k = cpu_normal((B, T, H, 128), 1, dtype).cuda(), cpu_normal((B, T, Hk, 128), 2, dtype).cuda()
        qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
        glide.glide_rope(q, k, freqs, qo, ko, interleaved=inter, mscale=m, backward=back, **kw)
        torch.cuda.synchronize()
        for got, x in ((qo, q), (ko, k)):
            _check(got, x, pos, f64(freqs), m, inter, back)


@pytest.mark.parametrize("inter", [False, True], ids=["half", "inter"])
@pytest.mark.parametrize("rot", [128, 50])
def test_in_place_on_a_fused_projection(inter, rot):
    """Queries and keys as slices of one [B, T, (H + 2 Hk) * D] projection,
    turned in place: the values beside them stay as they are."""
    require_gpu()
    B, T, H, Hk = 2, 9, 6, 2
    freqs, _ = glide.rope_frequencies(rot)
    x = cpu_normal((B, T, H + 2 * Hk, 128), 3, BF).cuda()
    before = x.clone()
    q, k = x[:, :, :H], x[:, :, H:H + Hk]
    lens = torch.tensor([5, 900], dtype=I32, device="cuda")
    glide.glide_rope(q, k, freqs, q, k, seq_lens=lens, interleaved=inter)
    torch.cuda.synchronize()
    pos = np.array([[5], [900]]) + np.arange(T)
    _check(x[:, :, :H + Hk], before[:, :, :H + Hk], pos, f64(freqs), 1.0, inter, False)
    assert torch.equal(x[:, :, H + Hk:], before[:, :, H + Hk:])
    # ... and from heads-first storage into a contiguous tensor, without keys
    t = before[:, :, :H].transpose(1, 2).contiguous().transpose(1, 2)
    out = torch.empty_like(before[:, :, :H].contiguous())
    glide.glide_rope(t, None, freqs, out, None, seq_lens=lens, interleaved=inter)
    torch.cuda.synchronize()
    assert torch.equal(out, x[:, :, :H])


@pytest.mark.parametrize("inter", [False, True], ids=["half", "inter"])
def test_backward_is_the_gradient(inter):
    """<g, f(x)> = <f'(g), x> for every pair of float32 tensors, and the map's
    differences: float32 sums of 128 products a row."""
    require_gpu()
    x, g = cpu_normal((2, 6, 3, 128), 4, F32).cuda(), cpu_normal((2, 6, 3, 128), 5, F32).cuda()
    freqs, m = glide.rope_frequencies(96, scaling="yarn", factor=4.0, original_len=256)
    y, gx, y2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    kw = dict(interleaved=inter, mscale=m)
    glide.glide_rope(x, None, freqs, y, None, **kw)
    glide.glide_rope(g, None, freqs, gx, None, backward=True, **kw)
    a, b = (g.double() * y.double()).sum(), (gx.double() * x.double()).sum()
    size = (g.double().abs() * y.double().abs()).sum()
    assert abs(float(a - b)) <= 4e-6 * float(size)
    step = torch.zeros_like(x)
    step[1, 4, 2, 11] = 0.5
    glide.glide_rope(x + step, None, freqs, y2, None, **kw)
    torch.cuda.synchronize()
    diff = float((g.double() * (y2.double() - y.double())).sum() / 0.5)
    assert abs(diff - float(gx[1, 4, 2, 11])) <= 2e-5 * float(g.abs().max() + x.abs().max())


def test_copied_dims_may_be_anything():
    require_gpu()
    freqs, _ = glide.rope_frequencies(32)
    x = cpu_normal((1, 2, 1, 128), 6, BF).cuda()
    x[..., 40], x[..., 41], x[..., 127] = float("inf"), float("nan"), -float("inf")
    for inter in (False, True):
        y = torch.empty_like(x)
        glide.glide_rope(x, None, freqs, y, None, interleaved=inter)
        assert torch.equal(y[..., 32:].view(torch.int16), x[..., 32:].view(torch.int16))
        assert torch.isfinite(y[..., :32]).all()


def test_bad_parents_are_roots_and_validation_refuses_them(monkeypatch):
    require_gpu()
    freqs, _ = glide.rope_frequencies(128)
    q = cpu_normal((1, 4, 1, 128), 7, F32).cuda()
    bad = torch.tensor([[-1, 5, -7, 2]], dtype=I32, device="cuda")
    good = torch.tensor([[-1, -1, -1, 2]], dtype=I32, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(q)
    glide.glide_rope(q, None, freqs, a, None, tree_parents=bad)
    glide.glide_rope(q, None, freqs, b, None, tree_parents=good)
    assert torch.equal(a, b)
    monkeypatch.setenv("GLIDE_VALIDATE", "1")
    with pytest.raises(glide.GlideError) as e:
        glide.glide_rope(q, None, freqs, a, None, tree_parents=bad)
    assert e.value.status == glide.GLIDE_ERANGE
    glide.glide_rope(q, None, freqs, a, None, tree_parents=good)


def test_refusals():
    require_gpu()
    q, k = torch.zeros((2, 4, 3, 128), dtype=BF, device="cuda"), torch.zeros((2, 4, 1, 128), dtype=BF, device="cuda")
    freqs, _ = glide.rope_frequencies(128)
    pos, lens, par = (torch.zeros(s, dtype=I32, device="cuda") for s in ((2, 4), (2,), (2, 4)))
    wide = torch.zeros((2, 65, 1, 128), dtype=BF, device="cuda")
    odd = torch.zeros((2, 4, 3, 132), dtype=BF, device="cuda")
    for args, kw in (
            ((q.half(), None, freqs, q.half(), None), {}),
            ((q, None, freqs, q.float(), None), {}),
            ((q, k.float(), freqs, q, k.float()), {}),
            ((q, k, freqs, q, None), {}),
            ((q, None, freqs, q, k), {}),
            ((q, k[:1], freqs, q, k[:1]), {}),
            ((q, k, freqs, q, q), {}),
            ((q[..., :64], None, freqs, q[..., :64], None), {}),
            ((q[0], None, freqs, q[0], None), {}),
            ((odd[..., 2:130], None, freqs, q, None), {}),
            ((q, None, freqs, odd[..., :128], None), {}),
            ((q, None, freqs, k.expand(2, 4, 3, 128), None), {}),
            ((q, None, freqs.float(), q, None), {}),
            ((q, None, torch.ones(65, dtype=torch.float64, device="cuda"), q, None), {}),
            ((q, None, freqs.cpu(), q, None), {}),
            ((q, None, freqs, q, None), dict(positions=pos, seq_lens=lens)),
            ((q, None, freqs, q, None), dict(positions=pos, tree_parents=par)),
            ((q, None, freqs, q, None), dict(positions=pos[:1])),
            ((q, None, freqs, q, None), dict(seq_lens=lens.long())),
            ((q, None, freqs, q, None), dict(tree_parents=par[:, :3])),
            ((wide, None, freqs, wide, None), dict(tree_parents=torch.zeros((2, 65), dtype=I32, device="cuda")))):
        with pytest.raises((ValueError, glide.GlideError)):
            glide.glide_rope(*args, **kw)
    glide.glide_rope(k.expand(2, 4, 3, 128), None, freqs, q, None)  # rows that are read may share memory


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rot", [50, 126, 12])
def test_pairs_across_pieces_over_many_heads(dtype, rot):
    """Pairs whose dims lie in different pieces, more heads than a workgroup's
    threads take at once, so that a row's copy in LDS is replaced several times;
    into other rows and in place."""
    require_gpu()
    B, T, H, Hk = 2, 3, 96, 37
    freqs, m = glide.rope_frequencies(rot)
    q, k = cpu_normal((B, T, H, 128), 8, dtype).cuda(), cpu_normal((B, T, Hk, 128), 9, dtype).cuda()
    pos = np.array([[0, 7, 100001], [5, 6, 4000]], dtype=np.int32)
    where = torch.from_numpy(pos).cuda()
    for back in (False, True):
        say("many heads", str(dtype), rot, back)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        glide.glide_rope(q, k, freqs, qo, ko, positions=where, backward=back)
        qi, ki = q.clone(), k.clone()
        glide.glide_rope(qi, ki, freqs, qi, ki, positions=where, backward=back)
        torch.cuda.synchronize()
        for got, x in ((qo, q), (ko, k)):
            _check(got, x, pos, f64(freqs), m, False, back)
        assert torch.equal(qi, qo) and torch.equal(ki, ko)
