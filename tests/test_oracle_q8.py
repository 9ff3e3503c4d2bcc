"""Pins of the oracles of rotary positions and of the 8-bit cache (CPU): each is
checked against something other than itself."""

import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import q8 as OQ
from oracle import rope as OR


# -- rotary positions -------------------------------------------------------

def _rand(shape, seed=0):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_a_rotation_of_complex_pairs(interleaved):
    x, pos = _rand((2, 5, 3, 128)), np.array([[0, 1, 7, 100, 4000], [3, 3, 2, 1, 0]])
    freqs, m = OR.frequencies(64)
    y = OR.rope(x, pos, freqs, 1.5, interleaved)
    a, b = (np.arange(0, 64, 2), np.arange(1, 64, 2)) if interleaved else (np.arange(32), np.arange(32, 64))
    z = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(1j * pos[:, :, None, None] * freqs)
    assert np.allclose(y[..., a], z.real, atol=1e-12) and np.allclose(y[..., b], z.imag, atol=1e-12)
    assert np.array_equal(y[..., 64:], x[..., 64:])


def test_rope_scores_depend_on_distance_alone():
    q, k = _rand((1, 1, 1, 128), 1), _rand((1, 1, 1, 128), 2)
    freqs, _ = OR.frequencies(128)
    dots = [(OR.rope(q, [[p]], freqs) * OR.rope(k, [[p - 9]], freqs)).sum() for p in (9, 50, 12345)]
    assert np.allclose(dots, dots[0])


def test_rope_backward_is_the_transposed_map():
    x, g, pos = _rand((1, 4, 2, 128), 3), _rand((1, 4, 2, 128), 4), [[0, 5, 6, 70]]
    freqs, m = OR.frequencies(96, scaling="yarn", factor=4.0, original_len=64)
    assert m > 1.0
    for inter in (False, True):
        y = OR.rope(x, pos, freqs, m, inter)
        gx = OR.rope(g, pos, freqs, m, inter, backward=True)
        assert np.isclose((g * y).sum(), (gx * x).sum())
        # differences: the map is linear, so a step of any size gives its column
        e = np.zeros_like(x)
        e[0, 3, 1, 10] = 1e-3
        diff = (OR.rope(x + e, pos, freqs, m, inter) - y) / 1e-3
        assert np.isclose((g * diff).sum(), gx[0, 3, 1, 10], atol=1e-9)


def test_frequencies():
    f, m = OR.frequencies(128)
    assert m == 1.0 and f[0] == 1.0 and np.isclose(f[32], 0.01) and np.isclose(f[63], 10000.0 ** (-126 / 128))
    assert np.allclose(OR.frequencies(128, scaling="linear", factor=4.0)[0], f / 4)
    ntk = OR.frequencies(128, scaling="ntk", factor=4.0)[0]
    assert ntk[0] == 1.0 and np.isclose(ntk[63], f[63] / 4)  # the slowest pair as if positions were divided
    yarn, m = OR.frequencies(128, scaling="yarn", factor=4.0, original_len=4096)
    turns = 4096 * f / (2 * math.pi)
    assert np.allclose(yarn[turns >= 32], f[turns >= 32]) and np.allclose(yarn[turns <= 1], f[turns <= 1] / 4)
    assert np.all(yarn <= f) and np.all(yarn >= f / 4) and np.isclose(m, 0.1 * math.log(4) + 1)


def test_tree_positions():
    assert OR.tree_positions(10, [-1, 0, 1, 0, 3, -1]) == [10, 11, 12, 11, 12, 10]


# -- the 8-bit cache --------------------------------------------------------

def test_e4m3_rounding_equals_torch():
    assert len(OQ.e4m3_values()) == 127 and OQ.e4m3_values()[-1] == 448.0
    y = np.concatenate([_rand(20000, 5) * 100, _rand(20000, 6) * 0.02, OQ.e4m3_values(),
                        (OQ.e4m3_values()[1:] + OQ.e4m3_values()[:-1]) / 2])
    y = np.clip(np.concatenate([y, -y]), -448, 448).astype(np.float32).astype(np.float64)
    want = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(OQ.nearest_e4m3(y), want)


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_quantise(kind):
    x = _rand((32, 128), 7).astype(np.float32)
    codes, scale = OQ.quantise(x, kind)
    top = np.abs(x).argmax()
    assert abs(codes.flat[top]) == OQ.MOST[kind]  # the largest value is the largest code
    step = np.maximum(np.abs(codes) * 2.0 ** -4, 2.0 ** -10) if kind == "e4m3" else 0.5
    assert np.all(np.abs(codes * scale - x) <= scale * step * (1 + 1e-6))
    assert OQ.quantise(np.zeros((32, 128)), kind) == (pytest.approx(np.zeros((32, 128))), 0.0)
    tiny, s = OQ.quantise(np.full((32, 128), 1e-37, dtype=np.float32), kind)  # a scale below 2^-126
    assert s == 0.0 and not tiny.any()
    y = OQ.stored(np.concatenate([x, x[:5]]), kind)
    assert np.allclose(y[:32], codes * scale) and np.array_equal(y[32:], x[:5])


def test_block_bytes_hold_every_value_once():
    k, v = np.arange(4096.0).reshape(32, 128), 5000 + np.arange(4096.0).reshape(32, 128)
    out = OQ.block_bytes(k, v)
    assert sorted(out[:4096]) == sorted(k.flat) and sorted(out[4096:]) == sorted(v.flat)
    # a unit of 16 K bytes is 16 dims of a token; of V, two dims of eight tokens
    assert np.array_equal(out[:16], k[0, :16]) and np.array_equal(out[16:32], k[1, :16])
    assert np.array_equal(out[4096:4112], [5000 + 128 * t + d for d in (0, 1) for t in (0, 1, 2, 3, 16, 17, 18, 19)])


def test_attention_equals_plain_attention_over_stored_rows():
    B, N, H, Hk, L = 1, 3, 4, 2, 70
    q = _rand((B, N, H, 128), 8)
    k, v = _rand((B, Hk, L, 128), 9), _rand((B, Hk, L, 128), 10)
    kt, vt = _rand((B, N, Hk, 128), 11), _rand((B, N, Hk, 128), 12)
    par = [[-1, 0, 0]]
    got = OQ.tree_attention(q, k, v, [L], "int8", kt, vt, par)
    for h in range(H):
        kc = np.concatenate([OQ.stored(k[0, h // 2], "int8"), kt[0, :, h // 2]])
        vc = np.concatenate([OQ.stored(v[0, h // 2], "int8"), vt[0, :, h // 2]])
        want = OA.tree_attention_head(q[0, :, h], kc, vc, L, par[0])
        assert np.allclose(got[0, :, h], want)
    assert np.array_equal(OQ.tree_attention(q, k, v, [0], "int8"), np.zeros(q.shape))
