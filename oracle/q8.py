"""Oracle: a key/value cache held in 8 bits (test infrastructure only).

The cache is kept here as plain lists: ``Cache.tokens`` holds every final token
of a sequence and head, and what the 8-bit storage makes of a token is derived
from the definition: tokens of whole blocks of 32 are code * scale with
scale = fl32(max |x| / M) and code = the nearest value of the type to
fl32(x / scale), ties to even; tokens behind the last whole block are as given.
"""

import numpy as np

from .attention import ancestor_or_self, attention_rows

BLOCK = 32
MOST = {"e4m3": 448.0, "int8": 127.0}


def e4m3_values():
    """Every finite magnitude of the type, in order: 3 mantissa bits, exponents
    -6 .. 8 (the all-ones code is not a number), and the steps of 2^-9 below."""
    small = [i * 2.0 ** -9 for i in range(8)]
    large = [(1 + i / 8) * 2.0 ** e for e in range(-6, 9) for i in range(8)]
    return np.array(small + large[:-1])


def nearest_e4m3(y):
    """The nearest value of the type to y, ties to the even code."""
    table = e4m3_values()
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(table, a), 1, len(table) - 1)
    lo = hi - 1
    up = (table[hi] - a < a - table[lo]) | ((table[hi] - a == a - table[lo]) & (hi % 2 == 0))
    return np.copysign(np.where(up, table[hi], table[lo]), y)


def quantise(x, kind):
    """x [32, 128] -> (codes as numbers, scale)."""
    x = np.asarray(x, dtype=np.float32)
    scale = np.float32(np.abs(x).max()) / np.float32(MOST[kind])
    if scale < np.float32(2.0 ** -126):
        return np.zeros(x.shape), 0.0
    y = (x / scale).astype(np.float64)  # the float32 quotient
    y = np.clip(y, -MOST[kind], MOST[kind])
    return (nearest_e4m3(y) if kind == "e4m3" else np.rint(y)), float(scale)


def stored(rows, kind):
    """What the cache holds of the final tokens rows [L, 128]."""
    rows = np.asarray(rows, dtype=np.float64)
    out = rows.copy()
    for i in range(len(rows) // BLOCK):
        codes, scale = quantise(rows[i * BLOCK:(i + 1) * BLOCK], kind)
        out[i * BLOCK:(i + 1) * BLOCK] = codes * scale
    return out


def block_bytes(k_codes, v_codes):
    """[8192] code numbers of a block in the order of its bytes, loop by loop."""
    out = np.empty(8192)
    for kt in range(2):
        for h in range(2):
            for g in range(4):
                for c in range(16):
                    for e in range(16):
                        out[((kt * 2 + h) * 64 + 16 * g + c) * 16 + e] = k_codes[16 * kt + c, 64 * h + 16 * g + e]
    for u in range(4):
        for g in range(4):
            for c in range(16):
                for t in range(2):
                    for j in range(2):
                        for i in range(4):
                            out[4096 + (u * 64 + 16 * g + c) * 16 + 8 * t + 4 * j + i] = \
                                v_codes[16 * j + 4 * g + i, 8 * c + 2 * u + t]
    return out


def tree_attention(q, k, v, lens, kind, k_tree=None, v_tree=None, parents=None, scale=None):
    """q [B, N, H, D]; k, v [b][H_kv] final tokens [>= L, D]; k_tree, v_tree [B, N,
    H_kv, D] with parents [B, N] (tree mode).  Float64 [B, N, H, D]."""
    q = np.asarray(q, dtype=np.float64)
    B, N, H, D = q.shape
    h_kv = len(k[0])
    out = np.zeros(q.shape)
    for b in range(B):
        for j in range(h_kv):
            ks, vs = (stored(np.asarray(x[b][j])[:lens[b]], kind) for x in (k, v))
            for n in range(N):
                kk, vv = ks, vs
                if parents is not None:
                    own = ancestor_or_self(parents[b], n)
                    kk = np.concatenate([ks, np.asarray(k_tree[b], dtype=np.float64)[own, j]])
                    vv = np.concatenate([vs, np.asarray(v_tree[b], dtype=np.float64)[own, j]])
                heads = slice(j * (H // h_kv), (j + 1) * (H // h_kv))
                out[b, n, heads] = attention_rows(q[b, n, heads], kk, vv, 1 / np.sqrt(D) if scale is None else scale)
    return out
