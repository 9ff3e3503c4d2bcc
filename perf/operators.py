"""Performance cases of decoding over a key/value cache held in 8 bits.

Rotary positions of prompt, training and tree rows; a cache written in 8 bits
and read back; tree and cross attention over it; and the commit of accepted
rows.  ``prepare`` builds what a program holds before the call, ``run`` makes
one pass (the library's calls where ``own`` is true, else the same operators
in elementary torch operations), ``exact`` is the same result from the
definitions in float64, and ``draw`` gives further cases of the same ranges.

The cache of one layer is a triple:
  blocks [B, H_kv, blocks, 8192], one byte each: 32 tokens of K, then of V.
         K byte [kt][h][g][c][b] is token 16 kt + c, dim 64 h + 16 g + b;
         V byte [u][g][c][t][j][i] is token 16 j + 4 g + i, dim 8 c + 2 u + t.
         float8_e4m3fn values, or uint8 holding integers of -127..127 plus 128.
  scales [B, H_kv, blocks, 2] float32: what the K and V values are times.
  tail   [B, H_kv, 2, 128, 128] bfloat16: K and V rows of the tokens behind
         the last whole block; token j at row j % 128.

Sequence lengths of a batch are spread evenly over [lo, hi] in an order that
depends on the seed, so every seed has the same total work.
"""

import math

import torch

own = False

D, BLOCK, TAIL = 128, 32, 128
DEV = "cuda"
BF16, F32, F64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
MOST = dict(e4m3=448.0, int8=127.0)
TINY = 2.0 ** -126


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # Rotary positions of a 5-token chain's queries and keys in one 7B
        # layer: the smallest call of a decoding step.
        dict(name="rope_chain5", kind="rope", B=1, T=5, H=32, Hkv=32, rot=128, inter=False, dtype="bf16",
             where="tree", lo=512, hi=512, yarn=False, back=False),
        # A training batch's backward pass: four 2048-token sequences, grouped
        # heads, adjacent pairs, frequencies scaled for long contexts.
        dict(name="rope_train_back", kind="rope", B=4, T=2048, H=32, Hkv=8, rot=128, inter=True, dtype="bf16",
             where="start", lo=0, hi=0, yarn=True, back=True),
        # The tree rows of one 7B layer, written where verification reads
        # them; nothing is quantised before the tree is verified.
        dict(name="hold_tree16", kind="append", B=1, T=16, H=32, q8="e4m3", lo=2040, hi=2040, hold=True),
        # A batch of four 2048-token prompts written to one layer's cache.
        dict(name="append_prompt", kind="append", B=4, T=2048, H=32, q8="e4m3", lo=0, hi=0, hold=False),
        # A cache expanded for a consumer of bfloat16 rows: one long sequence.
        dict(name="read_long", kind="read", B=1, H=8, q8="int8", lo=32750, hi=32750, out="bf16"),
        # The same for a ragged batch, in float32.
        dict(name="read_batch_f32", kind="read", B=8, H=8, q8="e4m3", lo=100, hi=700, out="f32"),
        # One 7B layer verifying a 5-token chain early in a chat.
        dict(name="attn_chain5", kind="attn", B=1, H=32, Hkv=32, N=5, depth=5, lo=512, hi=512, q8="e4m3", cross=False),
        # A verification layer of a 13B target: ragged batch, 32-node trees.
        dict(name="attn_13b", kind="attn", B=4, H=40, Hkv=40, N=32, depth=6, lo=1024, hi=4096, q8="int8",
             cross=False),
        # Plain decoding, one query a sequence, four query heads to a cached
        # head, as in models with grouped heads.
        dict(name="attn_decode_gqa", kind="attn", B=16, H=32, Hkv=8, N=1, depth=1, lo=2048, hi=8192, q8="e4m3",
             cross=False),
        # The draft's 5-query cross attention over long contexts: the largest
        # call, 3.2 GB of keys and values.
        dict(name="attn_cross_long", kind="attn", B=16, H=32, Hkv=32, N=5, depth=5, lo=16384, hi=32768, q8="int8",
             cross=True),
        # The accepted paths of a 13B target committed in all 40 layers.
        dict(name="commit_13b", kind="commit", B=4, H=40, N=32, depth=6, lo=216, hi=232, layers=40, q8="e4m3",
             chain=False),
        # The same for a batch of sampled chains, grouped heads, in integers;
        # the end of the cache is read back.
        dict(name="commit_chains_int8", kind="commit", B=16, H=8, N=12, depth=12, lo=40, hi=72, layers=8, q8="int8",
             chain=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _nodes(rng):
    N = rng.choice([1, rng.randint(1, 16), rng.randint(17, 32), rng.randint(33, 64)])
    return N, min(N, rng.randint(max(3, (N + 7) // 8), 10))


def draw(rng):
    kind = rng.choice(["rope", "rope", "append", "append", "read", "attn", "attn", "attn", "attn", "commit"])
    q8 = rng.choice(["e4m3", "int8"])
    if kind == "rope":
        where = rng.choice(["tree", "start", "given"])
        T = _log_int(rng, 1, 64 if where == "tree" else 4096)
        H, Hkv = rng.choice([(8, 8), (12, 4), (20, 20), (32, 8), (32, 32), (40, 40)])
        B = _log_int(rng, 1, max(1, min(16, 16384 // T)))
        hi = _log_int(rng, 16, 200000)
        return dict(kind=kind, B=B, T=T, H=H, Hkv=Hkv, rot=rng.choice([128, 128, 64, 96, 2 * rng.randint(1, 64)]),
                    inter=rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]), where=where, lo=hi // 2,
                    hi=hi, yarn=rng.random() < 0.5, back=rng.random() < 0.4)
    if kind == "append":
        hold = rng.random() < 0.3
        T = _log_int(rng, 1, 64 if hold else 4096)
        B, H = _log_int(rng, 1, max(1, min(32, 12000 // T))), rng.choice([4, 8, 20, 32, 40])
        lo = rng.choice([0, _log_int(rng, 1, 4096)])
        return dict(kind=kind, B=B, T=T, H=H, q8=q8, lo=lo, hi=lo + rng.randint(0, 64), hold=hold)
    if kind == "read":
        B, H = _log_int(rng, 1, 16), rng.choice([4, 8, 20, 32])
        hi = _log_int(rng, 1, min(65536, 1500000 // (B * H)))
        return dict(kind=kind, B=B, H=H, q8=q8, lo=int(hi * rng.uniform(0.25, 1.0)), hi=hi,
                    out=rng.choice(["bf16", "f32"]))
    if kind == "attn":
        N, depth = _nodes(rng)
        B = _log_int(rng, 1, 32)
        H, Hkv = rng.choice([(8, 8), (20, 20), (32, 32), (40, 40), (52, 52), (32, 8), (64, 8), (12, 4)])
        hi = _log_int(rng, 1, max(1, min(65536, 9000000 // (B * Hkv), 250000000 // (B * N * H))))
        return dict(kind=kind, B=B, H=H, Hkv=Hkv, N=N, depth=depth, lo=int(hi * rng.uniform(0.25, 1.0)), hi=hi,
                    q8=q8, cross=rng.random() < 0.3)
    N, depth = _nodes(rng)
    B, H = _log_int(rng, 1, 16), rng.choice([4, 8, 20, 32, 40])
    lo = _log_int(rng, 1, 400)
    return dict(kind=kind, B=B, H=H, N=N, depth=depth, lo=lo, hi=lo + rng.randint(0, 40),
                layers=rng.randint(1, max(1, min(60, 9000 // (B * H)))), q8=q8, chain=rng.random() < 0.3)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

class _Rand:
    """Seeded draws on the GPU, and small host-side choices."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.h = torch.Generator()
        self.h.manual_seed(seed)

    def normal(self, shape, dtype=F32):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=self.g)

    def order(self, n):
        return torch.randperm(n, generator=self.h).tolist()

    def pick(self, n):
        return int(torch.randint(n, (1,), generator=self.h))


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _lengths(c):
    B = c["B"]
    return [c["lo"] + (c["hi"] - c["lo"]) * (2 * i + 1) // (2 * B) for i in range(B)]


def _lens(c, r):
    lens = _lengths(c)
    return [lens[i] for i in r.order(len(lens))]


def _tree(N, depth, r):
    """Parents of a chain of `depth` nodes followed by its leaves, in position
    order (the linearised form CaPE emits)."""
    leaves = sorted(r.pick(depth) for _ in range(N - depth))
    return [i - 1 for i in range(depth)] + [p - 1 for p in leaves]


def _key_channels(H, r):
    """Keys' channels differ in size, some by far."""
    return torch.exp(0.5 * r.normal((H, 1, D)))


def _rows(B, H, T, r, channels=None):
    x = r.normal((B, H, T, D))
    return (x if channels is None else x * channels).to(BF16)


def _cache(B, H, tokens, q8, r):
    """A cache with room for `tokens`, every block and every tail row filled."""
    n = -(-tokens // BLOCK)
    ch = _key_channels(H, r)
    blocks = torch.empty((B, H, n, 2 * BLOCK * D), dtype=E4M3 if q8 == "e4m3" else torch.uint8, device=DEV)
    scales = torch.empty((B, H, n, 2), dtype=F32, device=DEV)
    for b in range(B):
        for m in range(2):
            x = _rows(1, H, n * BLOCK, r, ch if m == 0 else None).view(1, H, n, BLOCK, D)
            codes, scales[b:b + 1, :, :, m] = _quantise(x, q8)
            half = _pack_k(codes) if m == 0 else _pack_v(codes)
            blocks[b:b + 1, :, :, m * BLOCK * D:(m + 1) * BLOCK * D] = half
    tail = torch.stack([_rows(B, H, TAIL, r, ch), _rows(B, H, TAIL, r)], dim=2)
    return blocks, scales, tail


def _frequencies(c):
    """Angles per position of each pair (float64), and the magnitude.  With
    yarn, frequencies that turn less than once over the original 4096
    positions are divided by 8, those that turn over 32 times are kept."""
    half = c["rot"] // 2
    f = [10000.0 ** (-i / half) for i in range(half)]
    if not c["yarn"]:
        return torch.tensor(f, dtype=F64, device=DEV), 1.0
    keep = [min(1.0, max(0.0, (4096 * x / (2 * math.pi) - 1.0) / 31.0)) for x in f]
    f = [x * k + x / 8 * (1 - k) for x, k in zip(f, keep)]
    return torch.tensor(f, dtype=F64, device=DEV), 0.1 * math.log(8.0) + 1.0


def _rope_state(c, r):
    dtype = BF16 if c["dtype"] == "bf16" else F32
    B, T = c["B"], c["T"]
    s = dict(c=c, q=r.normal((B, T, c["H"], D), dtype), k=r.normal((B, T, c["Hkv"], D), dtype), positions=None,
             lens=None, parents=None)
    s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    s["freqs"], s["m"] = _frequencies(c)
    if c["where"] == "given":
        s["positions"] = torch.randint(c["hi"] + 1, (B, T), generator=r.g, device=DEV, dtype=torch.int32)
    else:
        s["lens"] = _int32(_lens(c, r))
        if c["where"] == "tree":
            depth = min(T, 3 + T // 8)
            s["parents"] = _int32([_tree(T, depth, r) for _ in range(B)])
    return s


def _append_state(c, r):
    B, T, H = c["B"], c["T"], c["H"]
    s = dict(c=c, lens=_int32(_lens(c, r)), cache=_cache(B, H, c["hi"] + T + BLOCK, c["q8"], r))
    s["k"] = _rows(B, H, T, r, _key_channels(H, r)).transpose(1, 2).contiguous()
    s["v"] = _rows(B, H, T, r).transpose(1, 2).contiguous()
    if c["q8"] == "int8" and not c["hold"]:
        s["new_lens"] = s["lens"] + T
        _read_buffers(s, B)
    return s


def _start(c):
    return c["lo"] // BLOCK * BLOCK  # the first token that a call may have quantised


def _read_buffers(s, rows):
    """Where the end of an integer cache is read back to."""
    c = s["c"]
    shape = (rows, c["H"], c["hi"] + c.get("T", 64) - _start(c), D)
    s["k_out"], s["v_out"] = torch.zeros(shape, dtype=BF16, device=DEV), torch.zeros(shape, dtype=BF16, device=DEV)


def _read_state(c, r):
    dtype = BF16 if c["out"] == "bf16" else F32
    s = dict(c=c, lens=_int32(_lens(c, r)), cache=_cache(c["B"], c["H"], c["hi"], c["q8"], r))
    shape = (c["B"], c["H"], c["hi"], D)
    s["k_out"], s["v_out"] = torch.zeros(shape, dtype=dtype, device=DEV), torch.zeros(shape, dtype=dtype, device=DEV)
    return s


def _attn_state(c, r):
    B, N = c["B"], c["N"]
    s = dict(c=c, lens=_int32(_lens(c, r)), cache=_cache(B, c["Hkv"], c["hi"], c["q8"], r))
    s["q"] = r.normal((B, N, c["H"], D), BF16)
    s["parents"] = None if c["cross"] else _int32([_tree(N, c["depth"], r) for _ in range(B)])
    s["out"] = torch.empty_like(s["q"])
    return s


def _accepted(c):
    """Accepted tokens of each sequence: as many as the depth allows, in turn."""
    return [(2 * i + c["depth"] // 2) % (c["depth"] + 1) for i in range(c["B"])]


def _commit_state(c, r):
    B, N, H, L = c["B"], c["N"], c["H"], c["layers"]
    lens, accept, order = _lengths(c), _accepted(c), r.order(B)
    s = dict(c=c, lens=_int32([lens[i] for i in order]))
    accept = [accept[i] for i in order]
    paths = []
    for a in accept:
        # a path down the chain whose last node is a leaf, as often as not
        nodes = list(range(a))
        if a and N > c["depth"] and r.pick(2):
            nodes[-1] = c["depth"] + r.pick(N - c["depth"])
        paths.append(nodes + [-1] * (N - a))
    s["accept"], s["path"] = _int32(accept), None if c["chain"] else _int32(paths)
    s["lens_out"] = torch.empty_like(s["lens"])
    # the layers' caches are views of one; a sequence of a layer is a row
    s["all"] = _cache(L * B, H, c["hi"] + 64 + BLOCK, c["q8"], r)
    s["caches"] = [tuple(t[i * B:(i + 1) * B] for t in s["all"]) for i in range(L)]
    if c["q8"] == "int8":
        _read_buffers(s, L * B)
    return s


_STATES = dict(rope=_rope_state, append=_append_state, read=_read_state, attn=_attn_state, commit=_commit_state)


def prepare(case, seed):
    return _STATES[case["kind"]](case, _Rand(seed))


# ---------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------

def _run_own(s):
    import paper_2402_02082_amd as glide

    c = s["c"]
    if c["kind"] == "rope":
        glide.glide_rope(s["q"], s["k"], s["freqs"], s["q_out"], s["k_out"], positions=s["positions"],
                         seq_lens=s["lens"], tree_parents=s["parents"], interleaved=c["inter"], mscale=s["m"],
                         backward=c["back"])
        return dict(q=s["q_out"], k=s["k_out"])
    if c["kind"] == "append":
        glide.glide_q8_append(s["k"], s["v"], s["cache"], s["lens"], hold=c["hold"])
        if c["hold"]:
            return dict(tail=s["cache"][2])
        return _stored(s, s["cache"], lambda: glide.glide_q8_read(s["cache"], s["new_lens"], s["k_out"], s["v_out"],
                                                                  start=_start(c)))
    if c["kind"] == "read":
        glide.glide_q8_read(s["cache"], s["lens"], s["k_out"], s["v_out"])
        return dict(k=s["k_out"], v=s["v_out"])
    if c["kind"] == "attn":
        return glide.glide_q8_tree_attn(s["q"], s["cache"], s["lens"], s["parents"], s["out"])
    glide.glide_q8_commit(s["caches"], s["lens"], s["accept"], s["path"], s["lens_out"])
    stored = _stored(s, s["all"], lambda: glide.glide_q8_read(s["all"], s["lens_out"].repeat(c["layers"]), s["k_out"],
                                                              s["v_out"], start=_start(c)))
    return dict(stored, lens=s["lens_out"])


def _stored(s, cache, read):
    """What a cache holds: e4m3 values with their scales as they are, integers
    read back."""
    blocks, scales, tail = cache
    if s["c"]["q8"] == "e4m3":
        return dict(values=blocks, scales=scales, tail=tail)
    read()
    return dict(k=s["k_out"], v=s["v_out"], scales=scales, tail=tail)


def run(s):
    if own:
        return _run_own(s)
    return _PLAIN[s["c"]["kind"]](s)


# ---------------------------------------------------------------------------
# The plain form
# ---------------------------------------------------------------------------

def _quantise(x, q8):
    """x [..., 32, 128] -> (float32 values that 8 bits hold, scales [...])."""
    x = x.to(F32)
    scale = x.abs().amax(dim=(-1, -2))
    scale = scale / torch.full_like(scale, MOST[q8])  # a division: by a number, torch multiplies with its inverse
    scale = torch.where(scale < TINY, torch.zeros_like(scale), scale)
    s = scale[..., None, None]
    y = torch.where(s > 0, x / s, torch.zeros_like(x)).clamp(-MOST[q8], MOST[q8])
    return (y.to(E4M3) if q8 == "e4m3" else (torch.round(y) + 128).to(torch.uint8)), scale


def _pack_k(codes):
    lead = codes.shape[:-2]
    x = codes.reshape(*lead, 2, 16, 2, 4, 16)  # kt c h g b
    n = len(lead)
    return x.permute(*range(n), n, n + 2, n + 3, n + 1, n + 4).reshape(*lead, BLOCK * D)


def _pack_v(codes):
    lead = codes.shape[:-2]
    x = codes.reshape(*lead, 2, 4, 4, 16, 4, 2)  # j g i c u t
    n = len(lead)
    return x.permute(*range(n), n + 4, n + 1, n + 3, n + 5, n, n + 2).reshape(*lead, BLOCK * D)


def _unpack(blocks, scales, dtype):
    """(K, V) [..., 32 blocks, 128] that the blocks [..., blocks, 8192] stand for."""
    lead = blocks.shape[:-2]
    n = len(lead) + 1
    k = blocks[..., :BLOCK * D].reshape(*blocks.shape[:-1], 2, 2, 4, 16, 16)  # kt h g c b
    v = blocks[..., BLOCK * D:].reshape(*blocks.shape[:-1], 4, 4, 16, 2, 2, 4)  # u g c t j i
    k = k.permute(*range(n), n, n + 3, n + 1, n + 2, n + 4).reshape(*blocks.shape[:-1], BLOCK, D)
    v = v.permute(*range(n), n + 4, n + 1, n + 5, n + 2, n, n + 3).reshape(*blocks.shape[:-1], BLOCK, D)
    off = 128 if blocks.dtype == torch.uint8 else 0
    k = (k.to(dtype) - off) * scales[..., 0, None, None].to(dtype)
    v = (v.to(dtype) - off) * scales[..., 1, None, None].to(dtype)
    return k.reshape(*lead, -1, D), v.reshape(*lead, -1, D)


def _tree_depths(parents):
    """Ancestors of every node: the parents followed up until none is left."""
    B, N = parents.shape
    up = torch.eye(N, dtype=F32, device=DEV).repeat(B, 1, 1)
    one = torch.zeros((B, N, N + 1), dtype=F32, device=DEV)
    one.scatter_(2, (parents.long() + 1)[..., None], 1.0)
    reach, step = up, one[..., 1:]
    size = 1
    while size < N:  # relations of up to 2 * size steps from those of up to size
        reach, step, size = torch.clamp(reach + torch.matmul(step, reach), max=1.0), torch.matmul(step, step), 2 * size
    return reach > 0  # [B, N, N]: m is n or an ancestor of n


def _positions(s):
    c = s["c"]
    if s["positions"] is not None:
        return s["positions"]
    if s["parents"] is not None:
        return s["lens"][:, None] + _tree_depths(s["parents"]).sum(-1) - 1
    return s["lens"][:, None] + torch.arange(c["T"], device=DEV)


def _rope_plain(s):
    c, half = s["c"], s["c"]["rot"] // 2
    angle = _positions(s).to(F64)[..., None] * s["freqs"]
    cos, sin = (torch.cos(angle) * s["m"]).to(F32)[:, :, None], (torch.sin(angle) * s["m"]).to(F32)[:, :, None]
    sin = -sin if c["back"] else sin

    def turn(x):
        f = x.to(F32)
        a, b = (f[..., 0:c["rot"]:2], f[..., 1:c["rot"]:2]) if c["inter"] else (f[..., :half], f[..., half:c["rot"]])
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1 if c["inter"] else -2)
        return torch.cat([y.flatten(-2), f[..., c["rot"]:]], dim=-1).to(x.dtype)

    return dict(q=turn(s["q"]), k=turn(s["k"]))


def _write_blocks(cache, first, at, valid, source, q8):
    """Quantises tokens [first, first + 32 n) of each sequence where valid
    [B, n]; source(m) gives K (0) or V (1) as [B, H, 32 n, 128]."""
    blocks, scales, _ = cache
    B, H = blocks.shape[:2]
    n = valid.shape[1]
    b = torch.arange(B, device=DEV)[:, None, None]
    h = torch.arange(H, device=DEV)[None, :, None]
    at = at[:, None, :]
    raw = blocks.view(torch.uint8)
    old_scale = scales[b, h, at]
    new, new_scale = [], []
    for m, pack in ((0, _pack_k), (1, _pack_v)):
        codes, sc = _quantise(source(m).reshape(B, H, n, BLOCK, D), q8)
        new.append(pack(codes).view(torch.uint8))
        new_scale.append(sc)
    ok = valid[:, None, :, None]
    raw[b, h, at] = torch.where(ok, torch.cat(new, dim=-1), raw[b, h, at])
    scales[b, h, at] = torch.where(ok, torch.stack(new_scale, dim=-1), old_scale)


def _write_tail(cache, pos, valid, rows):
    """tail rows of positions pos [B, n] from rows(m) [B, H, n, 128] where valid."""
    tail = cache[2]
    B, H = tail.shape[:2]
    b = torch.arange(B, device=DEV)[:, None, None]
    h = torch.arange(H, device=DEV)[None, :, None]
    at = (pos % TAIL)[:, None, :]
    for m in range(2):
        tail[b, h, m, at] = torch.where(valid[:, None, :, None], rows(m), tail[b, h, m, at])


def _pick_rows(x, at):
    """x [B, H, T, 128], at [B, n] -> [B, H, n, 128]."""
    B, H = x.shape[:2]
    return x.gather(2, at[:, None, :, None].expand(B, H, at.shape[1], D))


def _append_plain(s):
    c, cache, T = s["c"], s["cache"], s["c"]["T"]
    L = s["lens"].long()[:, None]
    new = (s["k"].transpose(1, 2), s["v"].transpose(1, 2))
    if c["hold"]:
        i = torch.arange(T, device=DEV)[None]
        _write_tail(cache, L + i, torch.ones_like(L + i, dtype=torch.bool), lambda m: new[m])
        return dict(tail=cache[2])
    first, end = L // BLOCK * BLOCK, (L + T) // BLOCK * BLOCK
    n = (BLOCK - 1 + T) // BLOCK
    pos = first + torch.arange(n * BLOCK, device=DEV)[None]

    def source(m):
        held = _pick_rows(cache[2][:, :, m], pos % TAIL)
        given = _pick_rows(new[m], (pos - L).clamp(0, T - 1))
        return torch.where((pos < L)[:, None, :, None], held, given)

    at = first // BLOCK + torch.arange(n, device=DEV)[None]
    _write_blocks(cache, first, at, (at + 1) * BLOCK <= end, source, c["q8"])
    i = torch.maximum(L, end) + torch.arange(BLOCK - 1, device=DEV)[None]
    _write_tail(cache, i, i < L + T, lambda m: _pick_rows(new[m], (i - L).clamp(0, T - 1)))
    return _stored(s, cache, lambda: _read_into(cache, s["new_lens"], s["k_out"], s["v_out"], _start(c)))


def _read_into(cache, lens, k_out, v_out, start):
    blocks, scales, tail = cache
    n = k_out.shape[2]
    pos = start + torch.arange(n, device=DEV)
    first = start // BLOCK
    part = slice(first, first + -(-n // BLOCK))
    held = _unpack(blocks[:, :, part], scales[:, :, part], F32)
    whole = (lens.long() // BLOCK * BLOCK)[:, None]
    for m, out in ((0, k_out), (1, v_out)):
        x = torch.zeros_like(out, dtype=F32)
        take = min(n, held[m].shape[2])
        x[:, :, :take] = held[m][:, :, :take]
        x = torch.where((pos[None] < whole)[:, None, :, None], x, tail[:, :, m, pos % TAIL].to(F32))
        out.copy_(torch.where((pos[None] < lens[:, None])[:, None, :, None], x.to(out.dtype), out))


def _read_plain(s):
    _read_into(s["cache"], s["lens"], s["k_out"], s["v_out"], 0)
    return dict(k=s["k_out"], v=s["v_out"])


def _attn_plain(s):
    c = s["c"]
    B, N, H, Hkv = c["B"], c["N"], c["H"], c["Hkv"]
    blocks, scales, tail = s["cache"]
    L = s["lens"].long()
    whole = L // BLOCK * BLOCK
    held = _unpack(blocks, scales, F32)
    C = held[0].shape[2]
    near = whole[:, None] + torch.arange(BLOCK + 64, device=DEV)  # positions of the tail rows, [B, 96]
    k, v = (torch.cat([held[m], _pick_rows(tail[:, :, m], near % TAIL).to(F32)], dim=2) for m in range(2))
    seen = torch.zeros((B, N, C + BLOCK + 64), dtype=torch.bool, device=DEV)
    seen[:, :, :C] = (torch.arange(C, device=DEV)[None] < whole[:, None])[:, None]
    seen[:, :, C:] = (near < L[:, None])[:, None]
    if not c["cross"]:
        node = near - L[:, None]
        mine = _tree_depths(s["parents"]).gather(2, node.clamp(0, N - 1)[:, None].expand(B, N, -1))
        seen[:, :, C:] |= mine & ((node >= 0) & (node < N))[:, None]
    G = H // Hkv
    q = s["q"].to(F32).view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    x = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    x.masked_fill_(~seen.repeat_interleave(G, dim=1)[:, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.view(B, Hkv, N, G, D).permute(0, 2, 1, 3, 4).reshape(B, N, H, D).to(BF16)


def _commit_plain(s):
    c, cache = s["c"], s["all"]
    per = c["layers"]
    L, a = s["lens"].long()[:, None], s["accept"].long()[:, None]
    path = torch.arange(c["N"], device=DEV)[None].expand(c["B"], -1) if s["path"] is None else s["path"].long()
    L, a, path = L.repeat(per, 1), a.repeat(per, 1), path.repeat(per, 1)
    first, end = L // BLOCK * BLOCK, (L + a) // BLOCK * BLOCK
    n = (BLOCK - 1 + c["N"]) // BLOCK
    tail = cache[2].clone()

    def held(pos):  # where position pos's row lies before the commit
        node = path.gather(1, (pos - L).clamp(0, c["N"] - 1))
        return torch.where(pos < L, pos, L + node.clamp(min=0)) % TAIL

    pos = first + torch.arange(n * BLOCK, device=DEV)[None]
    at = first // BLOCK + torch.arange(n, device=DEV)[None]
    if n:
        _write_blocks(cache, first, at, (at + 1) * BLOCK <= end, lambda m: _pick_rows(tail[:, :, m], held(pos)),
                      c["q8"])
    i = torch.maximum(L, end) + torch.arange(BLOCK - 1, device=DEV)[None]
    _write_tail(cache, i, i < L + a, lambda m: _pick_rows(tail[:, :, m], held(i)))
    s["lens_out"].copy_(s["lens"] + s["accept"])
    stored = _stored(s, cache, lambda: _read_into(cache, s["lens_out"].repeat(per), s["k_out"], s["v_out"],
                                                  _start(c)))
    return dict(stored, lens=s["lens_out"])


_PLAIN = dict(rope=_rope_plain, append=_append_plain, read=_read_plain, attn=_attn_plain, commit=_commit_plain)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

ROW = D * 2  # bytes of a bfloat16 row
PAIR = 2 * BLOCK * D + 8  # bytes of a block of K and V with its scales


def _blocks_done(c, tokens):
    return sum((n + t) // BLOCK - n // BLOCK for n, t in zip(_lengths(c), tokens))


def work(c):
    kind, B = c["kind"], c["B"]
    if kind == "rope":
        n = B * c["T"] * (c["H"] + c["Hkv"]) * D
        return {"bytes": 2 * n * (2 if c["dtype"] == "bf16" else 4), "flops": 3 * n}
    if kind == "append":
        H, rows = c["H"], B * c["T"]
        if c["hold"]:
            return {"bytes": 4 * rows * H * ROW, "flops": 0}
        done = _blocks_done(c, [c["T"]] * B)
        kept = sum(min(c["T"], (n + c["T"]) % BLOCK) for n in _lengths(c))  # rows that stay behind the blocks
        held = sum(n % BLOCK for n in _lengths(c) if n % BLOCK + c["T"] >= BLOCK)
        nbytes = H * (2 * ROW * (rows + kept + held) + done * PAIR)
        if c["q8"] == "int8":
            nbytes += _read_bytes(c, [n + c["T"] - _start(c) for n in _lengths(c)], 2)
        return {"bytes": nbytes, "flops": 4 * rows * H * D}
    if kind == "read":
        return {"bytes": _read_bytes(c, _lengths(c), 2 if c["out"] == "bf16" else 4), "flops": 2 * sum(_lengths(c)) * c["H"] * D}
    if kind == "attn":
        lens, N = _lengths(c), c["N"]
        near = sum(n % BLOCK for n in lens) + (0 if c["cross"] else N * B)
        nbytes = c["Hkv"] * (sum(n // BLOCK for n in lens) * PAIR + near * 2 * ROW) + 2 * B * N * c["H"] * ROW
        return {"bytes": nbytes, "flops": 4 * D * c["H"] * N * (sum(lens) + (0 if c["cross"] else N * B))}
    done = _blocks_done(c, _accepted(c))
    L, H = c["layers"], c["H"]
    moved = sum(a > 0 for a in _accepted(c))  # about one row of a path lies elsewhere
    nbytes = L * H * (done * (PAIR + 2 * BLOCK * ROW) + (0 if c["chain"] else 2 * moved * 2 * ROW)) + 8 * B * (c["N"] + 4)
    if c["q8"] == "int8":
        nbytes += L * _read_bytes(c, [n + a - _start(c) for n, a in zip(_lengths(c), _accepted(c))], 2)
    return {"bytes": nbytes, "flops": 0}


def _read_bytes(c, tokens, size):
    """Expanding the last tokens of each sequence, at `size` bytes an element."""
    whole = sum(t // BLOCK for t in tokens)
    left = sum(t % BLOCK for t in tokens)
    return c["H"] * (whole * PAIR + left * 2 * ROW + sum(tokens) * 2 * D * size)


# ---------------------------------------------------------------------------
# Float64 results
# ---------------------------------------------------------------------------

def _round_e4m3(y):
    """The e4m3 value nearest to y (|y| <= 448), ties to even."""
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def _token_dims(part):
    """[4096] token and dim of every byte of a block's K or V part."""
    at = torch.arange(BLOCK * D)
    if part == 0:
        kt, h, g, c, b = at // 2048, at // 1024 % 2, at // 256 % 4, at // 16 % 16, at % 16
        return 16 * kt + c, 64 * h + 16 * g + b
    u, g, c, t, j, i = at // 1024, at // 256 % 4, at // 16 % 16, at // 8 % 2, at // 4 % 2, at % 4
    return 16 * j + 4 * g + i, 8 * c + 2 * u + t


def _exact_unpack(blocks, scales):
    """One sequence's [H, blocks, 8192] -> K, V [H, tokens, 128] float64."""
    out = []
    for m in range(2):
        tok, dim = (x.to(DEV) for x in _token_dims(m))
        y = blocks[..., m * BLOCK * D:(m + 1) * BLOCK * D].to(F64) - (128 if blocks.dtype == torch.uint8 else 0)
        x = torch.empty((*y.shape[:-1], BLOCK, D), dtype=F64, device=DEV)
        x[..., tok, dim] = y
        out.append((x * scales[..., m, None, None].to(F64)).flatten(1, 2))
    return out


def _exact_depth(parents):
    out = []
    for p in parents:
        out.append(0 if p < 0 else out[p] + 1)
    return out


def _exact_rope(s):
    c = s["c"]
    if s["positions"] is not None:
        pos = s["positions"].to(F64)
    else:
        lens = s["lens"].tolist()
        steps = [_exact_depth(p) for p in s["parents"].tolist()] if s["parents"] is not None else [range(c["T"])] * c["B"]
        pos = torch.tensor([[n + t for t in st] for n, st in zip(lens, steps)], dtype=F64, device=DEV)
    turn = torch.polar(torch.full_like(pos, s["m"])[..., None].expand(*pos.shape, c["rot"] // 2),
                       pos[..., None] * s["freqs"])
    if c["back"]:
        turn = turn.conj()
    out = {}
    for name in ("q", "k"):
        x = s[name].to(F64)
        body = x[..., :c["rot"]]
        pairs = body.unflatten(-1, (-1, 2)) if c["inter"] else body.unflatten(-1, (2, -1)).transpose(-1, -2)
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, :, None])
        y = y if c["inter"] else y.transpose(-1, -2)
        out[name] = torch.cat([y.flatten(-2), x[..., c["rot"]:]], dim=-1)
    return out


def _exact_row(cache, b, m, j):
    return cache[2][b, :, m, j % TAIL].to(F64)


def _exact_store(c, cache, todo):
    """Sequence by sequence: todo[b] = (first position, rows, end): rows[m]
    [H, n, 128] float64 of positions first .. end - 1, the first of them at a
    block's start; what is left behind the blocks stays in the tail at and
    past `keep`."""
    blocks, scales, tail = cache
    values = blocks.to(F64) if c["q8"] == "e4m3" else None
    new_scales, new_tail = scales.to(F64), tail.to(F64)
    whole = [None] * len(todo)
    for b, (first, rows, end, keep) in enumerate(todo):
        n = end // BLOCK - first // BLOCK
        whole[b] = []
        for i in range(n):
            for m in range(2):
                tok, dim = (x.to(DEV) for x in _token_dims(m))
                x = rows[m][:, i * BLOCK:(i + 1) * BLOCK]
                at = first // BLOCK + i
                scale = (x.abs().amax(dim=(1, 2)) / MOST[c["q8"]]).to(F32).to(F64)
                scale = torch.where(scale < TINY, 0.0, scale)
                # by definition the quotient is a float32: where it is a tie, the
                # scale's own rounding has no say
                y = torch.where(scale[:, None, None] > 0, x / scale[:, None, None], 0.0).to(F32).to(F64)
                y = y.clamp(-MOST[c["q8"]], MOST[c["q8"]])
                y = _round_e4m3(y) if c["q8"] == "e4m3" else torch.round(y)
                new_scales[b, :, at, m] = scale
                if values is not None:
                    values[b, :, at, m * BLOCK * D:(m + 1) * BLOCK * D] = y[:, tok, dim]
                whole[b].append((m, at, y * scale[:, None, None]))
        for j in range(max(keep, end // BLOCK * BLOCK), end):
            for m in range(2):
                new_tail[b, :, m, j % TAIL] = rows[m][:, j - first]
    return values, new_scales, new_tail, whole


def _exact_stored(s, cache, todo):
    c = s["c"]
    values, scales, tail, whole = _exact_store(c, cache, todo)
    if c["q8"] == "e4m3":
        return dict(values=values, scales=scales, tail=tail)
    start = _start(c)
    out = [torch.zeros_like(s["k_out"], dtype=F64), torch.zeros_like(s["v_out"], dtype=F64)]
    for b, (first, rows, end, keep) in enumerate(todo):
        done = end // BLOCK * BLOCK
        old = _exact_unpack(cache[0][b, :, start // BLOCK:], cache[1][b, :, start // BLOCK:])
        for m in range(2):
            if first > start:
                out[m][b, :, :first - start] = old[m][:, :first - start]
            if end > done:
                out[m][b, :, done - start:end - start] = rows[m][:, done - first:end - first]
        for m, at, y in whole[b]:
            out[m][b, :, at * BLOCK - start:(at + 1) * BLOCK - start] = y
    return dict(k=out[0], v=out[1], scales=scales, tail=tail)


def _exact_append(s):
    c, cache, T = s["c"], s["cache"], s["c"]["T"]
    if c["hold"]:
        tail = cache[2].to(F64)
        for b, L in enumerate(s["lens"].tolist()):
            for t in range(T):
                tail[b, :, 0, (L + t) % TAIL], tail[b, :, 1, (L + t) % TAIL] = s["k"][b, t].to(F64), s["v"][b, t].to(F64)
        return dict(tail=tail)
    todo = []
    for b, L in enumerate(s["lens"].tolist()):
        first = L // BLOCK * BLOCK
        rows = []
        for m, x in ((0, s["k"]), (1, s["v"])):
            held = [_exact_row(cache, b, m, j) for j in range(first, L)]
            new = x[b].to(F64).transpose(0, 1)
            rows.append(torch.cat([torch.stack(held, dim=1), new], dim=1) if held else new)
        todo.append((first, rows, L + T, L))
    return _exact_stored(s, cache, todo)


def _exact_read(s):
    c = s["c"]
    k, v = torch.zeros_like(s["k_out"], dtype=F64), torch.zeros_like(s["v_out"], dtype=F64)
    for b, L in enumerate(s["lens"].tolist()):
        whole = L // BLOCK * BLOCK
        held = _exact_unpack(s["cache"][0][b], s["cache"][1][b])
        for m, out in ((0, k), (1, v)):
            out[b, :, :whole] = held[m][:, :whole]
            for j in range(whole, L):
                out[b, :, j] = _exact_row(s["cache"], b, m, j)
    return dict(k=k, v=v)


def _exact_attn(s):
    c = s["c"]
    B, N, H, Hkv = c["B"], c["N"], c["H"], c["Hkv"]
    G = H // Hkv
    out = torch.zeros((B, N, H, D), dtype=F64, device=DEV)
    for b, L in enumerate(s["lens"].tolist()):
        whole, end = L // BLOCK * BLOCK, L if c["cross"] else L + N
        if end == 0:
            continue
        mask = torch.ones((N, end), dtype=torch.bool)
        if not c["cross"]:
            mask[:, L:] = False
            for n, p in enumerate(s["parents"][b].tolist()):
                if p >= 0:
                    mask[n] = mask[p]
                mask[n, L + n] = True
        mask = mask.to(DEV)
        ring = torch.arange(whole, end, device=DEV) % TAIL
        for h in range(Hkv):
            k, v = _exact_unpack(s["cache"][0][b, h:h + 1, :whole // BLOCK], s["cache"][1][b, h:h + 1, :whole // BLOCK])
            k = torch.cat([k[0], s["cache"][2][b, h, 0, ring].to(F64)])
            v = torch.cat([v[0], s["cache"][2][b, h, 1, ring].to(F64)])
            q = s["q"][b, :, h * G:(h + 1) * G].to(F64).reshape(N * G, D)
            x = torch.mm(q, k.t()) / math.sqrt(D)
            x = x.masked_fill(~mask.repeat_interleave(G, dim=0), -math.inf)
            out[b, :, h * G:(h + 1) * G] = torch.mm(torch.softmax(x, dim=-1), v).view(N, G, D)
    return out


def _exact_commit(s):
    c = s["c"]
    lens, accept = s["lens"].tolist(), s["accept"].tolist()
    paths = None if s["path"] is None else s["path"].tolist()
    todo = []
    for row in range(c["layers"] * c["B"]):
        b = row % c["B"]
        L, a = lens[b], accept[b]
        first = L // BLOCK * BLOCK
        at = list(range(first, L)) + [L + (d if paths is None else paths[b][d]) for d in range(a)]
        at = torch.tensor(at, dtype=torch.long, device=DEV) % TAIL
        rows = [s["all"][2][row, :, m, at].to(F64) for m in range(2)]
        todo.append((first, rows, L + a, L))
    stored = _exact_stored(s, s["all"], todo)
    return dict(stored, lens=None)


_EXACT = dict(rope=_exact_rope, append=_exact_append, read=_exact_read, attn=_exact_attn, commit=_exact_commit)


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))
