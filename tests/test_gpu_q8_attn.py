"""Attention over the 8-bit cache on the GPU against the float64 oracle.

Tolerance, per element, with A = sum_j p_j |v_j| the row's average magnitude
(p the softmax): the output is rounded once to bfloat16 (2^-8 of it); a
probability's product with scales is rounded to fp16 (2^-11) where it is not
below 2^-21 of the row's largest, and lies within 2^-32 of that one anyway
(keys * 2^-32 * max |v|); sums of n keys in float32 are off by n 2^-24; a score
is a float32 sum of 128 products of up to |q| |k| / sqrt(D) in all, scaled
twice: off by 131 * 2^-24 of that, and a probability by as much relatively, the
normaliser too.  Below 2^-126 the steps of a bfloat16 are 2^-133 whatever its
size, so that the output's rounding is off by up to 2^-134 there."""

import numpy as np
import pytest
import torch

import paper_2402_02082_amd as glide
from oracle import attention as OA
from oracle import q8 as OQ
from tests.gpu_common import cpu_normal, require_gpu, say
from tests.test_gpu_q8_cache import KINDS, f64, ints, junk_cache, rows

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def random_tree(N, rng, chain=False):
    return [n - 1 if chain else (int(rng.integers(-1, n)) if n else -1) for n in range(N)]


def fill(B, H, lens, kind, seed, cap=None, k_scale=1.0, v_scale=1.0):
    """A cache with lens tokens of seeded rows behind junk, and the rows."""
    n = max(max(lens), 1)
    k, v = (rows((B, n, H, 128), seed) * k_scale).to(BF), (rows((B, n, H, 128), seed + 1) * v_scale).to(BF)
    cache = junk_cache(B, H, cap or n + 1, kind)
    glide.glide_q8_append(k, v, cache, ints([0] * B), ints(lens))
    return cache, k, v


def check(got, q, k, v, lens, kind, tk=None, tv=None, par=None, scale=None, nodes=None, pairs=None):
    got, q = f64(got), f64(q)
    B, N, H, D = q.shape
    Hk = k.shape[2]
    G = H // Hk
    sc = 1 / np.sqrt(D) if scale is None else scale
    for b in range(B):
        for j in range(Hk):
            if pairs is not None and (b, j) not in pairs:
                continue
            ks, vs = (OQ.stored(f64(x[b, :lens[b], j]), kind) for x in (k, v))
            for n in range(N) if nodes is None else nodes:
                kk, vv = ks, vs
                if par is not None:
                    own = OA.ancestor_or_self(par[b], n)
                    kk, vv = np.concatenate([ks, f64(tk[b, own, j])]), np.concatenate([vs, f64(tv[b, own, j])])
                h = slice(j * G, (j + 1) * G)
                want = OA.attention_rows(q[b, n, h], kk, vv, sc)
                if not len(kk):
                    assert not got[b, n, h].any()
                    continue
                A = OA.attention_rows(q[b, n, h], kk, np.abs(vv), sc)
                score = np.linalg.norm(q[b, n, h], axis=1).max() * np.linalg.norm(kk, axis=1).max() * sc
                rel = 2.0 ** -11 + 2 * len(kk) * 2.0 ** -24 + 2 * 131 * 2.0 ** -24 * score
                tol = 2.0 ** -8 * np.abs(want) + rel * A + len(kk) * 2.0 ** -32 * np.abs(vv).max() + 2.0 ** -134
                err = np.abs(got[b, n, h] - want)
                assert np.all(err <= tol), (b, j, n, float((err / tol).max()))


def run(q, cache, lens, par=None, **kw):
    out = torch.full_like(q, float("nan"))
    glide.glide_q8_tree_attn(q, cache, ints(lens), None if par is None else ints(par), out, **kw)
    torch.cuda.synchronize()
    return out


LENS = [0, 1, 31, 32, 33, 95, 128, 417]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,H,Hk", [(1, 1, 1), (1, 8, 1), (5, 2, 2), (5, 12, 4), (16, 2, 2), (17, 2, 2), (33, 2, 1),
                                    (64, 2, 2), (64, 8, 1), (3, 10, 2)])
def test_tree(kind, N, H, Hk):
    """Ragged lengths around block ends, every row count of the query tiles, one
    and several heads to a cached head; nothing that holds no token is read."""
    require_gpu()
    say("tree", kind, N, H, Hk)
    rng = np.random.default_rng(N)
    B = len(LENS)
    cache, k, v = fill(B, Hk, LENS, kind, 3)
    tk, tv = rows((B, N, Hk, 128), 5), rows((B, N, Hk, 128), 6)
    glide.glide_q8_append(tk, tv, cache, ints(LENS), hold=True)
    par = [random_tree(N, rng, chain=b == 1) for b in range(B)]
    q = cpu_normal((B, N, H, 128), 7, BF).cuda()
    check(run(q, cache, LENS, par), q, k, v, LENS, kind, tk, tv, par)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N,H,Hk", [(1, 4, 4), (5, 8, 2), (32, 2, 2), (64, 3, 1)])
def test_cross(kind, N, H, Hk):
    require_gpu()
    say("cross", kind, N, H, Hk)
    B = len(LENS)
    cache, k, v = fill(B, Hk, LENS, kind, 8)
    q = cpu_normal((B, N, H, 128), 9, BF).cuda()
    out = run(q, cache, LENS)
    check(out, q, k, v, LENS, kind)
    assert not out[0].any()  # no key: zeros


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
def test_splits(kind, splits):
    """Long caches, forced split counts; two runs give the same bits."""
    require_gpu()
    lens = [4096, 1700, 40, 2500]
    cache, k, v = fill(4, 2, lens, kind, 10)
    tk, tv = rows((4, 6, 2, 128), 11), rows((4, 6, 2, 128), 12)
    glide.glide_q8_append(tk, tv, cache, ints(lens), hold=True)
    par = [random_tree(6, np.random.default_rng(b)) for b in range(4)]
    q = cpu_normal((4, 6, 4, 128), 13, BF).cuda()
    for scale in (0.0, 0.2):
        out = run(q, cache, lens, par, max_splits=splits, scale=scale)
        check(out, q, k, v, lens, kind, tk, tv, par, scale or None, nodes=[0, 3, 5])
        again = run(q, cache, lens, par, max_splits=splits, scale=scale)
        assert torch.equal(out, again)


@pytest.mark.parametrize("kind", KINDS)
def test_one_sequence_and_many_rows(kind):
    require_gpu()
    lens = [1111]
    cache, k, v = fill(1, 3, lens, kind, 14)
    for N, H in ((1, 3), (5, 3), (16, 3), (40, 6), (64, 24)):
        say("one sequence", kind, N, H)
        tk, tv = rows((1, N, 3, 128), 15), rows((1, N, 3, 128), 16)
        glide.glide_q8_append(tk, tv, cache, ints(lens), hold=True)
        par = [random_tree(N, np.random.default_rng(N))]
        q = cpu_normal((1, N, H, 128), 17, BF).cuda()
        check(run(q, cache, lens, par), q, k, v, lens, kind, tk, tv, par, nodes=sorted({0, N // 2, N - 1}))


@pytest.mark.parametrize("B,H,Hk,N,top", [
    (2, 4, 2, 5, 3000), (3, 16, 4, 30, 1500), (5, 64, 8, 9, 2100), (4, 40, 40, 7, 3500), (9, 20, 20, 33, 1900),
    (6, 32, 32, 1, 2600), (3, 80, 20, 25, 1800), (70, 8, 4, 3, 500), (70, 6, 6, 2, 300), (130, 1, 1, 6, 1800)])
def test_plans(B, H, Hk, N, top):
    """Few pairs, as many as half of the CUs, more, as many as all and more; up to
    64 sequences and beyond; several groups of query rows: unequal lengths, some
    of one token; some pairs against the oracle, all against one run a pair (each
    is within a rounding to bfloat16, 2^-8 of it, and 2^-10 of the largest value
    from the exact result), and two calls alike."""
    require_gpu()
    say("plans", B, H, Hk, N, top)
    rng = np.random.default_rng(B + N)
    lens = [int(x) for x in rng.integers(1, top, B)]
    lens[0], lens[-1] = top, 1
    cache, k, v = fill(B, Hk, lens, "int8", 50)
    tk, tv = rows((B, N, Hk, 128), 51), rows((B, N, Hk, 128), 52)
    glide.glide_q8_append(tk, tv, cache, ints(lens), hold=True)
    q = cpu_normal((B, N, H, 128), 53, BF).cuda()
    for par in (None, [random_tree(N, rng) for _ in range(B)]):
        out = run(q, cache, lens, par)
        pairs = {(0, 0), (B - 1, Hk - 1), (B // 2, Hk // 2)}
        check(out, q, k, v, lens, "int8", *((tk, tv, par) if par else ()), nodes=sorted({0, N - 1}), pairs=pairs)
        one = run(q, cache, lens, par, max_splits=1)
        size = float(v.abs().max().float())
        err = (out.float() - one.float()).abs()
        assert bool((err <= 2.0 ** -7 * one.float().abs() + 2.0 ** -9 * size).all())
        assert torch.equal(run(q, cache, lens, par), out)


@pytest.mark.parametrize("B,H,Hk,N", [(1, 60, 1, 64), (2, 88, 1, 64), (11, 24, 1, 64), (5, 12, 2, 50)])
def test_few_pairs_of_many_query_rows(B, H, Hk, N):
    """One or a few cached heads for all query heads: the groups of runs that do not
    fill the eight XCDs' turns are spread over all of them."""
    require_gpu()
    say("groups", B, H, Hk, N)
    rng = np.random.default_rng(H)
    lens = [int(x) for x in rng.integers(1, 500, B)]
    cache, k, v = fill(B, Hk, lens, "e4m3", 56)
    tk, tv = rows((B, N, Hk, 128), 57), rows((B, N, Hk, 128), 58)
    glide.glide_q8_append(tk, tv, cache, ints(lens), hold=True)
    q, par = cpu_normal((B, N, H, 128), 59, BF).cuda(), [random_tree(N, rng) for _ in range(B)]
    for splits in (0, 1, 3):
        out = run(q, cache, lens, par, max_splits=splits)
        check(out, q, k, v, lens, "e4m3", tk, tv, par, nodes=[0, N // 2, N - 1])


@pytest.mark.parametrize("pairs", [4, 140])
@pytest.mark.parametrize("N", [3, 7, 10, 13])
def test_rows_that_do_not_fill_the_waves(pairs, N):
    """The runs' states joined by four and by eight waves that share rows, of which
    some have a turn without rows (9 to 12 rows for eight waves)."""
    require_gpu()
    say("joined rows", pairs, N)
    lens = [330, 100]
    cache, k, v = fill(2, pairs // 2, lens, "e4m3", 54)
    q = cpu_normal((2, N, pairs // 2, 128), 55, BF).cuda()
    for splits in (3, 20):
        check(run(q, cache, lens, None, max_splits=splits), q, k, v, lens, "e4m3", pairs={(0, 0), (1, pairs // 2 - 1)})


@pytest.mark.parametrize("kind", KINDS)
def test_peaked_scores(kind):
    """Queries times 24: the reference maximum is passed by far and often."""
    require_gpu()
    lens = [700, 90]
    cache, k, v = fill(2, 2, lens, kind, 18)
    for N in (3, 20, 50):
        tk, tv = rows((2, N, 2, 128), 19), rows((2, N, 2, 128), 20)
        glide.glide_q8_append(tk, tv, cache, ints(lens), hold=True)
        par = [random_tree(N, np.random.default_rng(N)) for _ in range(2)]
        q = (cpu_normal((2, N, 2, 128), 21, F32) * 24).to(BF).cuda()
        check(run(q, cache, lens, par), q, k, v, lens, kind, tk, tv, par, nodes=[0, N - 1])


@pytest.mark.parametrize("kind", KINDS)
def test_values_of_very_different_size(kind):
    """Blocks whose V scales differ by powers of ten, in every order; a token
    that takes nearly all of the probability and has a value of zero."""
    require_gpu()
    L, H = 32 * 12 + 20, 2
    for order in ("up", "down", "mixed", "sink"):
        say("values", kind, order)
        k, v = rows((1, L, H, 128), 22, spread=False), rows((1, L, H, 128), 23, spread=False)
        power = {"up": np.arange(13) * 4 - 24, "down": 24 - 4 * np.arange(13),
                 "mixed": np.array([0, 30, -30, 5, -5, 20, -36, 1, 0, 33, -20, 2, 0]), "sink": np.zeros(13)}[order]
        for i in range(13):
            v[:, 32 * i:32 * i + 32] *= 10.0 ** float(power[i])
        q = cpu_normal((1, 4, H, 128), 24, BF).cuda()
        if order == "sink":
            v[:, 3] = 0
            k[:, 3] = q[:, 0]  # a score of about 11 for the first query
        cache = junk_cache(1, H, L + 1, kind)
        glide.glide_q8_append(k, v, cache, ints([0]))
        check(run(q, cache, [L]), q, k, v, [L], kind)
        tk, tv = rows((1, 4, H, 128), 25), (rows((1, 4, H, 128), 26) * 1e-20).to(BF)
        glide.glide_q8_append(tk, tv, cache, ints([L]), hold=True)
        par = [[-1, 0, 1, 0]]
        check(run(q, cache, [L], par), q, k, v, [L], kind, tk, tv, par)


@pytest.mark.parametrize("kind", KINDS)
def test_sizes_at_the_ends_of_bfloat16(kind):
    """Queries, keys and values near the type's largest and smallest numbers."""
    require_gpu()
    for ks, vs, qs in ((1e-30, 1e30, 1e28), (1e30, 1e-30, 1e-31), (1.0, 1e37, 1.0), (1.0, 1e-36, 1.0), (1e-38, 1.0, 1.0),
                       (1.0, 1.0, 1e-38)):
        say("sizes", kind, ks, vs, qs)
        lens = [70, 33]
        k, v = rows((2, 70, 1, 128), 27, spread=False), rows((2, 70, 1, 128), 28, spread=False)
        k, v = (k.double() * ks).to(BF), (v.double().clamp(-3, 3) * vs).to(BF)
        cache = junk_cache(2, 1, 96, kind)
        glide.glide_q8_append(k, v, cache, ints([0, 0]), ints(lens))
        q = (cpu_normal((2, 3, 1, 128), 29, F32).double() * qs).to(BF).cuda()
        check(run(q, cache, lens), q, k, v, lens, kind)


def test_zero_queries_and_zero_blocks():
    require_gpu()
    L = 100
    for kind in KINDS:
        k, v = rows((1, L, 1, 128), 30), rows((1, L, 1, 128), 31)
        v[:, :64] = 0
        k[:, 32:96] = 0
        cache = junk_cache(1, 1, 128, kind)
        glide.glide_q8_append(k, v, cache, ints([0]))
        q = cpu_normal((1, 2, 1, 128), 32, BF).cuda()
        q[:, 1] = 0
        check(run(q, cache, [L]), q, k, v, [L], kind)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_masked_tree_rows_that_are_not_finite(bad):
    """A node whose key and value hold NaN or infinities changes only the nodes
    that see it."""
    require_gpu()
    for N, H, Hk in ((6, 2, 2), (40, 4, 2)):
        lens = [45, 0, 64]
        cache, k, v = fill(3, Hk, lens, "e4m3", 33)
        par = [[-1, 0, 0, 1, 2, -1] + [5] * (N - 6)] * 3
        tk, tv = rows((3, N, Hk, 128), 34), rows((3, N, Hk, 128), 35)
        tk[:, 2, :, 5], tv[:, 2, :, ::3] = bad, bad  # nodes 2 and 4 see it
        glide.glide_q8_append(tk, tv, cache, ints(lens), hold=True)
        q = cpu_normal((3, N, H, 128), 36, BF).cuda()
        out = run(q, cache, lens, par)
        good = [n for n in range(N) if n not in (2, 4)]
        check(out, q, k, v, lens, "e4m3", tk, tv, par, nodes=good)
        # with a key that is finite, an infinite value gives infinities of its sign
        tk[:, 2, :, 5] = 0
        glide.glide_q8_append(tk, tv, cache, ints(lens), hold=True)
        out = run(q, cache, lens, par)
        check(out, q, k, v, lens, "e4m3", tk, tv, par, nodes=good)
        seen = out[:, [2, 4]][..., ::3].float()
        assert torch.isnan(seen).all() if bad != bad else bool((seen == bad).all())
        assert torch.isfinite(out[:, [2, 4]][..., 1::3]).all()


def test_clamped_lengths_bad_parents_and_validation(monkeypatch):
    require_gpu()
    lens = [64, 0]
    cache, k, v = fill(2, 1, lens, "int8", 37, cap=64)
    tk, tv = rows((2, 3, 1, 128), 38), rows((2, 3, 1, 128), 39)
    glide.glide_q8_append(tk, tv, cache, ints([64, 0]), hold=True)
    q = cpu_normal((2, 3, 1, 128), 40, BF).cuda()
    want = run(q, cache, [64, 0], [[-1, -1, 1]] * 2)
    got = run(q, cache, [500, -3], [[-1, 7, 1], [2, -9, 1]])
    assert torch.equal(got, want)
    monkeypatch.setenv("GLIDE_VALIDATE", "1")
    for lens, par in (([500, 0], [[-1, -1, 1]] * 2), ([64, -1], [[-1, -1, 1]] * 2), ([64, 0], [[-1, 7, 1]] * 2)):
        with pytest.raises(glide.GlideError) as e:
            run(q, cache, lens, par)
        assert e.value.status == glide.GLIDE_ERANGE
    assert torch.equal(run(q, cache, [64, 0], [[-1, -1, 1]] * 2), want)


def test_offsets_past_32_bits():
    """8 GiB of blocks: keys of zero make the softmax uniform, so the output is
    the mean of the values, which are zero but in the last blocks."""
    require_gpu()
    H, cap = 8, 1 << 22
    cache = glide.q8_cache(1, H, cap, "int8")
    cache.blocks.fill_(128)
    cache.scales.fill_(1.0)
    L = cap - 40
    L -= L % 32
    v = cpu_normal((1, 96, H, 128), 41, BF).cuda()
    glide.glide_q8_append(torch.zeros_like(v), v, cache, ints([L - 96]))
    q = cpu_normal((1, 2, H, 128), 42, BF).cuda()
    out = f64(run(q, cache, [L]))
    for h in range(H):
        want = OQ.stored(f64(v[0, :, h]), "int8").sum(0) / L
        # 2^22 equal terms summed in float32, split 4 ways a workgroup at least
        assert np.all(np.abs(out[0, :, h] - want) <= 2.0 ** -8 * np.abs(want) + 2e-3 * np.abs(want).max())


def test_workspace_is_shared_with_the_bfloat16_call():
    """One buffer serves both kinds of call in turn: the counters stay zero."""
    require_gpu()
    lens = [2000]
    cache, k, v = fill(1, 4, lens, "e4m3", 43)
    q = cpu_normal((1, 5, 4, 128), 44, BF).cuda()
    kb, vb = (torch.empty((1, 4, 2000, 128), dtype=BF, device="cuda") for _ in range(2))
    glide.glide_q8_read(cache, ints(lens), kb, vb)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    first = None
    for _ in range(3):
        a, b = torch.empty_like(q), torch.empty_like(q)
        glide.glide_tree_attn(q, kb, vb, ints(lens), None, a, workspace=ws)
        glide.glide_q8_tree_attn(q, cache, ints(lens), None, b, workspace=ws)
        torch.cuda.synchronize()
        assert not ws[:glide.ATTN_COUNTER_BYTES].any()
        first = first or (a, b)
        assert torch.equal(a, first[0]) and torch.equal(b, first[1])
    check(first[1], q, k, v, lens, "e4m3")


def test_refusals():
    require_gpu()
    c = glide.q8_cache(2, 2, 2048)
    q, lens = torch.zeros((2, 4, 4, 128), dtype=BF, device="cuda"), ints([0, 0])
    par = torch.zeros((2, 4), dtype=I32, device="cuda")
    ok = dict(q=q, cache=c, seq_lens=lens, tree_parents=par, out=torch.empty_like(q))
    glide.glide_q8_tree_attn(**ok)
    for kw in (dict(q=q.float()), dict(q=q[:1]), dict(q=q[:, :, :3]), dict(q=q[:, :, :1]), dict(q=q[..., :64]),
               dict(q=q.transpose(1, 2)), dict(q=q.cpu()), dict(out=q.float()), dict(out=q[:, :3]),
               dict(seq_lens=lens.long()), dict(seq_lens=lens[:1]), dict(tree_parents=par[:, :3]),
               dict(tree_parents=par.long()), dict(max_splits=65), dict(max_splits=-1), dict(scale=float("nan")),
               dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")),
               dict(workspace=torch.zeros(1 << 26, dtype=torch.uint8)), dict(cache=c[:2]),
               dict(cache=c._replace(blocks=c.blocks.view(torch.int8)))):
        with pytest.raises((ValueError, glide.GlideError)):
            glide.glide_q8_tree_attn(**{**ok, **kw})
    wide = torch.zeros((2, 65, 4, 128), dtype=BF, device="cuda")
    with pytest.raises((ValueError, glide.GlideError)):
        glide.glide_q8_tree_attn(wide, c, lens, None, torch.empty_like(wide))
