"""The calls on an 8-bit cache together, as a decoding loop makes them: against
the float64 oracle step by step, in captured graphs, on several streams, and
through either path of the binding."""

import numpy as np
import pytest
import torch

import paper_2402_02082_amd as glide
from oracle import rope as OR
from paper_2402_02082_amd import _lib
from tests.gpu_common import cpu_normal, require_gpu, say
from tests.test_gpu_q8_attn import check, random_tree
from tests.test_gpu_q8_cache import KINDS, check_cache, f64, ints, junk_cache, rows

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("N", [1, 12])
def test_decoding_loop(kind, N):
    """Prompt, then verification steps: rotary positions of the tree's rows, tree
    rows held, attention, greedy acceptance, commit -- in two layers.  The
    caches, lengths and outputs follow the oracle at every step."""
    require_gpu()
    B, H, Hk, V, layers, prompt = 2, 4, 2, 50, 2, 57
    rng = np.random.default_rng(N)
    freqs, m = glide.rope_frequencies(128)
    caches = [junk_cache(B, Hk, 256, kind) for _ in range(layers)]
    lens, lens_out = ints([prompt, prompt - 30]), ints([0, 0])
    known = [[[], []] for _ in range(layers)]  # [layer][K or V][b]: rows so far
    for i, c in enumerate(caches):
        k, v = rows((B, prompt, Hk, 128), 60 + i), rows((B, prompt, Hk, 128), 70 + i)
        glide.glide_rope(k, None, freqs, k, None)
        glide.glide_q8_append(k, v, c, ints([0, 0]), lens)
        n = lens.tolist()
        known[i] = [[k[b, :n[b]] for b in range(B)], [v[b, :n[b]] for b in range(B)]]
    for step in range(12):
        L = lens.tolist()
        say("step", kind, N, step, L)
        par = np.array([random_tree(N, rng) for _ in range(B)], dtype=np.int32)
        parents = torch.from_numpy(par).cuda()
        tree = []
        for i, c in enumerate(caches):
            seed = 1000 * step + 10 * i
            q, k, v = (rows((B, N, h, 128), seed + j, spread=False) for j, h in enumerate((H, Hk, Hk)))
            pos = np.array([OR.tree_positions(L[b], par[b]) for b in range(B)])
            want = OR.rope(f64(k), pos, f64(freqs))
            glide.glide_rope(q, k, freqs, q, k, seq_lens=lens, tree_parents=parents)
            assert np.all(np.abs(f64(k) - want) <= 2.0 ** -8 * np.abs(want) + 2e-5)
            glide.glide_q8_append(k, v, c, lens, hold=True)
            out = torch.full_like(q, float("nan"))
            glide.glide_q8_tree_attn(q, c, lens, parents, out)
            top = max(L)
            pad = [torch.stack([torch.cat([x, x.new_zeros((top - len(x), Hk, 128))]) for x in known[i][j]])
                   for j in range(2)]
            check(out, q, pad[0], pad[1], L, kind, k, v, par)
            tree.append((k, v))
        # a target that accepts a random root path, the whole of it
        logits = cpu_normal((B, N + 1, V), step, F32).cuda()
        tokens = torch.from_numpy(rng.integers(0, V, (B, N)).astype(np.int32)).cuda()
        for b in range(B):
            n = int(rng.integers(-1, N))
            while n >= 0:
                logits[b, par[b, n] + 1, tokens[b, n]] = 30.0
                n = int(par[b, n])
        acc, path, argmax = ints([0, 0]), torch.empty((B, N), dtype=I32, device="cuda"), torch.empty((B, N + 1), dtype=I32,
                                                                                                  device="cuda")
        glide.glide_verify_commit(logits, tokens, parents, [], [], lens, lens_out, argmax, acc, path=path)
        after = lens_out.tolist()
        lens_out.fill_(-1)
        glide.glide_q8_commit(caches, lens, acc, path, lens_out)
        assert lens_out.tolist() == after
        for i in range(layers):
            for b in range(B):
                nodes = path[b, :acc[b]].tolist()
                for j in range(2):
                    known[i][j][b] = torch.cat([known[i][j][b], tree[i][j][b, nodes]])
            check_cache(caches[i], known[i][0], known[i][1], after, kind)
        lens, lens_out = lens_out, lens
    assert max(lens.tolist()) > (prompt + 7 if N > 1 else prompt)


def test_single_token_decoding():
    """One token a step: append, then attention over the prefix (cross mode)."""
    require_gpu()
    B, H, Hk = 3, 8, 2
    cache = junk_cache(B, Hk, 160, "int8")
    k, v = rows((B, 100, Hk, 128), 80), rows((B, 100, Hk, 128), 81)
    first = [0, 20, 33]
    glide.glide_q8_append(k, v, cache, ints([0] * B), ints(first))
    for t in range(60):
        lens = [n + t for n in first]
        kt, vt = (torch.stack([x[b, n] for b, n in enumerate(lens)])[:, None].contiguous() for x in (k, v))
        glide.glide_q8_append(kt, vt, cache, ints(lens))
        lens = [n + 1 for n in lens]
        if t % 7 == 0 or 30 <= t <= 33:
            q = cpu_normal((B, 1, H, 128), t, BF).cuda()
            out = torch.empty_like(q)
            glide.glide_q8_tree_attn(q, cache, ints(lens), None, out)
            check(out, q, k, v, lens, "int8")


def _step_state(seed, L=700, N=9, B=1):
    H, Hk = 8, 4
    s = dict(lens=ints([L + 7 * b for b in range(B)]), out=ints([0] * B), acc=ints([min(4, N)] * B),
             par=ints([random_tree(N, np.random.default_rng(b)) for b in range(B)]))
    s["path"] = ints([[0, 2, 3, 6] + [-1] * (N - 4)] * B)
    s["cache"] = junk_cache(B, Hk, L + 128, "int8")
    k, v = rows((B, L + 7 * B, Hk, 128), seed), rows((B, L + 7 * B, Hk, 128), seed + 1)
    glide.glide_q8_append(k, v, s["cache"], ints([0] * B), s["lens"])
    s["q"], s["k"], s["v"] = (rows((B, N, h, 128), seed + j, spread=False) for j, h in ((2, H), (3, Hk), (4, Hk)))
    s["qr"], s["kr"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    s["freqs"], _ = glide.rope_frequencies(128)
    s["o"] = torch.zeros_like(s["q"])
    s["read"] = [torch.zeros((B, Hk, L + 64, 128), dtype=BF, device="cuda") for _ in range(2)]
    return s


def _step(s, **kw):
    glide.glide_rope(s["q"], s["k"], s["freqs"], s["qr"], s["kr"], seq_lens=s["lens"], tree_parents=s["par"], **kw)
    glide.glide_q8_append(s["kr"], s["v"], s["cache"], s["lens"], hold=True, **kw)
    glide.glide_q8_tree_attn(s["qr"], s["cache"], s["lens"], s["par"], s["o"], **kw)
    glide.glide_q8_commit([s["cache"]], s["lens"], s["acc"], s["path"], s["out"], **kw)
    glide.glide_q8_read(s["cache"], s["out"], *s["read"], **kw)


def _results(s):
    c = s["cache"]
    end = int(s["out"].max())
    return [s["o"].clone(), s["out"].clone(), s["read"][0].clone(), s["read"][1].clone(),
            c.scales[:, :, :end // 32].clone()]


def _same(a, b):
    return all(torch.equal(x.view(torch.uint8) if x.is_floating_point() else x,
                           y.view(torch.uint8) if y.is_floating_point() else y) for x, y in zip(a, b))


def test_captured_and_replayed():
    """All calls of a step in one graph, replayed with eager work and waits
    between: every replay as the eager step."""
    require_gpu()
    for B in (1, 3):
        s = _step_state(90, B=B)
        _step(s)
        torch.cuda.synchronize()
        want = _results(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _step(s)
        for _ in range(4):
            for x in (s["o"], s["out"], *s["read"]):
                x.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert _same(_results(s), want)
            _step(s)  # the eager step between uses the stream's own workspace
            torch.cuda.synchronize()
            assert _same(_results(s), want)


def test_two_graphs_and_eager_calls_at_once():
    """Two graphs captured one after the other and eager calls, on three streams
    at once: no workspace is shared."""
    require_gpu()
    states = [_step_state(100 + 10 * i, L=3000 + 500 * i) for i in range(3)]
    want = []
    for s in states:
        _step(s)
        torch.cuda.synchronize()
        want.append(_results(s))
    graphs = []
    for s in states[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _step(s)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        with torch.cuda.stream(streams[2]):
            _step(states[2])
    torch.cuda.synchronize()
    for s, w in zip(states, want):
        assert _same(_results(s), w)


def test_workspaces_of_the_two_attentions_are_apart():
    """A captured glide_tree_attn goes on using the workspace that its stream's
    eager calls left: neither a larger glide_q8_tree_attn nor what is allocated
    after it takes that memory's place, and every replay stays the same."""
    require_gpu()
    dev = torch.device("cuda")
    side = torch.cuda.Stream()
    B, N, H, L = 1, 5, 4, 2000
    q = cpu_normal((B, N, H, 128), 90, BF).cuda()
    k, v = cpu_normal((B, H, L + N, 128), 91, BF).cuda(), cpu_normal((B, H, L + N, 128), 92, BF).cuda()
    lens, out = ints([L]), torch.empty_like(q)
    cache, many = junk_cache(1, 32, 4096, "e4m3"), cpu_normal((1, 64, 32, 128), 93, BF).cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        glide.glide_tree_attn(q, k, v, lens, None, out)
        want = out.clone()
        kept = glide.attn_workspace(B, N, H, L + N, 0, dev)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            glide.glide_tree_attn(q, k, v, lens, None, out)
        glide.glide_q8_tree_attn(many, cache, ints([0]), None, torch.empty_like(many))
        own = glide.q8_attn_workspace(1, 64, 32, 32, 4096, 0, dev)
        assert own.numel() > kept.numel() and glide.attn_workspace(B, N, H, L + N, 0, dev) is kept
        junk = [torch.full((kept.numel(),), 0xFF, dtype=torch.uint8, device=dev) for _ in range(4)]
        for i in range(3):
            out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i
    assert len(junk) == 4


def test_an_explicit_stream():
    require_gpu()
    s = _step_state(130, L=2500)
    _step(s)
    torch.cuda.synchronize()
    want = _results(s)
    for x in (s["o"], s["out"], *s["read"]):
        x.zero_()
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    _step(s, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda.synchronize()
    assert _same(_results(s), want)


def test_native_equals_python_path():
    """The native checks take a plain call, and the Python checks give the same."""
    require_gpu()
    s = _step_state(140, L=2000)
    _step(s)  # workspaces exist from here on
    native = _lib._bind()
    assert native.rope(s["q"], s["k"], s["freqs"], s["qr"], s["kr"], None, s["lens"], s["par"], False, 1.0, False,
                       None) == 0
    assert native.q8_append(s["kr"], s["v"], s["cache"], s["lens"], None, True, None) == 0
    assert native.q8_tree_attn(s["qr"], s["cache"], s["lens"], s["par"], s["o"], 0.0, 0, None, None) == 0
    assert native.q8_commit([s["cache"]], s["lens"], s["acc"], s["path"], s["out"], 9, None) == 0
    assert native.q8_read(s["cache"], s["out"], *s["read"], 0, None) == 0
    torch.cuda.synchronize()
    want = _results(s)
    _step(s, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert _same(_results(s), want)
    # arguments that the Python checks refuse are declined
    q, k, c, lens = s["q"], s["k"], s["cache"], s["lens"]
    for args in ((q.float(), k, s["freqs"], q, k), (q, k, s["freqs"].float(), q, k), (q, k, s["freqs"], q, None),
                 (q, k, s["freqs"], q.expand_as(q)[..., :64], k)):
        assert native.rope(*args, None, None, None, False, 1.0, False, None) is None
    assert native.q8_append(k.float(), k, c, lens, None, True, None) is None
    assert native.q8_append(k, k[:, :2], c, lens, None, True, None) is None
    assert native.q8_append(k, k, list(c), lens, None, True, None) is None
    assert native.q8_append(k, k, c, lens.long(), None, True, None) is None
    assert native.q8_tree_attn(q, c, lens, s["par"][:, :2], q, 0.0, 0, None, None) is None
    assert native.q8_tree_attn(q.float(), c, lens, None, q, 0.0, 0, None, None) is None
    assert native.q8_commit((c,), lens, s["acc"], None, s["out"], 9, None) is None
    assert native.q8_commit([c], lens, s["acc"], s["path"], s["out"], 8, None) is None
    assert native.q8_read(c, lens, s["read"][0], s["read"][1].float(), 0, None) is None
