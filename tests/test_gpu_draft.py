"""Drafted-token trees on the GPU against the fp64 oracle, through the binding.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value (half a step), to fp32 by 2^-24.

attention: queries and keys are rounded after their rotation, weights before they meet the values, the output once.  A
  score's two rounded factors move it by at most e = (2 * 2^-8 + 2^-16) sum_d |q_d k_d| / sqrt(D), all weights together by a
  factor in [exp(-2e), exp(2e)]; so an output moves by at most 2^-8 |o| + (2^-8 + expm1(2e)) sum_j p_j |v_j|, and fp32 sums
  add less than 1e-5 of the same.
delta rule: q, k, v are exact; the state's product with them is formed from a split of S good to 2^-15 of its largest terms,
  sums over ancestors in at least as many bits: 2^-8 |o| + 2^-13 (G |S_row| |q| + sum_j |R_ij q_i.k_j| |u_j|) holds with room.
  States after a commit are fp32 throughout but for that: relative 2-norm 1e-5 a head.
with the short convolution: inputs rounded to bf16 after it: the relative 2-norm 5e-3 of the library's rounds.
verdicts, positions, moved rows: exact.
"""
import math

import numpy as np
import pytest

from oracle import kvm_oracle as O
from workload import synth as W

pytestmark = pytest.mark.gpu

THETA = 1.0e4


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_18935_gb300 import kvm
    kvm.load_library()


def _bf(bits):
    from harness import to_torch_bf16
    return to_torch_bf16(bits).cuda()


def _f64(t):
    from harness import torch_bf16_to_f64
    return torch_bf16_to_f64(t)


def tree(kind, n, seed=0):
    r = np.random.default_rng([seed, n])
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "star":
        return [-1 if i == 0 else 0 for i in range(n)]
    if kind == "roots":
        return [-1] * n
    if kind == "comb":                                          # a chain whose odd nodes are leaves
        return [-1 if i == 0 else (i - 1 if i % 2 == 1 else i - 2) for i in range(n)]
    if kind == "forest":
        return [-1 if i < 1 or r.random() < 0.15 else int(r.integers(0, i)) for i in range(n)]
    return [-1 if i == 0 else int(r.integers(max(0, i - 6), i)) for i in range(n)]      # "tree"


def cu_of(trees):
    return np.concatenate([[0], np.cumsum([len(t) for t in trees])]).astype(np.int32)


def packed(trees):
    return np.array(sum(trees, []), np.int32)


# ---------------------------------------------------------------------------- attention
class Attn:
    """One attention layer: a context with random caches and the oracle's copies of them."""

    def __init__(self, hq, hkv, d, rot, lives, seed, extra=64, cursor=0):
        from paper_2609_18935_gb300 import kvm
        self.hq, self.hkv, self.d, self.rot = hq, hkv, d, rot
        self.ctx = kvm.Context([kvm.LAYER_ATTN], hq, hkv, d, rot, THETA, 8, 64, 64, [max(1, l + extra) for l in lives],
                               64 * len(lives))
        self.ctx.draft_reserve(64 * len(lives))
        self.caches, self.cursor = [], [l + cursor for l in lives]
        for b, l in enumerate(lives):
            K = W.normal_bf16((seed, 1, b), (hkv, l, d), unit_last=True, scale=1.0)
            V = W.normal_bf16((seed, 2, b), (hkv, l, d))
            self.ctx.load_prefix(b, l, l + cursor, np.arange(l, dtype=np.int32) + cursor)
            if l:
                self.ctx.set_kv(0, b, _bf(K), _bf(V))
            self.caches.append(O.AttnCache(O.bf16_to_f64(K), O.bf16_to_f64(V), np.arange(l) + cursor))

    def inputs(self, n, seed, scale=1.0):
        return (W.normal_bf16((seed, 3), (n, self.hq, self.d)), W.normal_bf16((seed, 4), (n, self.hkv, self.d), unit_last=True),
                W.normal_bf16((seed, 5), (n, self.hkv, self.d)))

    def run(self, trees, x):
        import torch
        q, k, v = (_bf(t) for t in x)
        out = torch.full_like(q, float("nan"))
        self.ctx.draft_begin(cu_of(trees), packed(trees))
        self.ctx.draft_attn(0, q, k, v, out)
        self.ctx.check()
        return out

    def bound(self, b, parent, q, k, v):
        """(the oracle's outputs, how far each may be off) of one character's nodes."""
        c, g, s = self.caches[b], self.hq // self.hkv, 1.0 / math.sqrt(self.d)
        want, off = np.zeros(q.shape), np.zeros(q.shape)
        for i in range(len(parent)):
            t = O.draft_path(parent, i)
            pos = self.cursor[b] + np.arange(len(t))
            kr = O.rope(k[t], pos, self.rot, THETA)
            qr = O.rope(q[i][None], pos[-1:], self.rot, THETA)[0]
            for h in range(self.hq):
                K = np.concatenate([c.K[h // g], kr[:, h // g]])
                V = np.concatenate([c.V[h // g], v[t][:, h // g]])
                sc = K @ qr[h] * s
                w = np.exp(sc - sc.max())
                w /= w.sum()
                want[i, h] = w @ V
                e = (2 * 2.0 ** -8 + 2.0 ** -16) * (np.abs(K) @ np.abs(qr[h])).max() * s
                off[i, h] = 2.0 ** -8 * np.abs(want[i, h]) + (2.0 ** -8 + math.expm1(2 * e) + 1e-5) * (w @ np.abs(V))
        return want, off

    def check(self, trees, x, out):
        from harness import rel_l2
        got, at = _f64(out), 0
        q, k, v = (O.bf16_to_f64(t) for t in x)
        for b, t in enumerate(trees):
            if not t:
                continue
            sl = slice(at, at + len(t))
            want, off = self.bound(b, t, q[sl], k[sl], v[sl])
            assert np.all(np.abs(got[sl] - want) <= off), (b, np.abs(got[sl] - want).max())
            assert rel_l2(got[sl], want) <= 5e-3, b
            at += len(t)


SHAPES = [(16, 2, 256, 64), (8, 2, 64, 64), (16, 4, 128, 128), (4, 4, 64, 6), (64, 1, 128, 0), (8, 4, 256, 250)]


@pytest.mark.parametrize("hq,hkv,d,rot", SHAPES)
@pytest.mark.parametrize("kind,n", [("chain", 1), ("chain", 2), ("tree", 5), ("star", 17), ("comb", 33), ("forest", 63),
                                    ("tree", 64), ("chain", 64)])
def test_attention_of_one_tree(hq, hkv, d, rot, kind, n):
    for live in (0, 1, 61, 64, 200):
        a = Attn(hq, hkv, d, rot, [live], seed=live + n)
        x = a.inputs(n, seed=n)
        a.check([tree(kind, n)], x, a.run([tree(kind, n)], x))


@pytest.mark.parametrize("hq,hkv,d,rot", SHAPES[:3])
def test_attention_of_a_ragged_population(hq, hkv, d, rot):
    lives = [300, 0, 129, 64, 7, 1023, 63, 500, 0, 1]
    kinds = ["tree", "star", "chain", "roots", "forest", "comb", "tree", "chain", "tree", "chain"]
    sizes = [9, 3, 0, 64, 17, 1, 33, 0, 2, 5]
    a = Attn(hq, hkv, d, rot, lives, seed=11, cursor=100000)
    trees = [tree(k, n, b) for b, (k, n) in enumerate(zip(kinds, sizes))]
    x = a.inputs(sum(sizes), seed=12)
    a.check(trees, x, a.run(trees, x))


def test_attention_of_a_long_cache_split_over_blocks():
    for live, n in ((8192, 16), (5000, 64), (20000, 1)):
        a = Attn(16, 2, 256, 64, [live], seed=21)
        x = a.inputs(n, seed=22)
        a.check([tree("tree", n)], x, a.run([tree("tree", n)], x))


@pytest.mark.parametrize("hq,hkv,d,rot", [(16, 2, 256, 64), (8, 2, 64, 64), (16, 4, 128, 0)])
def test_nodes_appended_by_the_attention_or_before_it(hq, hkv, d, rot):
    """Characters of one query tile each are appended by the attention itself: one launch.  With a larger tree beside them their
    outputs and rows are the same bits (every tile here is one block's)."""
    import torch
    small, big = 128 * hkv // hq, 64
    lives = [130, 0, 63, 77]
    trees = [tree("tree", small, b) for b in range(3)]
    x = Attn(hq, hkv, d, rot, lives, seed=25).inputs(3 * small + big, seed=26)
    rows = []
    for extra in (False, True):
        a = Attn(hq, hkv, d, rot, lives, seed=25)
        t = trees + [tree("tree", big, 3) if extra else []]
        n = sum(map(len, t))
        q, k, v = (_bf(z[:n]) for z in x)
        out = torch.empty_like(q)
        a.ctx.draft_begin(cu_of(t), packed(t))
        before = a.ctx.launch_count()
        a.ctx.draft_attn(0, q, k, v, out)
        assert a.ctx.launch_count() - before == (2 if extra else 1)
        path = [O.draft_path(y, len(y) - 1) if y else [] for y in t]
        a.ctx.draft_commit(cu_of(path), packed(path))
        a.ctx.check()
        rows.append([out[:3 * small]] + [z for b in range(3) for z in (*a.ctx.get_kv(0, b), a.ctx.get_positions(b))])
    for y, z in zip(*rows):
        assert torch.equal(y, z) if torch.is_tensor(y) else np.array_equal(y, z)


def test_attention_of_many_trees_dealt_in_waves():
    lives = [700 + 37 * b for b in range(24)]
    trees = [tree("tree", 64 - b, b) for b in range(24)]
    a = Attn(16, 4, 64, 64, lives, seed=23)
    x = a.inputs(sum(map(len, trees)), seed=24)
    a.check(trees, x, a.run(trees, x))


@pytest.mark.parametrize("d", [64, 256])
def test_attention_of_many_small_trees_dealt_in_waves(d):
    """More than two waves of query tiles whose blocks append the nodes themselves."""
    lives = [100 + 11 * b for b in range(96)]
    trees = [tree("tree", 1 + b % 7, b) for b in range(96)]
    a = Attn(8, 4, d, 32, lives, seed=27)
    x = a.inputs(sum(map(len, trees)), seed=28)
    a.check(trees, x, a.run(trees, x))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("most", [3, 40])
def test_attention_of_segments_of_one_key_tile(d, most):
    """Blocks of several query tiles of one or two key tiles each, the first one among them: a block's second Q may be staged
    before its producers have looked for the first.  Nodes appended by the attention (up to 3 nodes) and before it."""
    lives = [(7 * b) % 61 for b in range(100)]
    trees = [tree("tree", 1 + b % most, b) for b in range(100)]
    a = Attn(16, 4, d, 32, lives, seed=29)
    x = a.inputs(sum(map(len, trees)), seed=30)
    out = a.run(trees, x).clone()
    a.check(trees, x, out)
    for _ in range(10):
        assert bool((a.run(trees, x) == out).all())


@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_node_outside_the_path_changes_nothing(d):
    """Bit for bit: other keys and values of node j move the outputs of j and its descendants only."""
    import torch
    n, live = 40, 90
    a = Attn(8, 2, d, 32, [live], seed=31)
    t = tree("tree", n, 5)
    x = a.inputs(n, seed=32)
    base = a.run([t], x).clone()
    for j in (0, 3, 17, 39):
        y = [z.copy() for z in x]
        y[1][j] = W.normal_bf16((33, j), y[1][j].shape, scale=3.0)
        y[2][j] = W.normal_bf16((34, j), y[2][j].shape, scale=300.0)
        out = a.run([t], y)
        for i in range(n):
            same = torch.equal(out[i].view(torch.int16), base[i].view(torch.int16))
            assert same == (j not in O.draft_path(t, i)), (i, j)


def test_a_chain_equals_a_tail():
    """What the tail call gives, and after a commit its rows and positions bit for bit.  A tile of one block alone is the same bit
    for bit too.  Where several blocks share a tile, the two calls cut its keys at other places: a part's weights are rounded to
    bf16 relative to the part's own largest score, so each side has roundings of its own, of at most the size that the bound on
    either against the oracle counts (2^-8 of sum p |v|); both are held to that bound."""
    import torch
    for live, n in ((50, 7), (3000, 64), (0, 1)):
        a, b = Attn(16, 2, 256, 64, [live], seed=41), Attn(16, 2, 256, 64, [live], seed=41)
        x = a.inputs(n, seed=42)
        out = a.run([tree("chain", n)], x)
        q, k, v = (_bf(t) for t in x)
        ref = torch.empty_like(q)
        cu = np.array([0, n], np.int32)
        b.ctx.tail_attn_prefill(0, cu, q, k, v, ref)
        b.ctx.advance(cu)
        if live < 256:
            assert torch.equal(out.view(torch.int16), ref.view(torch.int16))
        else:
            for got in (out, ref):
                a.check([tree("chain", n)], x, got)
        a.ctx.draft_commit(cu, np.arange(n))
        assert a.ctx.get_live(0) == b.ctx.get_live(0)
        for s, t in zip((*a.ctx.get_kv(0, 0), a.ctx.get_positions(0)), (*b.ctx.get_kv(0, 0), b.ctx.get_positions(0))):
            assert torch.equal(s.view(torch.int16) if s.dtype == torch.bfloat16 else s, t.view(torch.int16) if t.dtype == torch.bfloat16 else t)


@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 256), (8, 2, 64), (16, 4, 128)])
@pytest.mark.parametrize("spread", [3.0, 10.0])
def test_attention_of_scores_far_apart(hq, hkv, d, spread):
    """Scores with a standard deviation of 3 and 10: a few keys hold a row's weight, its maximum moves from tile to tile and from
    block to block, tiles and parts weigh nothing, and a tile that the tree masks throughout stands beside the one with the maximum.
    Without rotary dims queries and keys are exact, so a score is off by its sum in 32 bits alone, e = 2 D 2^-24 max sum_d |q_d k_d| /
    sqrt(D) (and 2^-21 for the exponential), and an output by 2^-8 |o| + (2^-8 + expm1(2 e) + 1e-5) sum_j p_j |v_j|."""
    for live, n, kind in ((0, 64, "roots"), (60, 64, "star"), (63, 2, "chain"), (200, 33, "comb"), (8192, 16, "tree"), (20000, 24, "tree")):
        a = Attn(hq, hkv, d, 0, [live], seed=35)
        V = W.normal_bf16((36, live, 1), (hkv, live, d))
        K = W.normal_bf16((36, live, 2), (hkv, live, d), scale=spread)
        if live:
            a.ctx.set_kv(0, 0, _bf(K), _bf(V))
        a.caches[0] = O.AttnCache(O.bf16_to_f64(K), O.bf16_to_f64(V), np.arange(live))
        x = list(a.inputs(n, seed=37))
        x[1] = W.normal_bf16((38, n), (n, hkv, d), scale=spread)
        t = tree(kind, n, 3)
        got = _f64(a.run([t], x))
        q, k, v = (O.bf16_to_f64(z) for z in x)
        c, far = a.caches[0], 0.0
        for i in range(n):
            p = O.draft_path(t, i)
            for h in range(hq):
                kk = np.concatenate([c.K[h // (hq // hkv)], k[p][:, h // (hq // hkv)]])
                vv = np.concatenate([c.V[h // (hq // hkv)], v[p][:, h // (hq // hkv)]])
                sc = kk @ q[i, h] / math.sqrt(d)
                w = np.exp(sc - sc.max())
                w /= w.sum()
                far = max(far, sc.max() - sc.min())
                e = 2 * d * 2.0 ** -24 * (np.abs(kk) @ np.abs(q[i, h])).max() / math.sqrt(d) + 2.0 ** -21
                off = 2.0 ** -8 * np.abs(w @ vv) + (2.0 ** -8 + math.expm1(2 * e) + 1e-5) * (w @ np.abs(vv))
                assert np.all(np.abs(got[i, h] - w @ vv) <= off), (live, i, h, np.abs(got[i, h] - w @ vv).max())
        assert live < 200 or far > 4 * spread


# ---------------------------------------------------------------------------- delta rule
class Gdn:
    def __init__(self, h, dk, dv, chars, seed, conv=False, layers=1):
        import torch
        from paper_2609_18935_gb300 import kvm
        self.h, self.dk, self.dv, self.chars, self.conv = h, dk, dv, chars, conv
        self.ctx = kvm.Context([kvm.LAYER_GDN] * layers, 8, 2, 64, 64, THETA, h, dk, dv, [256] * chars, 64 * chars,
                               conv_kernel=4 if conv else 0)
        self.ctx.draft_reserve(64 * chars)
        self.S = W.state_f32((seed, 1), (chars, h, dv, dk))
        self.ctx.set_state(0, torch.from_numpy(self.S).cuda())
        self.w = self.old = None
        if conv:
            c = h * (2 * dk + dv)
            self.w = W.conv_weights((seed, 2), c)
            self.old = W.normal_bf16((seed, 3), (chars, 3, c))
            self.ctx.set_conv_weights(0, torch.from_numpy(self.w).cuda())
            self.ctx.set_conv_state(0, _bf(self.old))

    def inputs(self, n, seed):
        a, b = W.gates((seed, 7), n, self.h)
        return {"q": W.normal_bf16((seed, 4), (n, self.h, self.dk)),
                "k": W.normal_bf16((seed, 5), (n, self.h, self.dk), unit_last=True),
                "v": W.normal_bf16((seed, 6), (n, self.h, self.dv)), "alpha": a, "beta": b}

    def tensors(self, x):
        import torch
        return [_bf(x[n]) for n in ("q", "k", "v")] + [torch.from_numpy(x[n]).cuda() for n in ("alpha", "beta")]

    def run(self, trees, x, begin=True):
        import torch
        q, k, v, al, be = self.tensors(x)
        out = torch.full_like(v, float("nan"))
        if begin:
            self.ctx.draft_begin(cu_of(trees), packed(trees))
        self.ctx.draft_gdn(0, q, k, v, al, be, out)
        self.ctx.check()
        return out

    def want(self, trees, x):
        """Per character the oracle's (outputs, states), None without nodes."""
        r, at = [], 0
        y = {n: O.bf16_to_f64(t) if t.dtype == np.uint16 else O.f32_to_f64(t) for n, t in x.items()}
        for b, t in enumerate(trees):
            sl = slice(at, at + len(t))
            r.append(O.draft_gdn(y["q"][sl], y["k"][sl], y["v"][sl], y["alpha"][sl], y["beta"][sl], O.f32_to_f64(self.S[b]), t,
                                 O.bf16_to_f64(self.old[b]) if self.conv else None, self.w) if t else None)
            at += len(t)
        return r

    def check(self, trees, x, out):
        from harness import rel_l2
        got, at = _f64(out), 0
        y = {n: O.bf16_to_f64(t) if t.dtype == np.uint16 else O.f32_to_f64(t) for n, t in x.items()}
        for b, (t, w) in enumerate(zip(trees, self.want(trees, x))):
            n = len(t)
            if not n:
                continue
            o, states = w
            sl = slice(at, at + n)
            if self.conv:
                assert rel_l2(got[sl], o) <= 5e-3, b
            else:
                S0 = O.f32_to_f64(self.S[b])
                off = 2.0 ** -8 * np.abs(o)
                q, k, v, al, be = (y[m][sl] for m in ("q", "k", "v", "alpha", "beta"))
                u = np.zeros((n, self.h, self.dv))
                for i in range(n):
                    Sp = S0 if t[i] < 0 else states[t[i]]
                    u[i] = be[i][:, None] * (v[i] - al[i][:, None] * np.einsum("hvk,hk->hv", Sp, k[i]))
                    path = O.draft_path(t, i)
                    mag = np.linalg.norm(S0, axis=-1) * np.linalg.norm(q[i], axis=-1)[:, None] * np.prod(al[path], 0)[:, None]
                    for z, j in enumerate(path):
                        R = np.prod(al[path[z + 1:]], 0)
                        mag = mag + (R * np.abs((q[i] * k[j]).sum(-1)))[:, None] * np.abs(u[j])
                    off[i] += 2.0 ** -13 * mag
                assert np.all(np.abs(got[sl] - o) <= off), (b, np.abs(got[sl] - o).max())
            at += n


GSHAPES = [(16, 128, 128), (3, 128, 32), (2, 64, 64), (1, 64, 96), (4, 128, 96), (2, 64, 128)]
GTREES = [("chain", 1), ("chain", 2), ("star", 8), ("tree", 9), ("comb", 17), ("roots", 31), ("forest", 33), ("tree", 64),
          ("chain", 64)]


@pytest.mark.parametrize("h,dk,dv", GSHAPES)
@pytest.mark.parametrize("conv", [False, True])
def test_delta_rule_of_one_tree(h, dk, dv, conv):
    for kind, n in GTREES:
        g = Gdn(h, dk, dv, 1, seed=n, conv=conv)
        x = g.inputs(n, seed=n)
        g.check([tree(kind, n)], x, g.run([tree(kind, n)], x))


@pytest.mark.parametrize("h,dk,dv", GSHAPES[:3])
@pytest.mark.parametrize("conv", [False, True])
def test_delta_rule_of_a_ragged_population_and_its_commit(h, dk, dv, conv):
    from harness import rel_l2
    sizes = [9, 0, 64, 1, 17, 33, 5, 0, 2]
    kinds = ["tree", "star", "tree", "chain", "comb", "forest", "star", "tree", "roots"]
    trees = [tree(k, n, b) for b, (k, n) in enumerate(zip(kinds, sizes))]
    g = Gdn(h, dk, dv, len(sizes), seed=51, conv=conv)
    x = g.inputs(sum(sizes), seed=52)
    g.check(trees, x, g.run(trees, x))
    before = g.ctx.get_state(0).cpu().numpy()
    assert np.array_equal(before, g.S)                          # a draft leaves the state alone
    # the longest path of each tree; character 4 keeps nothing
    paths = [max((O.draft_path(t, i) for i in range(len(t))), key=len) if t else [] for t in trees]
    paths[4] = []
    live = [g.ctx.get_live(b) for b in range(len(sizes))]
    g.ctx.draft_commit(cu_of(paths), np.array(sum(paths, []), np.int32))
    g.ctx.check()
    after = g.ctx.get_state(0).cpu().numpy()
    for b, (path, w) in enumerate(zip(paths, g.want(trees, x))):
        assert g.ctx.get_live(b) == (live[b][0] + len(path), live[b][1] + len(path))
        if not path:
            assert np.array_equal(after[b], before[b])
            continue
        for hh in range(h):
            assert rel_l2(after[b, hh], w[1][path[-1]][hh]) <= (5e-3 if conv else 1e-5), (b, hh)
    if conv:
        from harness import torch_bf16_bits
        st, cu = torch_bf16_bits(g.ctx.get_conv_state(0)), cu_of(trees)
        raw = np.concatenate([x[m].reshape(len(x[m]), -1) for m in ("q", "k", "v")], 1)
        for b, path in enumerate(paths):
            assert np.array_equal(st[b], np.concatenate([g.old[b], raw[cu[b] + np.array(path, np.int64)]])[-3:]), b


@pytest.mark.parametrize("conv", [False, True])
def test_a_dead_gate_and_a_full_one(conv):
    """alpha = 0 forgets everything before the node, alpha = 1 nothing; beta = 0 and 1 too."""
    g = Gdn(2, 64, 64, 1, seed=61, conv=conv)
    t = tree("tree", 20, 6)
    x = g.inputs(20, seed=62)
    x["alpha"][3], x["alpha"][7], x["alpha"][0] = 0.0, 0.0, 1.0
    x["beta"][4], x["beta"][5] = 0.0, 1.0
    g.check([t], x, g.run([t], x))
    path = max((O.draft_path(t, i) for i in range(20)), key=len)
    g.ctx.draft_commit([0, len(path)], path)
    S = g.ctx.get_state(0).cpu().numpy()[0]
    from harness import rel_l2
    assert rel_l2(S, g.want([t], x)[0][1][path[-1]]) <= (5e-3 if conv else 1e-5)


def test_delta_rule_outside_the_path_changes_nothing():
    import torch
    g = Gdn(2, 128, 64, 1, seed=71)
    t = tree("tree", 30, 8)
    x = g.inputs(30, seed=72)
    base = g.run([t], x).clone()
    for j in (0, 4, 11, 29):
        y = {m: z.copy() for m, z in x.items()}
        y["k"][j] = W.normal_bf16((73, j), y["k"][j].shape, unit_last=True)
        y["v"][j] = W.normal_bf16((74, j), y["v"][j].shape, scale=100.0)
        y["alpha"][j], y["beta"][j] = 0.3, 0.9
        out = g.run([t], y)
        for i in range(30):
            assert torch.equal(out[i], base[i]) == (j not in O.draft_path(t, i)), (i, j)


@pytest.mark.parametrize("h,dk,dv", [(16, 128, 128), (5, 64, 96)])
def test_convolved_inputs_are_those_of_a_tail(h, dk, dv):
    """Bit for bit: from a state of 0, gates of 1 and one token a committed node leaves v k^T (exact products of two bf16 numbers),
    and so does a tail."""
    import torch
    chars = 64
    a, b = (Gdn(h, dk, dv, chars, seed=63, conv=True) for _ in range(2))
    x = a.inputs(chars, seed=64)
    for m in ("q", "k", "v"):                                   # pre-activations from small to about -40
        x[m][::2] = W.f64_to_bf16_bits(8.0 * O.bf16_to_f64(x[m][::2])) if m != "k" else W.f64_to_bf16_bits(60.0 * O.bf16_to_f64(x[m][::2]))
    x["alpha"][:], x["beta"][:] = 1.0, 1.0
    for g in (a, b):
        g.ctx.set_state(0, torch.zeros(chars, h, dv, dk, device="cuda"))
    a.run([[-1]] * chars, x)
    cu = np.arange(chars + 1, dtype=np.int32)
    a.ctx.draft_commit(cu, np.zeros(chars, np.int32))
    q, k, v, al, be = b.tensors(x)
    b.ctx.gdn_chunk_scan_from_state(0, cu, q, k, v, al, be, torch.empty_like(v))
    S, T = a.ctx.get_state(0), b.ctx.get_state(0)
    assert bool((T != 0).any()) and int((S != T).sum()) == 0


@pytest.mark.parametrize("h,dk,dv", [(16, 128, 128), (5, 64, 96)])
@pytest.mark.parametrize("kind,n", [("chain", 30), ("tree", 64), ("comb", 40), ("forest", 50), ("star", 12)])
def test_a_convolved_path_leaves_the_state_of_a_tail(h, dk, dv, kind, n):
    """The state after the commit of a path, and after a tail of the path's tokens (at most 30: token by token, in 32 bits), from the
    same inputs bit for bit (the test above): within the 1e-5 of either from the oracle without the convolution."""
    import torch
    from harness import rel_l2
    t = tree(kind, n, 7)
    path = max((O.draft_path(t, i) for i in range(n)), key=len)
    assert len(path) <= 32
    a, b = (Gdn(h, dk, dv, 1, seed=65, conv=True) for _ in range(2))
    x = a.inputs(n, seed=66)
    a.run([t], x)
    a.ctx.draft_commit([0, len(path)], path)
    q, k, v, al, be = b.tensors({m: np.ascontiguousarray(z[path]) for m, z in x.items()})
    b.ctx.gdn_chunk_scan_from_state(0, [0, len(path)], q, k, v, al, be, torch.empty_like(v))
    S, T = (c.ctx.get_state(0).cpu().numpy()[0] for c in (a, b))
    for hh in range(h):
        assert rel_l2(S[hh], T[hh]) <= 2e-5, hh
    assert torch.equal(a.ctx.get_conv_state(0).view(torch.int16), b.ctx.get_conv_state(0).view(torch.int16))


def _reported(ctx):
    from paper_2609_18935_gb300 import kvm
    with pytest.raises(kvm.KvmError) as ei:
        ctx.check()
    assert ei.value.code == kvm.KVM_E_DEVICE and "value-not-finite" in str(ei.value)
    ctx.check()


NOT_FINITE = (0x7FC0, 0x7F80, 0xFF80, 0xFFFF)                                   # NaN, inf, -inf, -NaN in bf16


@pytest.mark.parametrize("d,rot", [(64, 64), (128, 0), (256, 64)])
def test_keys_and_values_that_are_not_finite_stay_with_their_node(d, rot):
    """Other nodes' outputs bit for bit, and those of a later, shorter draft whose last tile holds the rows."""
    import torch
    n, live = 21, 70
    a = Attn(8, 2, d, rot, [live], seed=75)
    t = tree("tree", n, 5)
    x = a.inputs(n, seed=76)
    base = a.run([t], x).clone()
    y = [z[:3] for z in x]
    short = a.run([t[:3]], y).clone()
    for which in (1, 2):
        for j, bits in zip((0, 4, 13, 20), NOT_FINITE):
            bad = [z.copy() for z in x]
            bad[which][j, 1, 5] = bits
            bad[which][j, 0, -1] = bits
            q, k, v = (_bf(z) for z in bad)
            out = torch.zeros_like(q)
            a.ctx.draft_begin(cu_of([t]), packed([t]))
            a.ctx.draft_attn(0, q, k, v, out)
            _reported(a.ctx)
            for i in range(n):
                assert j in O.draft_path(t, i) or torch.equal(out[i], base[i]), (which, i, j)
            assert torch.equal(a.run([t[:3]], y), short)


@pytest.mark.parametrize("d,rot,n", [(64, 6, 21), (128, 48, 21), (256, 250, 21), (64, 64, 50), (128, 0, 50), (256, 16, 50), (128, 2, 64)])
def test_every_way_into_the_caches_keeps_what_is_not_finite_out(d, rot, n):
    """Rotary dims of any number, and trees of several query tiles: other nodes' outputs and the rows that a commit keeps bit for
    bit, a later tail's outputs too, and every call reports."""
    import torch
    live = 70
    a, ref = Attn(8, 2, d, rot, [live], seed=75), Attn(8, 2, d, rot, [live], seed=75)
    t = tree("tree", n, 5)
    x = a.inputs(n, seed=76)
    base = a.run([t], x).clone()
    one = [_bf(z[:1]) for z in x]
    cu = np.array([0, 1], np.int32)
    after = torch.empty_like(one[0])
    ref.ctx.tail_attn_prefill(0, cu, *one, after)
    for which in (1, 2):
        for j, bits in zip((0, 4, 13, n - 1), NOT_FINITE):
            bad = [z.copy() for z in x]
            bad[which][j, 1, 5 * d // 8] = bits
            bad[which][j, 0, -1] = bits
            bad[which][j, 1, 0] = bits
            q, k, v = (_bf(z) for z in bad)
            out = torch.zeros_like(q)
            a.ctx.draft_begin(cu_of([t]), packed([t]))
            a.ctx.draft_attn(0, q, k, v, out)
            _reported(a.ctx)
            for i in range(n):
                assert j in O.draft_path(t, i) or torch.equal(out[i], base[i]), (which, i, j)
            got = torch.zeros_like(after)
            a.ctx.tail_attn_prefill(0, cu, *one, got)
            a.ctx.check()
            assert torch.equal(got, after), (which, j)
    # a path through the last of them (the value of its first head's last dim): what was not finite went in as 0
    a.ctx.draft_begin(cu_of([t]), packed([t]))
    a.ctx.draft_attn(0, q, k, v, out)
    _reported(a.ctx)
    path = O.draft_path(t, n - 1)
    a.ctx.draft_commit([0, len(path)], path)
    K, V = a.ctx.get_kv(0, 0)
    want = x[2][path].copy()
    want[-1][0, -1] = want[-1][1, 5 * d // 8] = want[-1][1, 0] = 0
    assert torch.equal(V[:, live:].view(torch.int16), _bf(want).transpose(0, 1).contiguous().view(torch.int16))
    assert bool(torch.isfinite(K).all())
    a.ctx.check()


@pytest.mark.parametrize("conv", [False, True])
def test_a_delta_rule_node_that_is_not_finite_stays_alone(conv):
    """Other nodes' outputs bit for bit, and the state after a commit of a path without it."""
    import torch
    n = 37
    t = tree("tree", n, 8)
    g = Gdn(2, 128, 64, 1, seed=77, conv=conv)
    x = g.inputs(n, seed=78)
    base = g.run([t], x).clone()
    path = O.draft_path(t, 36)
    out_of_path = [i for i in range(n) if i not in path and not set(O.draft_path(t, i)[1:]) & set(path[1:])]
    for name in ("k", "v", "alpha", "beta"):
        for j, bits in zip((5, out_of_path[0], out_of_path[-1]), NOT_FINITE):
            bad = {m: z.copy() for m, z in x.items()}
            if name in ("k", "v"):
                bad[name][j, 0, 3] = bits
            else:
                bad[name][j, 0] = np.array([bits << 16], np.uint32).view(np.float32)[0]
            dev = {m: _bf(z) if z.dtype == np.uint16 else torch.from_numpy(z).cuda() for m, z in bad.items()}
            out = torch.zeros_like(dev["v"])
            g.ctx.draft_begin(cu_of([t]), packed([t]))
            g.ctx.draft_gdn(0, dev["q"], dev["k"], dev["v"], dev["alpha"], dev["beta"], out)
            _reported(g.ctx)
            for i in range(n):
                assert j in O.draft_path(t, i) or torch.equal(out[i], base[i]), (name, i, j)
    # the last draft's bad node is off this path
    assert j not in path
    g.ctx.draft_commit([0, len(path)], path)
    got = g.ctx.get_state(0).cpu().numpy()[0]
    other = Gdn(2, 128, 64, 1, seed=77, conv=conv)
    other.run([t], x)
    other.ctx.draft_commit([0, len(path)], path)
    assert np.array_equal(got, other.ctx.get_state(0).cpu().numpy()[0])


@pytest.mark.parametrize("conv", [False, True])
@pytest.mark.parametrize("bits", NOT_FINITE)
def test_a_committed_key_that_is_not_finite_counts_as_0(conv, bits):
    """Without the convolution the state is, bit for bit, what a key of 0 leaves in the head (in 32-bit sums a coefficient of 0 and an
    update of 0 both add nothing); with it the state is finite."""
    import torch
    n = 37
    t = tree("tree", n, 8)
    path = O.draft_path(t, 36)
    assert len(path) > 4
    got = []
    for put in (bits, 0):
        g = Gdn(2, 128, 64, 1, seed=77, conv=conv)
        x = g.inputs(n, seed=78)
        x["k"][path[2], 0, :] = 0
        x["k"][path[2], 0, 3] = put
        q, k, v, al, be = g.tensors(x)
        out = torch.zeros_like(v)
        g.ctx.draft_begin(cu_of([t]), packed([t]))
        g.ctx.draft_gdn(0, q, k, v, al, be, out)
        if put:
            _reported(g.ctx)
        g.ctx.draft_commit([0, len(path)], path)
        g.ctx.check()
        got.append(g.ctx.get_state(0))
    assert bool(torch.isfinite(got[0]).all()) and bool(torch.isfinite(got[1]).all())
    if not conv:
        assert torch.equal(got[0], got[1])
    assert torch.equal(got[0][0, 1], got[1][0, 1])              # the other head


@pytest.mark.parametrize("h,dk,dv", [(16, 128, 128), (4, 64, 32)])
@pytest.mark.parametrize("name", ["k", "v", "alpha"])
def test_lanes_of_a_warp_that_part_ways(h, dk, dv, name):
    """64 nodes, one of them not finite: rows of a warp with and without a coefficient in a block of nodes, with and without
    something to clear, and (a small decay) with paths of their own length to multiply along.  Again and again the same bits, those of
    the draft without it where they do not depend on it."""
    import torch
    for kind in ("tree", "comb", "forest"):
        t = tree(kind, 64, 9)
        g = Gdn(h, dk, dv, 2, seed=79)
        x = g.inputs(128, seed=80)
        x["alpha"][5] = 2.0 ** -60
        base = g.run([t, t], x).clone()
        g.check([t, t], x, base)
        bad = {m: z.copy() for m, z in x.items()}
        bad[name][40, 0, ...] = np.nan if name == "alpha" else 0x7FC0
        dev = g.tensors(bad)
        first = None
        for _ in range(10):
            out = torch.zeros_like(dev[2])
            g.ctx.draft_begin(cu_of([t, t]), packed([t, t]))
            g.ctx.draft_gdn(0, *dev, out)
            _reported(g.ctx)
            for i in range(64):
                assert 40 in O.draft_path(t, i) or torch.equal(out[i], base[i]), (kind, i)
            assert torch.equal(out[64:], base[64:])
            bits = out.view(torch.int16)
            first = bits.clone() if first is None else first
            assert torch.equal(bits, first)


# ---------------------------------------------------------------------------- verdicts
class Verdict:
    def __init__(self, chars):
        from paper_2609_18935_gb300 import kvm
        self.chars = chars
        self.ctx = kvm.Context([kvm.LAYER_ATTN], 4, 2, 64, 64, THETA, 8, 64, 64, [128] * chars, 64 * chars)
        self.ctx.draft_reserve(64 * chars)

    def run(self, trees, tokens, target, draft, u, u_next, dtype=None):
        """target, draft: torch CPU tensors in the type under test."""
        import torch
        n = sum(map(len, trees))
        dev = lambda a, dt: torch.as_tensor(np.asarray(a), dtype=dt).cuda()
        path = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        count, nxt = (torch.full((self.chars,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
        self.ctx.draft_begin(cu_of(trees), packed(trees))
        self.ctx.draft_verify(dev(tokens, torch.int32), target.cuda(), draft.cuda(), dev(u, torch.float32), dev(u_next, torch.float32),
                              path, count, nxt)
        return path.cpu().numpy(), count.cpu().numpy(), nxt.cpu().numpy()

    def check(self, trees, tokens, target, draft, u, u_next):
        path, count, nxt = self.run(trees, tokens, target, draft, u, u_next)
        self.ctx.check()
        P, Q, at = target.double().numpy(), draft.double().numpy(), 0
        for b, t in enumerate(trees):
            n = len(t)
            if not n:
                assert count[b] == 0 and nxt[b] == -1
                continue
            sl = slice(at, at + n)
            want, x = O.draft_verdict(t, tokens[sl], P[sl], Q[sl], np.asarray(u, np.float32)[sl], np.float32(u_next[b]))
            assert list(path[sl]) == want + [-1] * (n - len(want)), b
            assert count[b] == len(want) and nxt[b] == x, (b, want, nxt[b], x)
            at += n


def _rows(r, n, V, dtype, sharp=2.0, near=0.7):
    import torch
    a = sharp * r.standard_normal((n, V))
    b = a + near * r.standard_normal((n, V))
    soft = lambda z: np.exp(z - z.max(1, keepdims=True)) / np.exp(z - z.max(1, keepdims=True)).sum(1, keepdims=True)
    return torch.tensor(soft(b), dtype=dtype), torch.tensor(soft(a), dtype=dtype)


@pytest.mark.parametrize("V", [1, 2, 3, 5, 31, 127, 128, 129, 1000, 4097, 33000, 131072])
@pytest.mark.parametrize("bf16", [False, True])
def test_verdicts(V, bf16):
    import torch
    r = np.random.default_rng(V)
    dtype = torch.bfloat16 if bf16 else torch.float32
    sizes = [5, 0, 1, 16, 9] if V > 30000 else [5, 0, 1, 64, 33, 16, 2, 7]
    trees = [tree(k, n, V + i) for i, (k, n) in enumerate(zip(["tree", "tree", "chain", "comb", "star", "tree", "chain", "star"], sizes))]
    v = Verdict(len(trees))
    n = sum(sizes)
    for near in (0.3, 1.5):
        target, draft = _rows(r, n, V, dtype, near=near)
        # each token drawn from its parent's draft row
        cu, tokens = cu_of(trees), np.zeros(n, np.int64)
        for b, t in enumerate(trees):
            for i, p in enumerate(t):
                cum = np.cumsum(draft[cu[b] + max(p, 0)].double().numpy())
                tokens[cu[b] + i] = min(V - 1, np.searchsorted(cum, r.random() * cum[-1]))
        v.check(trees, tokens, target, draft, r.random(n), r.random(len(trees)))


def test_verdicts_at_their_edges():
    import torch
    r = np.random.default_rng(81)
    v = Verdict(4)
    t = [tree("star", 6, 0)] * 4
    n, V = 24, 700
    target, draft = _rows(r, n, V, torch.float32)
    tokens = r.integers(0, V, n)
    same = draft.clone()
    v.check(t, tokens, same, draft, np.full(n, 0.99999994), r.random(4))           # the draft is the target: the first guess stands
    v.check(t, tokens, target, draft, np.zeros(n), np.zeros(4))                    # uniforms of 0
    v.check(t, tokens, target, draft, np.full(n, 0.99999994), np.full(4, 0.99999994))
    v.check(t, np.repeat(tokens[:4], 6), target, draft, r.random(n), r.random(4))  # the same guess again and again
    zero = target.clone()
    zero[:] = 0.0
    v.check(t, tokens, zero, draft, r.random(n), r.random(4))                      # nothing to draw from
    odd = target.clone()
    odd[:, ::3], odd[:, 1::7], odd[:, 2::11] = -1.0, float("nan"), float("inf")
    v.check(t, tokens, odd, draft, r.random(n), r.random(4))
    hot = torch.zeros_like(target)
    hot[torch.arange(n), torch.as_tensor(r.integers(0, V, n))] = 1.0               # a greedy target
    v.check(t, tokens, hot, draft, r.random(n), r.random(4))
    half = target * 0.5
    v.check(t, tokens, half, draft * 2.0, r.random(n), r.random(4))                # rows that do not sum to 1
    less = torch.minimum(target, draft)                                            # p <= q everywhere: no residual at all
    v.check(t, tokens, less, draft, np.full(n, 0.999), r.random(4))


@pytest.mark.parametrize("V", [700, 5003])
def test_verdicts_over_rows_that_hold_no_probabilities(V):
    """What is not a finite positive number counts as 0, in the target's rows, the draft's and both, after none, one and several
    guesses that fail."""
    import torch
    r = np.random.default_rng([87, V])
    v = Verdict(4)
    n = 24
    rows = _rows(r, n, V, torch.float32)
    odd = []
    for z in rows:
        z = z.clone()
        z[:, ::5], z[:, 1::7], z[:, 2::11], z[:, 3::13] = -1.0, float("nan"), float("inf"), float("-inf")
        odd.append(z)
    tokens = r.integers(0, V, n)
    for kind in ("star", "chain"):
        t = [tree(kind, 6, 0)] * 4
        for target, draft in ((rows[0], odd[1]), (odd[0], rows[1]), odd):
            for u in (np.zeros(n), r.random(n), np.full(n, 0.99999994)):
                v.check(t, tokens, target, draft, u, r.random(4))


def test_a_token_outside_the_vocabulary_is_refused_and_reported():
    import torch
    from paper_2609_18935_gb300 import kvm
    r = np.random.default_rng(82)
    v = Verdict(1)
    target, draft = _rows(r, 3, 50, torch.float32)
    path, count, nxt = v.run([[-1, 0, 0]], [0, 50, -3], target, draft, [0, 0, 0], [0.4])
    assert list(path) == [0, -1, -1] and count[0] == 1 and 0 <= nxt[0] < 50
    with pytest.raises(kvm.KvmError) as ei:
        v.ctx.check()
    assert ei.value.code == kvm.KVM_E_DEVICE
    v.ctx.check()


def test_a_verdict_refuses_outputs_over_its_inputs_and_each_other():
    import torch
    from paper_2609_18935_gb300 import kvm
    v = Verdict(2)
    r = np.random.default_rng(85)
    target, draft = (t.cuda() for t in _rows(r, 5, 40, torch.float32))
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    tokens, path, u, u_next = ints(5), ints(5), torch.zeros(5, device="cuda"), torch.zeros(2, device="cuda")
    count, nxt = ints(2), ints(2)
    v.ctx.draft_begin([0, 3, 5], [-1, 0, 0, -1, 0])
    as_int = lambda t, n: t.view(torch.int32).flatten()[:n]
    for bad in (dict(path=tokens), dict(path=as_int(target, 5)), dict(path=as_int(draft[4], 5)), dict(path=as_int(u, 5)),
                dict(nxt=as_int(u_next, 2)), dict(count=nxt), dict(count=as_int(path, 2)), dict(nxt=as_int(tokens, 2))):
        a = dict(dict(path=path, count=count, nxt=nxt), **bad)
        with pytest.raises(kvm.KvmError) as ei:
            v.ctx.draft_verify(tokens, target, draft, u, u_next, a["path"], a["count"], a["nxt"])
        assert ei.value.code == kvm.KVM_E_INVAL, bad
    v.ctx.draft_verify(tokens, target, draft, u, u_next, path, count, nxt)
    v.ctx.check()


def test_a_verdict_always_writes_its_token():
    """Where nothing can be drawn the token is -1: an empty row, and a uniform below its range."""
    import torch
    r = np.random.default_rng(86)
    for V in (40, 5000):
        target, draft = _rows(r, 2, V, torch.float32)
        target[0] = 0.0
        _, count, nxt = Verdict(2).run([[-1], [-1]], [0, 0], target, draft, [0, 0], [0.5, -0.25])
        assert list(count) == [1, 1] and list(nxt) == [-1, -1], V


def test_verdicts_keep_the_targets_distribution():
    """256 characters, 64 calls: tokens that follow a decided one, with three guesses from the draft, against p.  A frequency of
    16384 draws is within 5 sigma = 5 sqrt(p (1 - p) / 16384) of p but for one in 10^6."""
    import torch
    r = np.random.default_rng(83)
    V, chars, calls = 7, 256, 64
    p, q = r.random(V), r.random(V)
    p, q = (p / p.sum()).astype(np.float32), (q / q.sum()).astype(np.float32)
    v = Verdict(chars)
    trees = [[-1, 0, 0, 0]] * chars
    target, draft = (torch.tensor(np.tile(x, (4 * chars, 1))) for x in (p, q))
    got = np.zeros(V)
    for _ in range(calls):
        tokens = r.choice(V, 4 * chars, p=q.astype(np.float64) / q.astype(np.float64).sum())
        path, count, nxt = v.run(trees, tokens, target, draft, r.random(4 * chars), r.random(chars))
        for b in range(chars):
            got[tokens[4 * b + path[4 * b + 1]] if count[b] > 1 else nxt[b]] += 1
    m = got.sum()
    pd = p.astype(np.float64) / p.astype(np.float64).sum()
    assert np.all(np.abs(got / m - pd) <= 5 * np.sqrt(pd * (1 - pd) / m)), got / m - pd


# ---------------------------------------------------------------------------- steps
def _stack(conv, chars, lives, seed, shape=(8, 2, 128, 64, 4, 128, 64), kinds=None):
    """A context of delta-rule and attention layers and the oracle's states of its characters."""
    from harness import Pair
    hq, hkv, d, rot, h, dk, dv = shape
    s = W.ModelShape(kinds or [W.GDN, W.ATTN, W.GDN, W.ATTN], hq, hkv, d, rot, THETA, h, dk, dv)
    pair = Pair(s, lives, [l + 200 for l in lives], 64 * chars, seed_index=seed, conv=conv)
    pair.ctx.draft_reserve(64 * chars)
    return pair


def _step_inputs(pair, n, seed):
    s, x = pair.shape, {}
    for l, kind in enumerate(s.layer_kind):
        if kind == W.ATTN:
            x[l] = {"q": W.normal_bf16((seed, l, 1), (n, s.n_q_heads, s.head_dim)),
                    "k": W.normal_bf16((seed, l, 2), (n, s.n_kv_heads, s.head_dim), unit_last=True),
                    "v": W.normal_bf16((seed, l, 3), (n, s.n_kv_heads, s.head_dim))}
        else:
            a, b = W.gates((seed, l, 4), n, s.n_gdn_heads)
            x[l] = {"q": W.normal_bf16((seed, l, 1), (n, s.n_gdn_heads, s.d_k)),
                    "k": W.normal_bf16((seed, l, 2), (n, s.n_gdn_heads, s.d_k), unit_last=True),
                    "v": W.normal_bf16((seed, l, 3), (n, s.n_gdn_heads, s.d_v)), "alpha": a, "beta": b}
    return x


def _layers(pair, x, stream=None):
    import torch
    outs = {}
    for l, y in x.items():
        t = {m: _bf(z) if z.dtype == np.uint16 else torch.from_numpy(z).cuda() for m, z in y.items()}
        if pair.shape.layer_kind[l] == W.ATTN:
            outs[l] = torch.empty_like(t["q"])
            pair.ctx.draft_attn(l, t["q"], t["k"], t["v"], outs[l], stream=stream)
        else:
            outs[l] = torch.empty_like(t["v"])
            pair.ctx.draft_gdn(l, t["q"], t["k"], t["v"], t["alpha"], t["beta"], outs[l], stream=stream)
        outs[l].keep = t
    return outs


def _advance_oracle(pair, trees, paths, x):
    """Commit the paths in the oracle: each layer's chain of the accepted nodes."""
    s, cu = pair.shape, cu_of(trees)
    for b, path in enumerate(paths):
        st = pair.oracle[b]
        if not path:
            continue
        rows = cu[b] + np.array(path)
        for l, y in x.items():
            z = {m: O.bf16_to_f64(t[rows]) if t.dtype == np.uint16 else O.f32_to_f64(t[rows]) for m, t in y.items()}
            if s.layer_kind[l] == W.ATTN:
                st.caches[l] = O.tail_attn_prefill(st.caches[l], z["q"], z["k"], z["v"], st.cursor, s.rotary_dim, THETA)[1]
            else:
                q, k, v = z["q"], z["k"], z["v"]
                if pair.conv_w is not None:
                    q, k, v, st.conv[l] = O.gdn_conv_inputs(q, k, v, st.conv[l], pair.conv_w[l])
                st.states[l] = O.gdn_recurrent(q, k, v, z["alpha"], z["beta"], st.states[l])[1]
        st.cursor += len(path)


def _compare_states(pair):
    from harness import rel_l2
    for b, st in enumerate(pair.oracle):
        for l, c in st.caches.items():
            k, v = pair.ctx.get_kv(l, b)
            assert pair.ctx.get_live(b) == (c.live, st.cursor)
            assert np.array_equal(_f64(v), c.V), (l, b)
            assert rel_l2(_f64(k), c.K) <= 2.0 ** -8, (l, b)
            assert np.array_equal(pair.ctx.get_positions(b).cpu().numpy(), c.pos)
        for l, S in st.states.items():
            got = pair.ctx.get_state(l)[b].cpu().numpy()
            assert rel_l2(got, S) <= 5e-3, (l, b)


def _outputs_match(pair, trees, x, outs):
    from harness import rel_l2
    s, cu = pair.shape, cu_of(trees)
    for l, y in x.items():
        got = _f64(outs[l])
        for b, t in enumerate(trees):
            if not t:
                continue
            sl = slice(cu[b], cu[b + 1])
            z = {m: O.bf16_to_f64(u[sl]) if u.dtype == np.uint16 else O.f32_to_f64(u[sl]) for m, u in y.items()}
            st = pair.oracle[b]
            if s.layer_kind[l] == W.ATTN:
                want = O.draft_attention(st.caches[l], z["q"], z["k"], z["v"], t, st.cursor, s.rotary_dim, THETA)
            else:
                want = O.draft_gdn(z["q"], z["k"], z["v"], z["alpha"], z["beta"], st.states[l], t, st.conv.get(l),
                                   pair.conv_w[l] if pair.conv_w is not None else None)[0]
            assert rel_l2(got[sl], want) <= 5e-3, (l, b)


@pytest.mark.parametrize("conv", [False, True])
def test_steps_of_a_population(conv):
    """Three steps: trees drafted through every layer, judged on the GPU, the accepted paths committed; a maintenance round in
    between.  Outputs, caches, positions and states follow the oracle's."""
    import torch
    lives = [70, 0, 200, 129]
    pair = _stack(conv, 4, lives, 91)
    V, r = 60, np.random.default_rng(92)
    for step in range(3):
        sizes = [[9, 3, 0, 20], [1, 12, 33, 0], [64, 2, 5, 7]][step]
        trees = [tree("tree", n, 10 * step + b) for b, n in enumerate(sizes)]
        n = sum(sizes)
        x = _step_inputs(pair, n, 93 + step)
        pair.ctx.draft_begin(cu_of(trees), packed(trees))
        outs = _layers(pair, x)
        _outputs_match(pair, trees, x, outs)
        target, draft = _rows(r, n, V, torch.float32, near=0.3)
        tokens, u, un = r.integers(0, V, n), 0.3 * r.random(n), r.random(4)
        path, count, nxt = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n, 4, 4))
        dev = lambda a, dt: torch.as_tensor(a, dtype=dt).cuda()
        pair.ctx.draft_verify(dev(tokens, torch.int32), target.cuda(), draft.cuda(), dev(u, torch.float32), dev(un, torch.float32), path,
                              count, nxt)
        cu, paths = cu_of(trees), []
        for b, t in enumerate(trees):
            got = [int(i) for i in path[cu[b]:cu[b] + int(count[b])].cpu()]
            if t:
                sl = slice(cu[b], cu[b + 1])
                assert (got, int(nxt[b])) == O.draft_verdict(t, tokens[sl], target[sl].double().numpy(), draft[sl].double().numpy(),
                                                            u[sl].astype(np.float32), np.float32(un[b]))
            paths.append(got)
        pair.ctx.draft_commit(cu_of(paths), sum(paths, []))
        _advance_oracle(pair, trees, paths, x)
        pair.ctx.check()
        _compare_states(pair)
        if step == 0:
            tails = [5, 0, 40, 1]
            live = [pair.ctx.get_live(b)[0] for b in range(4)]
            tx = W.tail_inputs(W.Workload("custom", 95, pair.shape, list(live), 1), 0, tails)
            errs = pair.run_round(np.array([0, 1, 1, 1, 1], np.int32), np.array([3], np.int32), np.array([9], np.int32), tails, tx)
            assert all(e <= 5e-3 for e in errs.values()), errs


def test_deep_paths_of_wide_rows():
    """Paths of up to 64 nodes scattered over their trees, in caches of every row width: rows moved exactly."""
    import torch
    for d in (64, 128, 256):
        pair = _stack(False, 2, [10, 77], 101, shape=(4, 2, d, 32, 2, 64, 32))
        trees = [tree("comb", 64), tree("chain", 64)]
        x = _step_inputs(pair, 128, 102)
        paths = [O.draft_path(trees[0], 62), O.draft_path(trees[1], 63)]
        pair.ctx.draft_begin(cu_of(trees), packed(trees))
        outs = _layers(pair, x)
        pair.ctx.draft_commit(cu_of(paths), sum(paths, []))
        pair.ctx.check()
        _advance_oracle(pair, trees, paths, x)
        _compare_states(pair)
        del outs


def test_a_dropped_draft_leaves_no_trace():
    """Drafts that end without a commit: the state, and what later calls compute, is as if they had never been."""
    import torch
    a, b = _stack(True, 2, [40, 65], 111), _stack(True, 2, [40, 65], 111)
    trees = [tree("tree", 30), tree("tree", 11)]
    a.ctx.draft_begin(cu_of(trees), packed(trees))
    outs = _layers(a, _step_inputs(a, 41, 112))
    a.ctx.draft_begin([0, 1, 1], [-1])                           # another draft, dropped too
    tails = [9, 4]
    tx = W.tail_inputs(W.Workload("custom", 113, a.shape, [40, 65], 1), 0, tails)
    zero = np.zeros(3, np.int32)
    for p in (a, b):
        errs = p.run_round(zero, np.zeros(0, np.int32), np.zeros(0, np.int32), tails, tx)
        assert all(e <= 5e-3 for e in errs.values()), errs
    for l, kind in enumerate(a.shape.layer_kind):
        if kind == W.ATTN:
            for c in range(2):
                for s, t in zip(a.ctx.get_kv(l, c), b.ctx.get_kv(l, c)):
                    assert torch.equal(s.view(torch.int16), t.view(torch.int16))
        else:
            assert torch.equal(a.ctx.get_state(l), b.ctx.get_state(l))
            assert torch.equal(a.ctx.get_conv_state(l).view(torch.int16), b.ctx.get_conv_state(l).view(torch.int16))
    del outs


def test_rows_behind_a_commit_are_left_alone():
    """The other characters' caches and states, and a neighbour's first slot, keep their bytes."""
    pair = _stack(False, 3, [64, 10, 128], 121)
    before = pair.snapshot_kv()
    S = {l: pair.ctx.get_state(l).cpu().numpy() for l in pair.shape.gdn_layers}
    trees = [[], tree("comb", 21), []]
    x = _step_inputs(pair, 21, 122)
    pair.ctx.draft_begin(cu_of(trees), packed(trees))
    _layers(pair, x)
    path = O.draft_path(trees[1], 20)
    pair.ctx.draft_commit([0, 0, len(path), len(path)], path)
    _advance_oracle(pair, trees, [[], path, []], x)
    _compare_states(pair)
    after = pair.snapshot_kv()
    for key, val in before.items():
        n = val[0].shape[1]
        for u, w in zip(val[:2], after[key][:2]):
            assert np.array_equal(u, w[:, :n]), key
    for l, s in S.items():
        t = pair.ctx.get_state(l).cpu().numpy()
        assert np.array_equal(s[0], t[0]) and np.array_equal(s[2], t[2])


def test_a_step_on_a_side_stream_and_in_a_graph():
    """A step on a stream of its own, and the same layers captured and replayed with new inputs in the old buffers."""
    import torch
    pair, ref = _stack(True, 2, [90, 33], 131), _stack(True, 2, [90, 33], 131)
    trees = [tree("tree", 25), tree("star", 6)]
    x, y = _step_inputs(pair, 31, 132), _step_inputs(pair, 31, 133)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pair.ctx.draft_begin(cu_of(trees), packed(trees))
        outs = _layers(pair, x)
    side.synchronize()
    _outputs_match(pair, trees, x, outs)
    graph = torch.cuda.CUDAGraph()
    keep = {l: o.keep for l, o in outs.items()}
    with torch.cuda.graph(graph, stream=side):
        pair.ctx.draft_begin(cu_of(trees), packed(trees))
        for l, t in keep.items():
            if pair.shape.layer_kind[l] == W.ATTN:
                pair.ctx.draft_attn(l, t["q"], t["k"], t["v"], outs[l])
            else:
                pair.ctx.draft_gdn(l, t["q"], t["k"], t["v"], t["alpha"], t["beta"], outs[l])
    for l, t in keep.items():
        for m, z in y[l].items():
            t[m].copy_(_bf(z) if z.dtype == np.uint16 else torch.from_numpy(z))
        outs[l].fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    _outputs_match(pair, trees, y, outs)
    path = O.draft_path(trees[0], 24)
    pair.ctx.draft_commit([0, len(path), len(path)], path)
    _advance_oracle(pair, trees, [path, []], y)
    _compare_states(pair)
    del ref


def test_a_character_behind_a_long_slab():
    """Cache offsets past 2^31 elements: the second character's slots lie behind 2.2M slots of the first, in the second of two
    layers."""
    import torch
    from harness import rel_l2
    from paper_2609_18935_gb300 import kvm
    first = 2_200_000
    assert 2 * (first + 256) * 256 > 2 ** 30 and 4 * (first + 256) * 256 > 2 ** 31
    ctx = kvm.Context([kvm.LAYER_ATTN, kvm.LAYER_ATTN], 8, 2, 256, 64, THETA, 8, 64, 64, [first, 200], 64)
    ctx.draft_reserve(32)
    live, n = 70, 20
    t = tree("comb", n)
    path = O.draft_path(t, 18)
    cache, x = {}, {}
    ctx.load_prefix(1, live, live, np.arange(live, dtype=np.int32))
    ctx.draft_begin([0, 0, n], t)
    for l in range(2):
        cache[l] = (W.normal_bf16((161, l, 1), (2, live, 256), unit_last=True), W.normal_bf16((161, l, 2), (2, live, 256)))
        x[l] = (W.normal_bf16((161, l, 3), (n, 8, 256)), W.normal_bf16((161, l, 4), (n, 2, 256), unit_last=True),
                W.normal_bf16((161, l, 5), (n, 2, 256)))
        ctx.set_kv(l, 1, _bf(cache[l][0]), _bf(cache[l][1]))
    ctx.draft_begin([0, 0, n], t)
    for l in range(2):
        q, k, v = (_bf(y) for y in x[l])
        out = torch.empty_like(q)
        ctx.draft_attn(l, q, k, v, out)
        c = O.AttnCache(*(O.bf16_to_f64(y) for y in cache[l]), np.arange(live))
        assert rel_l2(_f64(out), O.draft_attention(c, *(O.bf16_to_f64(y) for y in x[l]), t, live, 64, THETA)) <= 5e-3
    ctx.draft_commit([0, 0, len(path)], path)
    ctx.check()
    for l in range(2):
        k, v = (_f64(y) for y in ctx.get_kv(l, 1))
        assert np.array_equal(v[:, :live], O.bf16_to_f64(cache[l][1])) and np.array_equal(k[:, :live], O.bf16_to_f64(cache[l][0]))
        assert np.array_equal(v[:, live:], O.bf16_to_f64(x[l][2])[path].transpose(1, 0, 2))
        rot = O.rope(O.bf16_to_f64(x[l][1])[path], live + np.arange(len(path)), 64, THETA).transpose(1, 0, 2)
        assert np.all(np.abs(k[:, live:] - rot) <= 2.0 ** -8 * np.abs(rot) + 1e-6)
    assert np.array_equal(ctx.get_positions(1).cpu().numpy(), np.arange(live + len(path)))


def test_as_many_characters_as_a_context_holds():
    """256 characters of zero to four nodes, a draft that fills every cache to its last slot."""
    import torch
    r = np.random.default_rng(171)
    sizes = [int(n) for n in r.integers(0, 5, 256)]
    trees = [tree("tree", n, b) for b, n in enumerate(sizes)]
    a = Attn(4, 1, 64, 32, [64 - n for n in sizes], seed=172, extra=0)
    x = a.inputs(sum(sizes), seed=173)
    a.check(trees, x, a.run(trees, x))
    g = Gdn(1, 64, 32, 256, seed=174, conv=True)
    y = g.inputs(sum(sizes), seed=175)
    g.check(trees, y, g.run(trees, y))
    V = 40
    v = Verdict(256)
    target, draft = _rows(r, sum(sizes), V, torch.float32, near=0.4)
    v.check(trees, r.integers(0, V, sum(sizes)), target, draft, 0.5 * r.random(sum(sizes)), r.random(256))


def test_two_contexts_on_two_streams():
    """Steps of two contexts at once, on a stream each: what each computes alone, bit for bit."""
    import torch
    trees = [tree("tree", 30), tree("star", 9)]
    pairs = [_stack(True, 2, [300, 120], 181 + i) for i in range(2)]
    xs = [_step_inputs(p, 39, 183 + i) for i, p in enumerate(pairs)]
    alone = []
    for p, x in zip(pairs, xs):
        p.ctx.draft_begin(cu_of(trees), packed(trees))
        alone.append({l: o.clone() for l, o in _layers(p, x).items()})
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(5):
        outs = []
        for p, st in zip(pairs, streams):
            p.ctx.draft_begin(cu_of(trees), packed(trees), stream=st)
        for p, x, st in zip(pairs, xs, streams):
            with torch.cuda.stream(st):
                outs.append(_layers(p, x))
        torch.cuda.synchronize()
        for o, ref in zip(outs, alone):
            for l in ref:
                assert torch.equal(o[l].view(torch.int16), ref[l].view(torch.int16)), l
    for p in pairs:
        p.ctx.check()


@pytest.mark.parametrize("nodes", [(12, 5), (64, 40)])
def test_inputs_written_just_before_the_calls_that_read_them(nodes):
    """Steps enqueued one after another without a wait of the host, their trees and the same buffers' contents alternating (the
    copies right before each layer's call, which starts while they may still run): every output is that of the step alone, bit for
    bit.  Trees of one query tile and of several."""
    import torch
    pair = _stack(True, 2, [300, 77], 191)
    trees = [[tree("tree", nodes[0], i), tree("comb", nodes[1], i)] for i in range(2)]
    trees[1][0] = tree("star", nodes[0])
    xs = [_step_inputs(pair, sum(nodes), 192 + i) for i in range(2)]
    dev = [{l: {m: _bf(z) if z.dtype == np.uint16 else torch.from_numpy(z).cuda() for m, z in y.items()} for l, y in x.items()} for x in xs]
    V, r = 2000, np.random.default_rng(194)
    rows = [[z.cuda() for z in _rows(r, sum(nodes), V, torch.float32, near=0.4)] for _ in range(2)]
    n = sum(nodes)
    tok = [torch.as_tensor(r.integers(0, V, n), dtype=torch.int32).cuda() for _ in range(2)]
    u, un = torch.as_tensor(0.4 * r.random(n), dtype=torch.float32).cuda(), torch.as_tensor(r.random(2), dtype=torch.float32).cuda()
    buf = {l: {m: torch.empty_like(z) for m, z in y.items()} for l, y in dev[0].items()}
    target, draft = (torch.empty_like(z) for z in rows[0])

    def step(i):
        outs = []
        pair.ctx.draft_begin(cu_of(trees[i]), packed(trees[i]))
        for l, t in buf.items():
            for m, z in t.items():
                z.copy_(dev[i][l][m])
            if pair.shape.layer_kind[l] == W.ATTN:
                outs.append(torch.empty_like(t["q"]))
                pair.ctx.draft_attn(l, t["q"], t["k"], t["v"], outs[-1])
            else:
                outs.append(torch.empty_like(t["v"]))
                pair.ctx.draft_gdn(l, t["q"], t["k"], t["v"], t["alpha"], t["beta"], outs[-1])
        target.copy_(rows[i][0])
        draft.copy_(rows[i][1])
        path, count, nxt = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n, 2, 2))
        pair.ctx.draft_verify(tok[i], target, draft, u, un, path, count, nxt)
        return outs + [path, count, nxt]

    alone = []
    for i in range(2):
        alone.append(step(i))
        torch.cuda.synchronize()
    got = [step(k % 2) for k in range(60)]
    pair.ctx.check()
    for k, outs in enumerate(got):
        for a, b in zip(outs, alone[k % 2]):
            assert torch.equal(a, b), k


DEBUG = r"""
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import test_gpu_draft as T
T.test_steps_of_a_population(True)
T.test_deep_paths_of_wide_rows()
print("bands intact")
"""


def test_drafts_write_nothing_outside_their_buffers():
    """The canary-checking build: steps whose every check reads the bands around the context's buffers (those of the drafts
    among them)."""
    import os
    import subprocess
    import sys
    from paper_2609_18935_gb300 import build_lib
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, KVM_LIB=build_lib.build(debug=True))
    r = subprocess.run([sys.executable, "-c", DEBUG.format(root=root, tests=os.path.join(root, "tests"))], capture_output=True,
                       text=True, timeout=600, env=env)
    assert r.returncode == 0 and "bands intact" in r.stdout, r.stdout[-2000:] + r.stderr[-3000:]


# ---------------------------------------------------------------------------- refusals
def test_refusals():
    import torch
    from paper_2609_18935_gb300 import kvm
    pair = _stack(False, 2, [60, 100], 141)
    ctx = pair.ctx
    trees = [tree("tree", 6), tree("chain", 3)]
    cu, par = cu_of(trees), packed(trees)
    x = _step_inputs(pair, 9, 142)
    t = {l: {m: _bf(z) if z.dtype == np.uint16 else torch.from_numpy(z).cuda() for m, z in y.items()} for l, y in x.items()}
    oa, og = torch.empty_like(t[1]["q"]), torch.empty_like(t[0]["v"])
    attn = lambda l=1: ctx.draft_attn(l, t[1]["q"], t[1]["k"], t[1]["v"], oa)
    gdn = lambda l=0: ctx.draft_gdn(l, *(t[0][m] for m in ("q", "k", "v", "alpha", "beta")), og)

    def refused(code, f, *a, **kw):
        with pytest.raises(kvm.KvmError) as ei:
            f(*a, **kw)
        assert ei.value.code == code, ei.value
    inval, cap, uns = kvm.KVM_E_INVAL, kvm.KVM_E_CAPACITY, kvm.KVM_E_UNSUPPORTED
    before = pair.snapshot_kv()
    refused(inval, attn)                                          # no draft
    refused(inval, gdn)
    refused(inval, ctx.draft_commit, [0, 0, 0], [])
    refused(inval, ctx.draft_reserve, 0)
    refused(inval, ctx.draft_reserve, 129)                        # more than max_tail_tokens
    refused(inval, ctx.draft_begin, [0, 2, 2], [-1, 1])
    refused(uns, ctx.draft_begin, [0, 65, 65], [-1] * 65)
    with pytest.raises(ValueError):
        ctx.draft_begin([0, 2, 2], [-1])
    with pytest.raises(ValueError):
        ctx.draft_begin([0, 2], [-1, 0])
    small = _stack(False, 1, [200], 143)
    small.ctx.draft_begin([0, 64], [-1] * 64)
    tight = kvm.Context([kvm.LAYER_ATTN], 4, 2, 64, 64, THETA, 8, 64, 64, [64], 64)
    refused(cap, tight.draft_begin, [0, 1], [-1])                 # nothing reserved
    tight.draft_reserve(8)
    refused(cap, tight.draft_begin, [0, 9], [-1] * 9)
    tight.load_prefix(0, 60, 60, np.arange(60))
    refused(cap, tight.draft_begin, [0, 5], [-1] * 5)             # past the character's capacity
    tight.draft_begin([0, 4], [-1] * 4)
    ctx.draft_begin(cu, par)
    refused(inval, attn, 0)                                       # a delta-rule layer
    refused(inval, gdn, 1)
    refused(inval, attn, 7)
    with pytest.raises(ValueError):                               # a tensor of another draft's size
        ctx.draft_attn(1, t[1]["q"][:8], t[1]["k"], t[1]["v"], oa)
    with pytest.raises(ValueError):
        ctx.draft_attn(1, t[1]["q"].transpose(0, 1).contiguous().transpose(0, 1), t[1]["k"], t[1]["v"], oa)
    with pytest.raises(ValueError):
        ctx.draft_gdn(0, t[0]["q"].cpu(), *(t[0][m] for m in ("k", "v", "alpha", "beta")), og)
    with pytest.raises(ValueError):
        ctx.draft_gdn(0, t[0]["q"].half(), *(t[0][m] for m in ("k", "v", "alpha", "beta")), og)
    refused(inval, ctx.draft_attn, 1, t[1]["q"], t[1]["k"], t[1]["v"], t[1]["q"])       # out over an input
    refused(inval, ctx.draft_gdn, 0, *(t[0][m] for m in ("q", "k", "v", "alpha", "beta")), t[0]["v"])
    flat = torch.empty(t[1]["q"].numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(t[1]["q"].shape)
    refused(inval, ctx.draft_attn, 1, flat, t[1]["k"], t[1]["v"], oa)                   # off the 16-byte grid
    gdn(0), gdn(2), attn(1)
    refused(inval, ctx.draft_commit, [0, 1, 1], [0])              # layer 3 has not run
    ctx.draft_attn(3, t[1]["q"], t[1]["k"], t[1]["v"], oa)
    refused(inval, ctx.draft_commit, [0, 1, 2], [1, 0])           # not from a root
    refused(inval, ctx.draft_commit, [0, 0, 4], [0, 1, 2, 2])
    forest = [[-1, -1], [-1]]
    ctx.draft_begin(cu_of(forest), packed(forest))
    row = lambda n: torch.full((n, 8), 0.125, device="cuda")
    i = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    f = lambda n: torch.zeros(n, device="cuda")
    refused(inval, ctx.draft_verify, i(3), row(3), row(3), f(3), f(2), i(3), i(2), i(2))   # several roots
    with pytest.raises(ValueError):
        ctx.draft_verify(i(3), row(3), row(3).bfloat16(), f(3), f(2), i(3), i(2), i(2))
    with pytest.raises(ValueError):
        ctx.draft_verify(i(3), row(3), row(3)[:, :7], f(3), f(2), i(3), i(2), i(2))
    # every call that changes caches, states or lengths ends the draft
    fork = _stack(False, 2, [60, 100], 141)
    q, k, v = t[1]["q"][:1].contiguous(), t[1]["k"][:1].contiguous(), t[1]["v"][:1].contiguous()
    one = [0, 1, 1]
    K, V = ctx.get_kv(1, 0)
    enders = [lambda: ctx.load_prefix(0, 60, 60, np.arange(60)), lambda: ctx.set_kv(1, 0, K, V),
              lambda: ctx.set_state(0, ctx.get_state(0)), lambda: ctx.kv_compact([0, 0, 0], [], []),
              lambda: ctx.tail_attn_prefill(1, one, q, k, v, torch.empty_like(q)),
              lambda: ctx.rerotate_keys(0, 0, 1, [0]), lambda: ctx.advance([0, 0, 0]), lambda: ctx.fork_from(fork.ctx),
              lambda: ctx.draft_commit([0, 0, 0], [])]
    for end in enders:
        ctx.draft_begin(cu, par)
        end()
        refused(inval, attn)
    ctx.check()
    for key, val in pair.snapshot_kv().items():
        for u, w in zip(before[key], val):
            assert np.array_equal(u, w), key


def test_an_allocation_that_failed_is_reported_once():
    """Room that the device does not have (8 TB a cache) is refused; the next calls of another context do not report it again."""
    from paper_2609_18935_gb300 import kvm
    a = Attn(4, 2, 64, 64, [70], seed=155)
    x = a.inputs(5, seed=156)
    for _ in range(2):
        with pytest.raises(kvm.KvmError) as ei:
            kvm.Context([kvm.LAYER_ATTN] * 4, 8, 2, 256, 64, THETA, 8, 64, 64, [2_000_000_000], 64)
        assert ei.value.code == kvm.KVM_E_CUDA
        a.check([tree("tree", 5)], x, a.run([tree("tree", 5)], x))


def test_a_context_without_drafts_or_attention():
    """An empty draft commits nothing; a stack of delta-rule layers alone drafts too; room can grow."""
    import torch
    g = Gdn(2, 64, 32, 2, seed=151)
    g.ctx.draft_begin([0, 0, 0], [])
    g.ctx.draft_commit([0, 0, 0], [])
    assert g.ctx.get_live(0) == (0, 0)
    from paper_2609_18935_gb300 import kvm
    ctx = kvm.Context([kvm.LAYER_GDN], 8, 2, 64, 64, THETA, 2, 64, 32, [64], 64)
    ctx.set_state(0, torch.from_numpy(g.S[:1]).cuda())
    for room in (2, 64):
        ctx.draft_reserve(room)
        t = tree("tree", room)
        x = g.inputs(room, seed=152)
        q, k, v, al, be = g.tensors(x)
        out = torch.empty_like(v)
        ctx.draft_begin([0, room], t)
        ctx.draft_gdn(0, q, k, v, al, be, out)
        one = Gdn(2, 64, 32, 1, seed=151)
        one.S = g.S[:1]
        one.check([t], x, out)
    ctx.check()
