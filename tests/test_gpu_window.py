"""Attention layers with a sliding window and sinks (kvm_set_window) on the GPU against 64 bits, element by element within
the bounds of attn64: tails, one-token rounds, drafts, whole rounds and the probe."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_18935_gb300 import kvm
    kvm.load_library()


HYBRID, MID, SMALL = (16, 2, 256, 64), (16, 4, 128, 128), (8, 2, 64, 64)


def _normal(g, *shape, unit=False):
    import torch
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float64)
    return (x / x.norm(dim=-1, keepdim=True) if unit else x).bfloat16()


class Pop:
    """Attention layers of one population with random caches; keys and values in 64 bits beside them, [layer][character]."""

    def __init__(self, shape, lives, seed, windows=((0, 0),), extra=64, most=None, cursor=0):
        import torch
        from paper_2609_18935_gb300 import kvm
        self.hq, self.hkv, self.d, self.rot = shape
        self.lives, self.windows = list(lives), list(windows)
        self.cap = [l + extra for l in lives]
        self.new = lambda: kvm.Context([kvm.LAYER_ATTN] * len(windows), *shape, 1.0e4, 8, 64, 64, self.cap, most or extra * len(lives))
        self.ctx = self.new()
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.pos = [torch.arange(l, device="cuda") + cursor for l in lives]
        self.cursor = [l + cursor for l in lives]
        self.K, self.V = [], []
        for b, l in enumerate(lives):
            self.ctx.load_prefix(b, l, l + cursor, np.arange(l, dtype=np.int32) + cursor)
        for i, (w, s) in enumerate(windows):
            if w:
                self.ctx.set_window(i, w, s)
            ks = [_normal(self.g, self.hkv, l, self.d, unit=True) for l in lives]
            vs = [_normal(self.g, self.hkv, l, self.d) for l in lives]
            for b, l in enumerate(lives):
                if l:
                    self.ctx.set_kv(i, b, ks[b], vs[b])
            self.K.append([x.double() for x in ks])
            self.V.append([x.double() for x in vs])

    def tail(self, n, scale=1.0):
        return (_normal(self.g, n, self.hq, self.d) * scale, _normal(self.g, n, self.hkv, self.d, unit=True),
                _normal(self.g, n, self.hkv, self.d))

    def want(self, layer, tails, x, tail_pos=None, keep=False):
        """(outputs, bounds) of a tail, packed; with keep it becomes live in the copies."""
        import torch
        from attn64 import attend, in_sight, rope
        q, k, v = (t.double() for t in x)
        outs, offs, at = [], [], 0
        for b, m in enumerate(tails):
            if not m:
                continue
            sl = slice(at, at + m)
            L = self.K[layer][b].shape[1]
            pos = torch.as_tensor(tail_pos[sl]) if tail_pos is not None else self.cursor[b] + torch.arange(m)
            K = torch.cat([self.K[layer][b], rope(k[sl], pos, self.rot).transpose(0, 1)], 1)
            V = torch.cat([self.V[layer][b], v[sl].transpose(0, 1)], 1)
            seen = in_sight(np.arange(L, L + m), L + m, *self.windows[layer])
            o, e = attend(rope(q[sl], pos, self.rot), K, V, seen)
            outs.append(o)
            offs.append(e)
            if keep:
                self.K[layer][b], self.V[layer][b] = K, V
            at += m
        return torch.cat(outs), torch.cat(offs)

    def check(self, layer, tails, x, out, what="", most=5e-3, **kw):
        """`most`: for scores of size 1 and below, where the weights' and the output's roundings count: each at most
        2^-8 / sqrt(3) of the values in the root mean square, together 3.2e-3."""
        from attn64 import inside
        rel = inside(out, *self.want(layer, tails, x, **kw), what)
        assert rel < most, (what, rel)


def _cu(tails):
    return np.concatenate([[0], np.cumsum(tails)]).astype(np.int32)


def _run(p, layer, tails, x, **kw):
    import torch
    out = torch.full_like(x[0], float("nan"))
    p.ctx.tail_attn_prefill(layer, _cu(tails), *x, out, **kw)
    p.ctx.check()
    return out


@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL, (8, 8, 128, 64), (64, 1, 64, 6), (16, 1, 256, 0)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (63, 0), (64, 64), (65, 1), (200, 4), (1000, 130), (5000, 2), (7, 4000)])
def test_tails(shape, window, sinks):
    lives, tails = [500, 0, 63, 1300, 64], [70, 5, 1, 33, 0]
    p = Pop(shape, lives, 11 + window, [(window, sinks)], extra=128)
    x = p.tail(sum(tails))
    p.check(0, tails, x, _run(p, 0, tails, x), (shape, window, sinks))


@pytest.mark.parametrize("shape", [HYBRID, SMALL])
@pytest.mark.parametrize("lives,tails", [([4000], [1]), ([0], [1]), ([1], [1]), ([4000] * 9, [1] * 9), ([0], [700]), ([9000], [300])])
@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 4), (1024, 100)])
def test_lengths(shape, lives, tails, window, sinks):
    p = Pop(shape, lives, 5, [(window, sinks)], extra=max(tails) + 1, most=sum(tails))
    x = p.tail(sum(tails))
    p.check(0, tails, x, _run(p, 0, tails, x), (shape, lives, tails, window, sinks))


@pytest.mark.parametrize("window,sinks", [(300, 0), (301, 5)])
def test_whole_tiles_dealt_in_waves(window, sinks):
    from paper_2609_18935_gb300 import kvm
    tails = [1400, 900, 0, 1200]
    p = Pop(HYBRID, [100, 2000, 10, 0], 8, [(window, sinks)], extra=1400, most=sum(tails))
    assert kvm.plan_attention_window(p.lives, _cu(tails), 16, 2, window, sinks, 152)["n_waves"] > 1
    x = p.tail(sum(tails))
    p.check(0, tails, x, _run(p, 0, tails, x))


def test_scores_far_apart():
    """Rows whose newest keys weigh nothing beside a sink, and the other way round."""
    import torch
    p = Pop(SMALL, [800], 9, [(100, 3)], extra=64)
    x = p.tail(40, scale=64.0)
    # a score is q . k / 8 with |q| = 64 sqrt(64), |k| = 1: the rounding of q, at most 2^-8 / sqrt(3) a dim in the root mean square,
    # moves it by 64 * 2^-8 / sqrt(3) / 8 = 0.018, that of k as much again, weights by the factor e^0.026
    p.check(0, [40], x, _run(p, 0, [40], x), most=2.7e-2)


@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL])
def test_a_window_over_everything_changes_no_bit(shape):
    import torch
    outs = []
    for w in [(0, 0), (2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2, 2 ** 31 - 1)]:
        p = Pop(shape, [3000, 17], 10, [w], extra=200, most=300)
        outs.append(_run(p, 0, [200, 9], p.tail(209)))
    assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_positions_of_their_own_and_far_ones():
    """The window counts live entries, whatever their ids."""
    p = Pop(HYBRID, [700, 50], 12, [(90, 4)], extra=64, cursor=10 ** 9)
    tails = [30, 20]
    x = p.tail(50)
    pos = np.concatenate([np.arange(5, 35), 7 * np.arange(20)]).astype(np.int32)
    p.check(0, tails, x, _run(p, 0, tails, x, tail_pos=pos), tail_pos=pos)
    p.check(0, tails, x, _run(p, 0, tails, x))


def _rounds(p, steps, via_graph=False):
    """Rounds over all layers: spans removed, tails kept, outputs checked after each."""
    import torch
    for n, (spans, tails) in enumerate(steps):
        flat = [s for t in spans for s in t]
        cu, sb, se = _cu([len(t) for t in spans]), [a for a, _ in flat], [b for _, b in flat]
        xs = [p.tail(sum(tails)) for _ in p.windows]
        outs = {i: torch.full_like(x[0], float("nan")) for i, x in enumerate(xs)}
        p.ctx.update_round(cu, sb, se, _cu(tails), {i: dict(zip("qkv", x)) for i, x in enumerate(xs)}, outs)
        p.ctx.check()
        for b, t in enumerate(spans):
            for i in range(len(p.windows)):
                L = p.K[i][b].shape[1]
                keep = [j for j in range(L) if not any(a <= j < e for a, e in t)]
                p.K[i][b], p.V[i][b] = p.K[i][b][:, keep], p.V[i][b][:, keep]
        for i, x in enumerate(xs):
            p.check(i, tails, x, outs[i], (n, i), keep=True)
        for b, m in enumerate(tails):
            p.cursor[b] += m
            assert p.ctx.get_live(b) == (p.K[0][b].shape[1], p.cursor[b])


def test_rounds_and_one_token_rounds():
    """Removals move entries into the sinks' and the window's sight; one token after another slides it."""
    p = Pop(MID, [900, 130, 3], 13, [(0, 0), (128, 4), (100, 0), (1, 70)], extra=256, most=256)
    steps = [([[(0, 2), (800, 850)], [(5, 60)], []], [60, 1, 2]), ([[(10, 500)], [], [(0, 3)]], [1, 1, 1])]
    steps += [([[], [], []], [1, 1, 1])] * 4 + [([[], [(0, 1)], []], [0, 100, 1])]
    _rounds(p, steps)


def test_fork_copies_windows():
    import torch
    p = Pop(SMALL, [600, 20], 14, [(50, 4), (0, 0)], extra=64)
    other = p.new()
    other.set_window(1, 8)
    other.fork_from(p.ctx)
    p.ctx = other
    for i in range(2):
        x = p.tail(40)
        p.check(i, [33, 7], x, _run(p, i, [33, 7], x), i)


def test_a_window_that_changes_between_calls():
    p = Pop(SMALL, [600], 15, [(0, 0)], extra=64)
    x = p.tail(9)
    for w in [(64, 0), (0, 0), (3, 1), (300, 64)]:
        p.ctx.set_window(0, *w)
        p.windows[0] = w
        p.check(0, [9], x, _run(p, 0, [9], x), w)


# ---------------------------------------------------------------------------- drafts
def _tree(kind, n, seed=0):
    r = np.random.default_rng([seed, n])
    if kind == "chain":
        return list(range(-1, n - 1))
    if kind == "roots":
        return [-1] * n
    return [-1 if i == 0 else int(r.integers(max(0, i - 6), i)) for i in range(n)]


def _draft(p, layer, trees, x):
    """(outputs, wanted, bounds)."""
    import torch
    from attn64 import attend, in_sight, rope
    out = torch.full_like(x[0], float("nan"))
    p.ctx.draft_attn(layer, *x, out)
    p.ctx.check()
    q, k, v = (t.double() for t in x)
    outs, offs, at = [], [], 0
    for b, t in enumerate(trees):
        n = len(t)
        if not n:
            continue
        anc = np.eye(n, dtype=bool)
        for i, up in enumerate(t):
            if up >= 0:
                anc[i] |= anc[up]
        depth = anc.sum(1) - 1
        sl, L = slice(at, at + n), p.K[layer][b].shape[1]
        pos = p.cursor[b] + torch.as_tensor(depth)
        K = torch.cat([p.K[layer][b], rope(k[sl], pos, p.rot).transpose(0, 1)], 1)
        V = torch.cat([p.V[layer][b], v[sl].transpose(0, 1)], 1)
        live = in_sight(L + depth, L, *p.windows[layer])
        o, e = attend(rope(q[sl], pos, p.rot), K, V, torch.cat([live, torch.as_tensor(anc).cuda()], 1))
        outs.append(o)
        offs.append(e)
        at += n
    return out, torch.cat(outs), torch.cat(offs)


@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL, (8, 1, 64, 6), (64, 1, 128, 64), (8, 2, 256, 48)])
@pytest.mark.parametrize("kind", ["chain", "tree", "roots"])
def test_drafts(shape, kind):
    from attn64 import inside
    windows = [(64, 0), (64, 4), (100, 130), (0, 0), (1000, 3), (2 ** 31 - 1, 0), (64, 4)]
    lives = [700, 0, 64, 1500]
    p = Pop(shape, lives, 16, windows, extra=64)
    trees = [_tree(kind, 64, 1), _tree(kind, 13, 2), [], _tree(kind, 1, 3)]
    n = sum(len(t) for t in trees)
    p.ctx.draft_reserve(n)
    p.ctx.draft_begin(_cu([len(t) for t in trees]), np.array(sum(trees, []), np.int32))
    for i in range(len(windows)):
        got, want, off = _draft(p, i, trees, p.tail(n))
        assert inside(got, want, off, (shape, kind, windows[i])) < 5e-3


def test_a_drafts_path_becomes_live_and_the_window_moves_on():
    import torch
    from attn64 import inside, rope
    p = Pop(HYBRID, [900, 70], 17, [(64, 4), (0, 0)], extra=64)
    trees, paths = [_tree("tree", 20, 4), _tree("chain", 9, 5)], [[0], [0, 1, 2, 3, 4]]
    while True:
        nxt = [i for i, up in enumerate(trees[0]) if up == paths[0][-1]]
        if not nxt:
            break
        paths[0].append(nxt[-1])
    p.ctx.draft_reserve(29)
    p.ctx.draft_begin(_cu([20, 9]), np.array(sum(trees, []), np.int32))
    xs = []
    for i in range(2):
        xs.append(p.tail(29))
        assert inside(*_draft(p, i, trees, xs[i])) < 5e-3
    p.ctx.draft_commit(_cu([len(t) for t in paths]), np.array(sum(paths, []), np.int32))
    for i, x in enumerate(xs):
        for b, t in enumerate(paths):
            rows = torch.tensor(t).cuda() + (20 if b else 0)
            pos = p.cursor[b] + torch.arange(len(t))
            p.K[i][b] = torch.cat([p.K[i][b], rope(x[1][rows].double(), pos, p.rot).transpose(0, 1)], 1)
            p.V[i][b] = torch.cat([p.V[i][b], x[2][rows].double().transpose(0, 1)], 1)
    for b, t in enumerate(paths):
        p.cursor[b] += len(t)
    _rounds(p, [([[], []], [1, 1]), ([[(0, 1)], []], [5, 0])])


def test_a_draft_as_a_chain_equals_a_tail():
    import torch
    p = Pop(SMALL, [500, 40], 18, [(64, 5)], extra=64)
    x = p.tail(40)
    tail = _run(p, 0, [33, 7], x)
    p.ctx.draft_reserve(40)
    p.ctx.draft_begin(_cu([33, 7]), np.array(_tree("chain", 33) + _tree("chain", 7), np.int32))
    got, want, off = _draft(p, 0, [_tree("chain", 33), _tree("chain", 7)], x)
    assert bool(((got.double() - tail.double()).abs() <= 2 * off).all())


# ---------------------------------------------------------------------------- probe, refusals, graphs
@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 4), (350, 0), (3, 500)])
def test_probe(window, sinks):
    import torch
    from attn64 import in_sight, rope
    p = Pop(HYBRID, [333], 19, [(window, sinks)])
    q = _normal(p.g, 7, 16, 256)
    probs, _ = p.ctx.attn_probe(0, 0, q)
    p.ctx.check()
    qr = rope(q.double(), torch.arange(326, 333), 64)
    seen = in_sight(np.arange(326, 333), 333, window, sinks)
    s = torch.stack([(qr[:, h] @ p.K[0][0][h // 8].T) / 16.0 for h in range(16)])
    want = torch.softmax(s.masked_fill(~seen, -float("inf")), -1).mean((0, 1))
    # scores in 32 bits: 256 products of unit keys with |q| ~ 16, and expf: below 1e-5 of each probability
    assert float((probs.double() - want).abs().max()) < 1e-5 * float(want.max())
    assert bool((probs[~seen.any(0)] == 0).all()) and abs(float(probs.sum()) - 1) < 1e-5


def test_refusals():
    from paper_2609_18935_gb300 import kvm
    ctx = kvm.Context([kvm.LAYER_GDN, kvm.LAYER_ATTN], *SMALL, 1.0e4, 8, 64, 64, [128], 64)
    for bad in [(0, 64, 0), (2, 64, 0), (-1, 64, 0), (1, -1, 0), (1, 64, -1), (1, 0, 4)]:
        with pytest.raises(kvm.KvmError) as e:
            ctx.set_window(*bad)
        assert e.value.code == kvm.KVM_E_INVAL, bad
    ctx.draft_reserve(4)
    ctx.set_window(1, 63)
    with pytest.raises(kvm.KvmError) as e:
        ctx.draft_begin([0, 2], [-1, 0])
    assert e.value.code == kvm.KVM_E_UNSUPPORTED
    ctx.draft_begin([0, 0], [])                    # nothing to see
    ctx.set_window(1, 64)
    ctx.draft_begin([0, 2], [-1, 0])
    ctx.set_window(1, 65)                          # ends the draft
    with pytest.raises(kvm.KvmError):
        ctx.draft_commit([0, 0], [])


def test_a_captured_step_replayed_with_new_inputs():
    import torch
    p = Pop(HYBRID, [3000, 90], 20, [(128, 4)], extra=64)
    x = [t.clone() for t in p.tail(2)]
    out = torch.empty_like(x[0])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        p.ctx.tail_attn_prefill(0, [0, 1, 2], *x, out)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            p.ctx.tail_attn_prefill(0, [0, 1, 2], *x, out)
    for _ in range(3):
        for t, y in zip(x, p.tail(2)):
            t.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        p.ctx.check()
        p.check(0, [1, 1], x, out)


# ---------------------------------------------------------------------------- few rows (a launch that appends, too)
@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL, (8, 8, 64, 64), (4, 4, 256, 256), (8, 4, 128, 6), (16, 1, 256, 0)])
def test_few_rows_are_attended_to_and_appended(shape):
    """One row of a group to 16 and the next, over one block's end and into the next, several steps: outputs, and what the
    caches and positions hold then."""
    import torch
    from attn64 import rope
    g = shape[0] // shape[1]
    for n in sorted({1, max(1, 8 // g), 8 // g + 1, max(1, 16 // g), 16 // g + 1}):
        lives = [64 - n, 63, 64, 127, 1300, 0]
        p = Pop(shape, lives, 40 + n, [(1, 0), (70, 3), (2 ** 31 - 1, 0)], extra=4 * n, most=6 * n)
        for step in range(3):
            tails = [n, n, max(n - 1, 0), n, n, 1]
            xs = [p.tail(sum(tails)) for _ in p.windows]
            for i, x in enumerate(xs):
                p.check(i, tails, x, _run(p, i, tails, x), (shape, n, step, i), keep=True)
            p.ctx.advance(_cu(tails))
            for b, m in enumerate(tails):
                p.pos[b] = torch.cat([p.pos[b], p.cursor[b] + torch.arange(m, device="cuda")])
                p.cursor[b] += m
        for b in range(len(lives)):
            assert torch.equal(p.ctx.get_positions(b).long(), p.pos[b])
            for i in range(len(p.windows)):
                k, v = p.ctx.get_kv(i, b)
                assert torch.equal(v.double(), p.V[i][b])
                # rounded once after a rotation in 32 bits (2^-20 of the pair's numbers at most, see test_gpu_kv8.holds)
                off = 2.0 ** -8 * p.K[i][b].abs() + 2.0 ** -19 * p.K[i][b].abs().amax() if k.numel() else p.K[i][b]
                assert bool(((k.double() - p.K[i][b]).abs() <= off).all())


def test_few_rows_dealt_and_split():
    """256 characters' step in waves of whole tiles, and one long one's over many blocks."""
    r = np.random.default_rng(3)
    p = Pop((8, 4, 64, 64), [int(x) for x in r.integers(0, 700, 255)] + [9000], 41, [(300, 4), (5000, 0)], extra=2, most=256)
    for _ in range(2):
        tails = [int(x) for x in r.integers(0, 2, 255)] + [1]
        for i in range(2):
            x = p.tail(sum(tails))
            p.check(i, tails, x, _run(p, i, tails, x), i)


def test_a_query_that_is_not_finite_stays_with_its_row():
    import torch
    for window in (64, 3000):
        p = Pop(SMALL, [4000], 42, [(window, 0)])
        x = p.tail(2)
        x[0][1, 3, 5] = float("nan")
        out = _run(p, 0, [2], x)
        assert torch.isnan(out[1, 3]).all()
        out[1, 3] = 0
        assert torch.isfinite(out).all()
