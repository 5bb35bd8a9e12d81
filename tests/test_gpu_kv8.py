"""Caches in 8 bits (kvm_create_kv8) on the GPU: what they hold against the definition in 64 bits, number by number, and the
attention over them within the bounds of attn64."""
import ctypes as C

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
BLOCK = 64


def _normal(g, *shape, unit=False):
    import torch
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float64)
    return (x / x.norm(dim=-1, keepdim=True) if unit else x).bfloat16()


def _exponent(x):
    """Of each block of x [heads][rows][d] in 64 bits, from its first row on: [heads][blocks]."""
    import torch
    out = []
    for lo in range(0, x.shape[1], BLOCK):
        m, e = torch.frexp(x[:, lo:lo + BLOCK].abs().amax((1, 2)))
        out.append((e - 9 + (m > 0.875)).clamp(-117, 119))
    return torch.stack(out, 1) if out else torch.zeros(x.shape[0], 0, dtype=torch.int64, device=x.device)


def _pow2(e):
    """2^e in 64 bits, from its bits: pow and log2 of the GPU are not exact there."""
    import torch
    return ((e.long() + 1023) << 52).view(torch.float64)


def _steps(x, e):
    """The grid around x under the scales 2^e [heads][blocks]: the distance of the numbers next to it."""
    import torch
    s = _pow2(e).repeat_interleave(BLOCK, 1)[:, :x.shape[1], None]
    return s, s * _pow2(torch.frexp((x / s).abs().clamp(min=2.0 ** -6, max=448.0))[1] - 4)


def held(x):
    """x [heads][rows][d] in 64 bits as blocks from its first row on hold it."""
    import torch
    s, step = _steps(x, _exponent(x))
    return torch.minimum(torch.maximum(torch.round(x / step) * step, -448 * s), 448 * s)


def holds(got, x, what="", far=0):
    """got is x rounded, where x may be off: each number next to it or, at a border, the other one; a block's scale too.
    A rotation in 32 bits: the angle in half turns 2^-25 of them, 2^-23.3, the sine and cosine two units, 2^-23, each times
    two numbers; three roundings of up to sqrt 2 times the largest: 2^-20.6 of the largest.  At position `far` the product
    with a frequency in 64 bits, here and there: 2^-51 far."""
    import torch
    got, u = got.double(), 2.0 ** -20 + far * 2.0 ** -51
    slack = u * x.abs().amax((1, 2), keepdim=True) if x.numel() else x
    ok = torch.zeros_like(x, dtype=torch.bool)
    for k in (_exponent(x * (1 - u)), _exponent(x), _exponent(x * (1 + u))):
        s, step = _steps(x.abs() + slack, k)
        ok |= (got - x).abs() <= step / 2 + slack
    assert bool(ok.all()), (what, int((~ok).sum()), got[~ok][:4].tolist(), x[~ok][:4].tolist())


class Pop:
    """Attention layers in 8 bits; what their caches hold in 64 bits beside them, [layer][character] of [heads][rows][d]."""

    def __init__(self, shape, lives, seed, windows=((0, 0),), extra=64, most=None, cursor=0, kinds=None, size=1.0):
        import torch
        from paper_2609_18935_gb300 import kvm
        self.hq, self.hkv, self.d, self.rot = shape
        self.lives, self.windows = list(lives), list(windows)
        self.cap = [l + extra for l in lives]
        self.kinds = kinds or [kvm.LAYER_ATTN] * len(windows)
        self.at = [i for i, k in enumerate(self.kinds) if k == kvm.LAYER_ATTN]      # attention layers' places
        self.new = lambda: kvm.Context(self.kinds, *shape, 1.0e4, 8, 64, 64, self.cap, most or extra * len(lives), kv_bits=8)
        self.ctx = self.new()
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.cursor = [l + cursor for l in lives]
        self.K, self.V = [], []
        for b, l in enumerate(lives):
            self.ctx.load_prefix(b, l, l + cursor, np.arange(l, dtype=np.int32) + cursor)
        for i, (w, s) in enumerate(windows):
            if w:
                self.ctx.set_window(self.at[i], w, s)
            self.K.append([])
            self.V.append([])
            for b, l in enumerate(lives):
                k, v = _normal(self.g, self.hkv, l, self.d, unit=True), _normal(self.g, self.hkv, l, self.d) * size
                if l:
                    self.ctx.set_kv(self.at[i], b, k, v)
                self.K[i].append(held(k.double()))
                self.V[i].append(held(v.double()))
        self.same()

    def same(self, what=""):
        """The caches hold what the copies say, exactly."""
        import torch
        for i, l in enumerate(self.at):
            for b in range(len(self.lives)):
                for got, x in zip(self.ctx.get_kv(l, b), (self.K[i][b], self.V[i][b])):
                    assert torch.equal(got.double(), x), (what, i, b)
        self.ctx.check()

    def tail(self, n, scale=1.0, size=1.0):
        return (_normal(self.g, n, self.hq, self.d) * scale, _normal(self.g, n, self.hkv, self.d, unit=True),
                _normal(self.g, n, self.hkv, self.d) * size)

    def tail_done(self, i, tails, x, out, pos=None, most=4e-3, what=""):
        """After layer i's tail: its entries and the blocks they are in hold what they should, and `out` is the attention over
        what they hold.  The caches are read out over the appended rows too, so the rows must be live by now (advance).
        `most`: the weights' rounding and the output's, each at most 2^-8 / sqrt(3) in the root mean square, 3.2e-3 together, and
        a score's rounded query moves it little at scores of size 1."""
        import torch
        from attn64 import attend, in_sight, inside, rope
        q, k, v = (t.double() for t in x)
        want, off, at = [], [], 0
        for b, m in enumerate(tails):
            L = self.K[i][b].shape[1]
            sl = slice(at, at + m)
            p = torch.as_tensor(pos[sl]) if pos is not None else self.cursor[b] - m + torch.arange(m)
            got = self.ctx.get_kv(self.at[i], b)
            for mine, new, kv in ((self.K, rope(k[sl], p, self.rot), got[0]), (self.V, v[sl], got[1])):
                exact = torch.cat([mine[i][b], new.transpose(0, 1)], 1)
                lo = L // BLOCK * BLOCK if m else L
                assert torch.equal(kv[:, :lo].double(), exact[:, :lo]), (what, i, b)
                holds(kv[:, lo:], exact[:, lo:], (what, i, b), float(p.max()) if m else 0)
                mine[i][b] = kv.double()
            if m:
                seen = in_sight(np.arange(L, L + m), L + m, *self.windows[i])
                o, e = attend(rope(q[sl], p, self.rot), self.K[i][b], self.V[i][b], seen, rounded=1)
                want.append(o)
                off.append(e)
            at += m
        if want:
            rel = inside(out, torch.cat(want), torch.cat(off), what)
            assert rel < most, (what, rel)


def _cu(tails):
    return np.concatenate([[0], np.cumsum(tails)]).astype(np.int32)


def _tail(p, tails, xs=None, pos=None, what="", **kw):
    """A tail over all layers, kept and checked."""
    import torch
    xs = xs or [p.tail(sum(tails)) for _ in p.windows]
    outs = [torch.full_like(x[0], float("nan")) for x in xs]
    for i, x in enumerate(xs):
        p.ctx.tail_attn_prefill(p.at[i], _cu(tails), *x, outs[i], **({} if pos is None else {"tail_pos": pos}))
    p.ctx.check()
    p.ctx.advance(_cu(tails), **({} if pos is None else {"tail_pos": pos}))
    for b, m in enumerate(tails):
        p.cursor[b] = p.ctx.get_live(b)[1]
    for i, x in enumerate(xs):
        p.tail_done(i, tails, x, outs[i], pos, what=what, **kw)


# ---------------------------------------------------------------------------- what the blocks hold
@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL, (8, 8, 128, 64), (64, 1, 64, 6)])
def test_set_and_get(shape):
    Pop(shape, [500, 0, 63, 64, 65, 1], 1)


def test_every_size_of_number():
    """Blocks of zeros, of one number, of numbers 2^30 apart, the smallest and the largest of bf16, ties."""
    import torch
    p = Pop(SMALL, [64 * 12 + 5], 2)
    x = _normal(p.g, 2, 64 * 12 + 5, 64).float()
    blk = x[:, :768].view(2, 12, 64, 64)
    blk[:, 0] = 0
    blk[:, 1] = 0
    blk[:, 1, 5, 7] = -448.0
    blk[:, 2] *= torch.pow(2.0, torch.randint(-30, 31, (2, 64, 64), generator=p.g, device="cuda").float())
    blk[:, 3] = 2.0 ** -126 * torch.randint(-64, 65, (2, 64, 64), generator=p.g, device="cuda").float() / 64    # bf16's subnormal numbers
    blk[:, 4] *= 2.0 ** -120
    blk[:, 5] = torch.randint(-255, 256, (2, 64, 64), generator=p.g, device="cuda").float()       # most on ties of the grid
    blk[:, 5, 0, 0] = 256.0
    blk[:, 6] = 3.3895313892515355e38                                     # the largest number
    blk[:, 7] = 449.0                                                     # above 448 by less than the grid: 450 in bf16
    blk[:, 8] = 2.0 ** 127 * (1 + torch.rand(2, 64, 64, generator=p.g, device="cuda"))
    blk[:, 9] = 0.875 * 2.0 ** torch.arange(-31, 33, device="cuda").float()[:, None]
    blk[:, 10] = 2.0 ** -9 * torch.randint(-8, 9, (2, 64, 64), generator=p.g, device="cuda").float() / 2
    blk[:, 10, 0, 0] = 448.0
    x = x.bfloat16()
    x[~torch.isfinite(x)] = 0
    p.ctx.set_kv(0, 0, x, -x)
    p.K[0][0], p.V[0][0] = held(x.double()), held(-x.double())
    p.same()
    assert float(p.K[0][0].abs().max()) == 448.0 * 2.0 ** 119
    # a number of the cache goes in again as it is, in a block of the same rows
    k, v = p.ctx.get_kv(0, 0)
    p.ctx.set_kv(0, 0, k, v)
    p.same()


def test_what_is_not_finite_is_stored_as_zero_and_reported():
    import torch
    from paper_2609_18935_gb300 import kvm
    p = Pop(SMALL, [100], 3)
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), float("nan")], device="cuda").bfloat16()
    k, v = _normal(p.g, 2, 100, 64, unit=True), _normal(p.g, 2, 100, 64)
    v[1, 3, :4] = bad
    p.ctx.set_kv(0, 0, k, v)
    with pytest.raises(kvm.KvmError) as e:
        p.ctx.check()
    assert e.value.code == kvm.KVM_E_DEVICE and "not-finite" in str(e.value)
    v[1, 3, :4] = 0
    p.K[0][0], p.V[0][0] = held(k.double()), held(v.double())
    p.same()
    # a tail's
    x = p.tail(20)
    for t in x[1:]:
        t[2, 1, 30:34] = bad
    out = torch.empty_like(x[0])
    p.ctx.tail_attn_prefill(0, [0, 20], *x, out)
    with pytest.raises(kvm.KvmError) as e:
        p.ctx.check()
    assert e.value.code == kvm.KVM_E_DEVICE
    for t in x[1:]:
        t[2, 1, 30:34] = 0
    p.ctx.advance([0, 20])
    p.cursor[0] += 20
    p.tail_done(0, [20], x, out)


def test_a_query_that_is_not_finite_stays_with_its_row():
    import torch
    for n in (2, 40):
        p = Pop(SMALL, [300], 4)
        x = p.tail(n)
        x[0][1, 3, 5] = float("nan")
        out = torch.empty_like(x[0])
        p.ctx.tail_attn_prefill(0, [0, n], *x, out)
        assert torch.isnan(out[1, 3]).all()
        out[1, 3] = 0
        assert torch.isfinite(out).all()


def test_memory_that_no_kernel_reaches():
    """Host memory, and buffers off the 16-byte grid, in both directions."""
    import torch
    from paper_2609_18935_gb300 import kvm
    p = Pop(MID, [130, 70], 5)
    for b, host in ((0, False), (1, True)):
        n = p.hkv * p.lives[b] * p.d
        k, v = _normal(p.g, p.hkv, p.lives[b], p.d), _normal(p.g, p.hkv, p.lives[b], p.d)
        if host:
            buf = [torch.empty(n, dtype=torch.bfloat16).pin_memory() for _ in range(2)]
        else:
            buf = [torch.empty(n + 8, dtype=torch.bfloat16, device="cuda")[1:n + 1] for _ in range(2)]
        for t, y in zip(buf, (k, v)):
            t.copy_(y.flatten())
        torch.cuda.synchronize()
        ptr = [C.c_void_p(t.data_ptr()) for t in buf]
        assert kvm._lib.kvm_set_kv(p.ctx._h, 0, b, *ptr, None) == 0
        torch.cuda.synchronize()
        p.K[0][b], p.V[0][b] = held(k.double()), held(v.double())
        for t in buf:
            t.zero_()
        torch.cuda.synchronize()
        assert kvm._lib.kvm_get_kv(p.ctx._h, 0, b, *ptr, None) == 0
        torch.cuda.synchronize()
        for t, want in zip(buf, (p.K[0][b], p.V[0][b])):
            assert torch.equal(t.cuda().double(), want.flatten())
    p.same()


# ---------------------------------------------------------------------------- tails
@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL, (8, 8, 128, 64), (64, 1, 64, 6), (16, 1, 256, 0), (4, 4, 256, 256), (8, 2, 128, 24)])
@pytest.mark.parametrize("lives,tails", [([500, 0, 63, 1300, 64], [70, 5, 1, 33, 0]), ([500, 0, 63, 1300, 64, 1, 127], [1] * 7), ([0], [1]), ([0], [700]),
                                         ([4000, 10], [2, 1]), ([9000], [1]), ([3000] * 9, [1, 0, 1, 1, 1, 1, 1, 1, 1])])
def test_tails(shape, lives, tails):
    p = Pop(shape, lives, 11, extra=max(tails) + 3, most=sum(tails) + 1)
    _tail(p, tails)
    _tail(p, [min(t, 1) for t in tails])


@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (63, 0), (64, 64), (65, 1), (1000, 130), (5000, 2), (7, 4000), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_windows(shape, window, sinks):
    lives, tails = [2500, 0, 63, 1300, 64], [70, 5, 1, 33, 0]
    p = Pop(shape, lives, 12, [(window, sinks), (0, 0)], extra=128)
    _tail(p, tails)
    _tail(p, [1, 1, 1, 0, 1])


@pytest.mark.parametrize("shape", [HYBRID, MID, SMALL, (8, 8, 64, 64)])
def test_rows_around_the_direct_kernels_limit(shape):
    """One row of a group to 16, and the next: both forms give the same within their bounds."""
    g = shape[0] // shape[1]
    for n in sorted({1, 7 // g + 1, 8 // g, 9 // g + 1, 16 // g, 16 // g + 1}):
        p = Pop(shape, [777, 64], 13, [(0, 0), (100, 3)], extra=64)
        _tail(p, [n, max(n - 1, 0)], what=n)


@pytest.mark.parametrize("shape,n", [((8, 8, 64, 64), 16), ((4, 4, 256, 256), 13), ((8, 4, 128, 6), 8), (HYBRID, 2), ((16, 1, 256, 0), 1)])
def test_few_rows_over_two_blocks(shape, n):
    """A step whose new entries end one block and begin the next, at every place, with blocks split over ranges or not."""
    lives = [64 - n, 63, 64, 127, 5000 // 64 * 64 + 64 - (n + 1) // 2, 0]
    p = Pop(shape, lives, 31, [(0, 0), (1, 0), (70, 3)], extra=4 * n, most=6 * n)
    for size in (1.0, 8.0, 0.5):
        _tail(p, [n] * 6, [p.tail(6 * n, size=size) for _ in range(3)])


def test_values_of_many_sizes():
    """Blocks whose scales differ, and tails that raise the scale of the block they begin in."""
    p = Pop(MID, [200, 90], 14, extra=256, most=256)
    for size in (2.0 ** -7, 2.0 ** 5, 1.0, 2.0 ** 12, 2.0 ** -12):
        for tails in ([3, 1], [40, 20]):
            _tail(p, tails, [p.tail(sum(tails), size=size)])


def test_scores_far_apart():
    p = Pop(SMALL, [800, 90], 15, [(100, 3), (0, 0)])
    for tails in ([40, 1], [1, 1]):
        # as for windows in bf16, with one rounded factor: a score moves by 0.018 in the root mean square, weights by that factor
        _tail(p, tails, [p.tail(sum(tails), scale=64.0) for _ in range(2)], most=2.2e-2)


def test_positions_of_their_own_and_far_ones():
    p = Pop(HYBRID, [700, 50], 16, extra=128, most=64, cursor=2 ** 31 - 2000)
    _tail(p, [30, 20])
    _tail(p, [2, 1])
    p = Pop(MID, [700, 50], 17, extra=128, most=64, cursor=10 ** 9)
    _tail(p, [30, 20], pos=np.concatenate([np.arange(5, 35), 7 * np.arange(20)]).astype(np.int32))
    _tail(p, [1, 1], pos=np.array([7, 123456789], np.int32))


def test_whole_tiles_dealt_in_waves():
    p = Pop(HYBRID, [100, 2000, 10, 0], 18, extra=1400, most=3500)
    _tail(p, [1400, 900, 0, 1200])


def test_many_characters():
    p = Pop(SMALL, [int(x) for x in np.random.default_rng(1).integers(0, 300, 256)], 19, extra=4, most=256)
    _tail(p, [int(x) for x in np.random.default_rng(2).integers(0, 2, 256)])


def test_a_tail_that_does_not_become_live():
    """Its first block keeps the scale; called again with other inputs it leaves what that call gives."""
    import torch
    p = Pop(SMALL, [100], 20)
    x = p.tail(5, size=64.0)
    p.ctx.tail_attn_prefill(0, [0, 5], *x, torch.empty_like(x[0]))
    k, v = p.ctx.get_kv(0, 0)
    exact = torch.cat([p.V[0][0], x[2].double().transpose(0, 1)], 1)
    assert torch.equal(v[:, 64:].double(), held(exact[:, 64:])[:, :36])
    p.K[0][0], p.V[0][0] = k.double(), v.double()
    _tail(p, [5])


# ---------------------------------------------------------------------------- rounds
def _rounds(p, steps):
    import torch
    from paper_2609_18935_gb300 import kvm
    for n, (spans, tails) in enumerate(steps):
        flat = [s for t in spans for s in t]
        cu, sb, se = _cu([len(t) for t in spans]), [a for a, _ in flat], [b for _, b in flat]
        m = sum(tails)
        ins, outs, xs = {}, {}, []
        for l, kind in enumerate(p.kinds):
            if kind == kvm.LAYER_ATTN:
                xs.append(p.tail(m))
                ins[l] = dict(zip("qkv", xs[-1]))
                outs[l] = torch.full_like(xs[-1][0], float("nan"))
            else:
                mk = lambda unit: _normal(p.g, m, 8, 64, unit=unit)
                ins[l] = {"q": mk(True), "k": mk(True), "v": mk(False), "alpha": torch.full((m, 8), 0.9, device="cuda"),
                          "beta": torch.full((m, 8), 0.5, device="cuda")}
                outs[l] = torch.empty(m, 8, 64, device="cuda", dtype=torch.bfloat16)
        p.ctx.update_round(cu, sb, se, _cu(tails), ins, outs)
        p.ctx.check()
        for b, t in enumerate(spans):
            p.cursor[b] += tails[b]
            for i in range(len(p.windows)):
                for mine in (p.K, p.V):
                    x = mine[i][b]
                    keep = [j for j in range(x.shape[1]) if not any(a <= j < e for a, e in t)]
                    if t:
                        lo = t[0][0] // BLOCK * BLOCK
                        x = torch.cat([x[:, keep[:lo]], held(x[:, keep[lo:]])], 1)
                    mine[i][b] = x
        for i, x in enumerate(xs):
            p.tail_done(i, tails, x, outs[p.at[i]], what=(n, i))


STEPS = [([[(0, 2), (800, 850)], [(5, 60)], []], [60, 1, 2]), ([[(10, 500)], [], [(0, 3)]], [1, 1, 1]), ([[], [], []], [1, 1, 1]),
         ([[(64, 128)], [(0, 1)], []], [0, 100, 1]), ([[], [(100, 175)], [(0, 4)]], [0, 0, 0]), ([[(5, 6), (7, 8), (9, 10)], [], []], [3, 0, 64])]


def test_rounds():
    import torch
    p = Pop(MID, [900, 130, 3], 21, [(0, 0), (128, 4)], extra=256, most=256)
    # scales that differ from block to block, so that survivors meet others'
    for i in range(2):
        for b, l in enumerate(p.lives):
            k = _normal(p.g, p.hkv, l, p.d, unit=True)
            v = _normal(p.g, p.hkv, l, p.d) * torch.pow(2.0, torch.arange(l, device="cuda") // 50 % 9 - 4.0)[:, None].bfloat16()
            p.ctx.set_kv(i, b, k, v)
            p.K[i][b], p.V[i][b] = held(k.double()), held(v.double())
    p.same()
    _rounds(p, STEPS)


@pytest.mark.parametrize("shape", [HYBRID, SMALL])
def test_rounds_beside_delta_rule_layers(shape):
    """A removal that runs beside the recurrent layers, on its own stream."""
    from paper_2609_18935_gb300 import kvm
    p = Pop(shape, [900, 130, 3], 22, [(0, 0), (70, 1), (0, 0)], extra=256, most=256,
            kinds=[kvm.LAYER_GDN, kvm.LAYER_ATTN, kvm.LAYER_ATTN, kvm.LAYER_GDN, kvm.LAYER_ATTN])
    _rounds(p, STEPS)


def test_compaction_alone_and_positions():
    import torch
    p = Pop(SMALL, [1000, 70], 23, extra=64)
    p.ctx.kv_compact(_cu([2, 1]), [3, 700, 69], [10, 900, 70])
    keep = np.array([j for j in range(1000) if not (3 <= j < 10 or 700 <= j < 900)])
    assert np.array_equal(p.ctx.get_positions(0).cpu().numpy(), keep)
    assert np.array_equal(p.ctx.get_positions(1).cpu().numpy(), np.arange(69))
    p.lives = [len(keep), 69]
    for mine in (p.K, p.V):
        mine[0][0] = held(mine[0][0][:, keep])
        x = mine[0][1][:, :69]
        mine[0][1] = torch.cat([x[:, :64], held(x[:, 64:])], 1)
    p.same()


def test_delimiters_leave_after_the_round():
    import torch
    p = Pop(SMALL, [100], 24, extra=64)
    x = p.tail(30)
    out = torch.empty_like(x[0])
    p.ctx.update_round([0, 0], [], [], [0, 30], {0: dict(zip("qkv", x))}, {0: out}, delim=([0, 2], [0, 28], [3, 30]))
    p.ctx.check()
    assert p.ctx.get_live(0)[0] == 125
    # the round's blocks, then formed anew without the delimiters
    other = Pop(SMALL, [100], 24, extra=64)
    y = other.tail(30)
    assert all(torch.equal(s, t) for s, t in zip(x, y))
    _tail(other, [30], [y])
    keep = list(range(100)) + list(range(103, 128))
    for got, want in zip(p.ctx.get_kv(0, 0), (other.K[0][0], other.V[0][0])):
        want = want[:, keep]
        assert torch.equal(got.double(), torch.cat([want[:, :64], held(want[:, 64:])], 1))


def test_rounds_on_the_host():
    """A round whose tensors are in pinned memory gives what the same round on the device gives, bit for bit."""
    import torch
    from paper_2609_18935_gb300 import kvm
    a, b = (Pop(SMALL, [300, 20], 25, [(0, 0), (64, 1)], extra=64) for _ in range(2))
    xs = [a.tail(30) for _ in range(2)]
    ins = {i: dict(zip("qkv", x)) for i, x in enumerate(xs)}
    outs = {i: torch.empty_like(x[0]) for i, x in enumerate(xs)}
    a.ctx.update_round([0, 1, 1], [3], [99], [0, 25, 30], ins, outs)
    pinned = {i: torch.empty(x[0].shape, dtype=torch.bfloat16).pin_memory() for i, x in enumerate(xs)}
    b.ctx.update_round([0, 1, 1], [3], [99], [0, 25, 30], kvm.pinned_layer_inputs(ins), pinned, io_on_host=True)
    torch.cuda.synchronize()
    for p in (a, b):
        p.ctx.check()
    assert all(torch.equal(outs[i].cpu(), pinned[i]) for i in range(2))
    for i in range(2):
        for c in range(2):
            assert all(torch.equal(s, t) for s, t in zip(a.ctx.get_kv(i, c), b.ctx.get_kv(i, c)))


# ---------------------------------------------------------------------------- the rest of a context's calls
def test_fork():
    p = Pop(MID, [600, 20], 26, [(50, 4), (0, 0)], extra=64)
    other = p.new()
    other.fork_from(p.ctx)
    old, p.ctx = p.ctx, other
    p.same()
    _tail(p, [33, 7])
    # the source is as it was
    fresh = Pop(MID, [600, 20], 26, [(50, 4), (0, 0)], extra=64)
    fresh.ctx = old
    fresh.same()


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4), (1, 0)])
def test_probe(window, sinks):
    import torch
    from attn64 import in_sight, rope
    p = Pop(HYBRID, [20, 333], 27, [(0, 0), (window, sinks)])
    q = _normal(p.g, 7, 16, 256)
    probs, _ = p.ctx.attn_probe(1, 1, q)
    p.ctx.check()
    qr = rope(q.double(), torch.arange(326, 333), 64)
    seen = in_sight(np.arange(326, 333), 333, window, sinks)
    s = torch.stack([(qr[:, h] @ p.K[1][1][h // 8].T) / 16.0 for h in range(16)])
    want = torch.softmax(s.masked_fill(~seen, -float("inf")), -1).mean((0, 1))
    assert float((probs.double() - want).abs().max()) < 1e-5 * float(want.max())       # sums in 32 bits, as over bf16 caches
    p.same()


def test_refusals():
    from paper_2609_18935_gb300 import kvm
    p = Pop(SMALL, [100], 28)
    with pytest.raises(kvm.KvmError) as e:
        p.ctx.draft_reserve(4)
    assert e.value.code == kvm.KVM_E_UNSUPPORTED
    with pytest.raises(kvm.KvmError) as e:
        p.ctx.rerotate_keys(0, 3, 5, [200, 201])
    assert e.value.code == kvm.KVM_E_UNSUPPORTED
    wide = kvm.Context([kvm.LAYER_ATTN], *SMALL, 1.0e4, 8, 64, 64, p.cap, 64)
    for a, b in ((wide, p.ctx), (p.ctx, wide)):
        with pytest.raises(kvm.KvmError) as e:
            a.fork_from(b)
        assert e.value.code == kvm.KVM_E_INVAL
    with pytest.raises(ValueError):
        kvm.Context([kvm.LAYER_ATTN], *SMALL, 1.0e4, 8, 64, 64, [64], 64, kv_bits=4)
    p.same()


def test_captured_steps_replayed_with_new_inputs():
    import torch
    p = Pop(HYBRID, [3000, 90], 29, [(0, 0), (128, 4)], extra=128)
    for n in (1, 20):
        xs = [[t.clone() for t in p.tail(2 * n)] for _ in range(2)]
        outs = [torch.empty_like(x[0]) for x in xs]
        s = torch.cuda.Stream()
        cu = [0, n, 2 * n]
        with torch.cuda.stream(s):
            for i in range(2):
                p.ctx.tail_attn_prefill(i, cu, *xs[i], outs[i])
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                for i in range(2):
                    p.ctx.tail_attn_prefill(i, cu, *xs[i], outs[i])
        for _ in range(3):
            for x in xs:
                for t, y in zip(x, p.tail(2 * n)):
                    t.copy_(y)
            # what the blocks hold before the step: the last one may have raised a scale
            for i in range(2):
                for b in range(2):
                    p.K[i][b], p.V[i][b] = (t.double() for t in p.ctx.get_kv(i, b))
            graph.replay()
            torch.cuda.synchronize()
        p.ctx.check()
        p.ctx.advance(cu)
        p.cursor = [c + n for c in p.cursor]
        for i in range(2):
            p.tail_done(i, [n, n], xs[i], outs[i], what=(n, i))


def test_the_same_calls_give_the_same_bits():
    import torch
    got = []
    for _ in range(2):
        p = Pop(HYBRID, [5000, 700], 30, [(0, 0), (1000, 4)], extra=128)
        runs = []
        for tails in ([1, 1], [2, 1], [60, 40]):
            for i in range(2):
                x = p.tail(sum(tails))
                out = torch.empty_like(x[0])
                p.ctx.tail_attn_prefill(i, _cu(tails), *x, out)
                runs.append(out)
        got.append(runs)
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("bits,window", [(8, 0), (8, 100), (16, 100)])
def test_offsets_past_32_bits(bits, window):
    """A character behind another's nine million slots (its caches' offsets are past 2^32 bytes) gives the bits that it gives
    on its own: few rows, a tail, a removal, what is read out."""
    import torch
    from paper_2609_18935_gb300 import kvm
    hq, hkv, d, rot = HYBRID
    g = torch.Generator(device="cuda").manual_seed(33)
    k, v = _normal(g, hkv, 700, d, unit=True), _normal(g, hkv, 700, d)
    steps = [[_normal(g, n, h, d, unit=h == hkv) for h in (hq, hkv, hkv)] for n in (1, 40, 2)]
    got = []
    for ahead in (64, 9_000_000):
        ctx = kvm.Context([kvm.LAYER_ATTN], hq, hkv, d, rot, 1.0e4, 8, 64, 64, [ahead, 1000], 64, kv_bits=bits)
        if window:
            ctx.set_window(0, window, 4)
        ctx.load_prefix(1, 700, 700, np.arange(700, dtype=np.int32))
        ctx.set_kv(0, 1, k, v)
        out = []
        for i, x in enumerate(steps):
            n = x[0].shape[0]
            o = torch.empty_like(x[0])
            ctx.update_round([0, 0, 2], [5, 300], [9, 391], [0, 0, n], {0: dict(zip("qkv", x))}, {0: o})
            ctx.check()
            out += [o, *ctx.get_kv(0, 1), ctx.get_positions(1)]
        if bits == 8:
            out.append(ctx.attn_probe(0, 1, steps[2][0])[0])
        got.append(out)
        ctx.destroy()
        torch.cuda.empty_cache()
    assert all(torch.equal(a, b) for a, b in zip(*got))
