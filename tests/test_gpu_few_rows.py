"""Steps and short tails of windowed layers and 8-bit caches whose output lies over an input: at most 16 rows of a KV head run in
one launch that reads the inputs and stores the outputs, more of them read every input in a launch before."""
import numpy as np
import pytest

import test_gpu_kv8 as kv8
import test_gpu_window as win

pytestmark = pytest.mark.gpu

HYBRID, SMALL = (16, 2, 256, 64), (8, 2, 64, 64)


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_18935_gb300 import kvm
    kvm.load_library()


def _placed(x, over, shift):
    """q, k_new, v_new and an output that begins `shift` numbers behind (before) the one named; and the memory that they share,
    as it was, with the output's place in it."""
    import torch
    i, n = "qkv".index(over), x[0].numel()
    first = max(0, -shift)
    room = torch.full((abs(shift) + n + x[i].numel(),), 7.0, dtype=torch.bfloat16, device="cuda")
    room[first:first + x[i].numel()] = x[i].flatten()
    ins = [room[first:first + t.numel()].view(t.shape) if j == i else t.clone() for j, t in enumerate(x)]
    at = slice(first + shift, first + shift + n)
    return ins, room[at].view(x[0].shape), room, room.clone(), at


def _rest_is_left(room, was, at):
    import torch
    assert torch.equal(room[:at.start], was[:at.start]) and torch.equal(room[at.stop:], was[at.stop:])


OVER = [("q", 0), ("q", 512), ("q", -2048), ("k", 0), ("k", 1024), ("k", -512), ("v", 0), ("v", 512), ("v", -1024)]


@pytest.mark.parametrize("shape", [HYBRID, SMALL])
@pytest.mark.parametrize("over,shift", OVER)
@pytest.mark.parametrize("bits", [16, 8])
def test_an_output_over_an_input(shape, over, shift, bits):
    """Tails of up to 16 rows of a KV head, one with the next token more, short caches and split ones."""
    import torch
    g = shape[0] // shape[1]
    for more in (0, 1):
        lives = [100] * 18 + [5000, 64, 63, 0, 1, 900]
        tails = [16 // g] * 23 + [16 // g + more]
        mod = win if bits == 16 else kv8
        p = mod.Pop(shape, lives, 50, [(70, 3), (0, 0)], extra=20, most=sum(tails))
        xs = [p.tail(sum(tails)) for _ in p.windows]
        outs = []
        for i, x in enumerate(xs):
            ins, out, *rest = _placed(x, over, shift)
            p.ctx.tail_attn_prefill(i, win._cu(tails), *ins, out)
            p.ctx.check()
            _rest_is_left(*rest)
            outs.append(out.clone())
            if bits == 16:
                p.check(i, tails, x, outs[i], (more, i), keep=True)
        p.ctx.advance(win._cu(tails))
        for b, m in enumerate(tails):
            p.cursor[b] += m
        for i, x in enumerate(xs):
            if bits == 8:
                p.tail_done(i, tails, x, outs[i], what=(more, i))
                continue
            for b in range(len(lives)):
                k, v = p.ctx.get_kv(i, b)
                assert torch.equal(v.double(), p.V[i][b])
                # rounded once after a rotation in 32 bits (see test_gpu_window)
                off = 2.0 ** -8 * p.K[i][b].abs() + 2.0 ** -19 * p.K[i][b].abs().amax()
                assert bool(((k.double() - p.K[i][b]).abs() <= off).all())


@pytest.mark.parametrize("bits", [16, 8])
def test_which_outputs_one_launch_bears(bits):
    """Whole tiles of two units: one launch with an output of its own or in q's place, two where blocks would read what others store."""
    import torch
    mod = win if bits == 16 else kv8
    p = mod.Pop(HYBRID, [100] * 24, 51, [(70, 3)], extra=8, most=48)
    x = p.tail(48)

    def launches(ins, out):
        n = p.ctx.launch_count()
        p.ctx.tail_attn_prefill(0, win._cu([2] * 24), *ins, out)
        p.ctx.check()
        return p.ctx.launch_count() - n

    assert launches(x, torch.empty_like(x[0])) == 1
    for over, shift in OVER:
        ins, out, *_ = _placed(x, over, shift)
        assert launches(ins, out) == (1 if (over, shift) == ("q", 0) else 2), (over, shift)
    # next to each other is not over each other
    room = torch.empty(x[0].numel() + x[1].numel() + x[2].numel(), dtype=torch.bfloat16, device="cuda")
    k, out, v = (t.view(y.shape) for t, y in zip(room.split([x[1].numel(), x[0].numel(), x[2].numel()]), (x[1], x[0], x[2])))
    k.copy_(x[1])
    v.copy_(x[2])
    assert launches([x[0], k, v], out) == 1


@pytest.mark.parametrize("bits", [16, 8])
def test_a_captured_step_with_its_output_over_its_keys(bits):
    import torch
    mod = win if bits == 16 else kv8
    p = mod.Pop(SMALL, [3000, 90], 52, [(128, 4)], extra=8, most=2)
    x = p.tail(2)
    ins, out, room, *_ = _placed(x, "k", 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        s.synchronize()
        with torch.cuda.graph(graph, stream=s):
            p.ctx.tail_attn_prefill(0, [0, 1, 2], *ins, out)
    for _ in range(3 if bits == 16 else 1):          # (8 bits: what is run again may round older entries again)
        x = p.tail(2)
        for t, y in zip(ins, x):
            t.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        p.ctx.check()
        if bits == 16:
            p.check(0, [1, 1], x, out)
    if bits == 8:
        p.ctx.advance([0, 1, 2])
        p.cursor = [c + 1 for c in p.cursor]
        p.tail_done(0, [1, 1], x, out)
