"""Attention over caches that stay small: a sliding window with a few first entries that stay visible, and caches in 8 bits.

  tail    tail_attn_prefill: a tail's keys and values go behind the live entries, its queries attend to what they see.  With
          a window W and S sinks, the token at live index x sees the entries j <= x with j > x - W or j < S.  With 8 bits
          the caches hold e4m3 numbers times a power of two for each block of 64 live slots and KV head, K and V apart: the
          smallest power 2^e, e >= -117, for which the block's largest magnitude is at most 448 2^e; each value is rounded to
          the nearest, ties to even.  A tail's entries are rounded as they are appended, a block they share with older
          entries again as a whole, and the attention reads what the cache then holds
  draft   draft_attn in a windowed layer: a node at depth e counts as live index L + e, and sees all its ancestors
  round   update_round over two attention layers in 8 bits, the first windowed: entries are removed (the blocks from the
          first removed one on are formed anew), a tail of as many tokens follows

Several characters are packed and ragged: `prefix` and `tail` are upper ends, lengths are spread below them, and a character
may have no tail at all.  Value distributions: q, v ~ N(0, 1), unit keys; values here are scaled per character by powers of two,
as layers' values differ in size.
"""
import math

import numpy as np
import torch

own = False

# the hybrid stack of the library's benchmark, a middle one, and the small test shape
HYBRID = {"hq": 16, "hkv": 2, "d": 256, "rot": 64}
MID = {"hq": 16, "hkv": 4, "d": 128, "rot": 128}
SMALL = {"hq": 8, "hkv": 2, "d": 64, "rot": 64}
THETA = 1.0e4
BLOCK = 64


def _case(kind, shape, **kw):
    c = {"kind": kind, "bits": 16, "chars": 1, "prefix": 0, "tail": 1, "window": 0, "sinks": 0, "lens": 1}
    if kind == "draft":
        c["width"] = 4
    c.update(shape)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: one token of one character, a short window in a short cache
        _case("tail", SMALL, name="window_small", prefix=512, window=128, sinks=4),
        # a population decoding together, each far past its window
        _case("tail", HYBRID, name="window_decode_population", chars=32, prefix=16384, window=4096, sinks=4, lens=3),
        # a game character's maintenance round, an odd tail over 8K
        _case("tail", HYBRID, name="window_npc", prefix=8192, tail=251, window=1024, sinks=16),
        # a long-lived character's replacement text, a wide window
        _case("tail", HYBRID, name="window_long", prefix=32768, tail=1024, window=8192, sinks=64),
        # two texts read from (nearly) nothing, without sinks, an odd window
        _case("tail", MID, name="window_fill", chars=2, prefix=100, tail=4001, window=1000, lens=5),
        # a bushy tree of guesses over a windowed layer
        _case("draft", HYBRID, name="window_draft", prefix=8192, tail=16, window=2048, sinks=4),
        # the smallest call over a cache in 8 bits
        _case("tail", SMALL, name="kv8_small", bits=8, prefix=512),
        # one long-lived character's decode step
        _case("tail", HYBRID, name="kv8_decode_long", bits=8, prefix=32768),
        # a population's decode step: what 8 bits are for
        _case("tail", HYBRID, name="kv8_decode_population", bits=8, chars=32, prefix=16384, lens=3),
        # a game character's maintenance round
        _case("tail", HYBRID, name="kv8_npc", bits=8, prefix=8192, tail=256),
        # a population's tails in a windowed layer of a middle stack
        _case("tail", MID, name="kv8_window_population", bits=8, chars=8, prefix=8192, tail=96, window=2000, sinks=10, lens=7),
        # whole rounds: entries of several characters replaced in a windowed and a full layer
        _case("round", HYBRID, name="kv8_round", bits=8, chars=3, prefix=8192, tail=256, window=2048, sinks=4, lens=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tail"] * 6 + ["draft", "round", "round"])
    shape = rng.choice([HYBRID, HYBRID, MID, SMALL])
    chars = 1 if rng.random() < 0.4 else _log(rng, 2, 32 if kind == "tail" else 4)
    kw = {"chars": chars, "lens": rng.randrange(1, 1 << 20)}
    if kind == "tail":
        bits = rng.choice([16, 8, 8])
        tail = 1 if rng.random() < 0.4 else _log(rng, 1, min(2048, 16384 // chars))
        # no more entries, and no more scores of the plain form, than the largest listed calls
        prefix = _log(rng, 1, max(64, min(32768, 524_288 // chars, 30_000_000 // (chars * tail) - tail)))
        kw.update(bits=bits, tail=tail, prefix=prefix)
        if bits == 16 or rng.random() < 0.3:
            kw.update(window=_log(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 10, 64, 100]))
        return _case(kind, shape, **kw)
    if kind == "draft":
        return _case(kind, shape, prefix=_log(rng, 64, 16384), tail=_log(rng, 1, 64), width=rng.choice([1, 2, 4, 8]),
                     window=_log(rng, 64, 8192), sinks=rng.choice([0, 4, 100]), **kw)
    prefix = _log(rng, 300, 8192)
    return _case(kind, shape, bits=8, prefix=prefix, tail=_log(rng, 1, min(256, prefix // 8)), window=_log(rng, 1, 4096),
                 sinks=rng.choice([0, 4, 100]), **kw)


# ---------------------------------------------------------------------------- sizes of a case
def _lengths(case):
    """(live entries, tail tokens or nodes) per character."""
    n, hi_l, hi_n = case["chars"], case["prefix"], case["tail"]
    if n == 1:
        return [hi_l], [hi_n]
    r = np.random.default_rng(case["lens"])
    L = [int(x) for x in r.integers(hi_l // 8, hi_l + 1, size=n)]
    if hi_n == 1:
        return L, [1] * n
    return L, [min(hi_n, L[0]) if case["kind"] == "round" else hi_n] + [
        int(min(x, l)) if case["kind"] == "round" else int(x) for x, l in zip(r.integers(0, hi_n + 1, size=n - 1), L[1:])]


def _trees(case):
    """Per character the parents of its nodes, level by level: one root, then up to `width` nodes under random ones of the
    level before."""
    r = np.random.default_rng([case["lens"], 77])
    out = []
    for n in _lengths(case)[1]:
        parent, level = [], []
        while len(parent) < n:
            take = 1 if not parent else min(case["width"], n - len(parent))
            new = [-1] if not parent else sorted(int(x) for x in r.choice(level, size=take))
            level = list(range(len(parent), len(parent) + take))
            parent += new
        out.append(parent)
    return out


def _ancestors(parent):
    """[n][n] truth values: node j is i or an ancestor of i."""
    a = np.eye(len(parent), dtype=bool)
    for i, p in enumerate(parent):
        if p >= 0:
            a[i] |= a[p]
    return a


def _spans(case):
    """Per character the live-index spans that a round removes: as many entries as its tail has, in up to three spans."""
    r = np.random.default_rng([case["lens"], 79])
    out = []
    for l, m in zip(*_lengths(case)):
        k = min(3, m)
        sizes = np.diff(np.concatenate([[0], np.sort(r.choice(np.arange(1, m), k - 1, replace=False)), [m]])) if k else []
        gaps = np.sort(r.integers(0, l - m + 1, size=k))
        spans, gone = [], 0
        for g, s in zip(gaps, sizes):
            lo = int(g) + gone
            if spans and spans[-1][1] == lo:
                spans[-1] = (spans[-1][0], lo + int(s))
            else:
                spans.append((lo, lo + int(s)))
            gone += int(s)
        out.append(spans)
    return out


def _kept(l, spans):
    keep = np.ones(l, bool)
    for a, b in spans:
        keep[a:b] = False
    return np.flatnonzero(keep)


def _cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _windows(case):
    """(window, sinks) per layer; 0: the whole cache."""
    w = (case["window"], case["sinks"])
    return [w, (0, 0)] if case["kind"] == "round" else [w]


def _room(case):
    L, N = _lengths(case)
    most = max(l if case["kind"] == "round" else l + n for l, n in zip(L, N))
    return -(-most // BLOCK) * BLOCK


def _plan(case):
    """Index tables.  Padded: packed rows and truth values [chars][most tokens].  Packed, a row a token: its character, its
    slot, its block in the list of blocks that the tail touches, its row there."""
    L, N = _lengths(case)
    if case["kind"] == "round":
        L = [l - n for l, n in zip(L, N)]
    n = max(N)
    cu = _cu(N)
    row = np.zeros((len(N), n), np.int64)
    real = np.zeros((len(N), n), bool)
    anc = np.zeros((len(N), n, n), bool)
    who, slot, at, blocks = [], [], [], []
    for b, (l, m) in enumerate(zip(L, N)):
        row[b, :m] = cu[b] + np.arange(m)
        real[b, :m] = True
        first = len(blocks)
        if m:
            blocks += [(b, x) for x in range(l // BLOCK, (l + m - 1) // BLOCK + 1)]
        who += [b] * m
        slot += list(range(l, l + m))
        at += [first + (l + i) // BLOCK - l // BLOCK for i in range(m)]
    if case["kind"] == "draft":
        for b, t in enumerate(_trees(case)):
            anc[b, :len(t), :len(t)] = _ancestors(t)
    dev = lambda x: torch.as_tensor(np.array(x, np.int64)).cuda()
    p = {"row": dev(row), "flat": dev(np.flatnonzero(real.reshape(-1))), "live": dev(L), "who": dev(who), "slot": dev(slot),
         "at": dev(at), "in": dev([x % BLOCK for x in slot]), "blk": dev(np.array(blocks, np.int64).reshape(-1, 2)),
         "count": dev(N), "anc": torch.as_tensor(anc).cuda()}
    if case["kind"] == "round":
        was, T = _lengths(case)[0], _room(case)
        keep = np.zeros((len(N), T), np.int64)
        new = []
        for b, (l, spans) in enumerate(zip(was, _spans(case))):
            k = _kept(l, spans)
            keep[b, :len(k)] = k
            if spans:
                new += [(b, x) for x in range(spans[0][0] // BLOCK, -(-len(k) // BLOCK))]
        p["keep"], p["formed"] = dev(keep), dev(np.array(new, np.int64).reshape(-1, 2))
        p["stay"] = torch.arange(T, device="cuda") < p["live"][:, None]
    return p


# ---------------------------------------------------------------------------- inputs
def _gen(seed, k):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + k)


def _normal(g, *shape, unit=False):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if unit:
        x = x / x.norm(dim=-1, keepdim=True)
    return x


def _held(x):
    """x [..][64 rows][d] in 32 bits as 8 bits hold it: a scale for each block of rows."""
    m, e = torch.frexp(x.abs().amax((-1, -2), keepdim=True))
    e = (e - 9 + (m > 0.875).int()).clamp(min=-117)                    # 448 = 0.875 2^9
    y = torch.ldexp(x, -e)
    step = torch.frexp(y)[1].clamp(min=-5) - 4                         # four significant bits, subnormal below 2^-6
    return torch.ldexp(torch.round(torch.ldexp(y, -step)), step + e)


def _parts(case, seed):
    """Per layer: the tail's q, k, v and every character's cache, [chars][hkv][room][d] in bf16 with room for the tail."""
    L, N = _lengths(case)
    m, T, d, hkv = sum(N), _room(case), case["d"], case["hkv"]
    out = []
    for i in range(len(_windows(case))):
        g = _gen(seed, i)
        x = {"q": _normal(g, m, case["hq"], d).bfloat16(), "k": _normal(g, m, hkv, d, unit=True).bfloat16(),
             "v": _normal(g, m, hkv, d).bfloat16()}
        size = torch.pow(2.0, torch.randint(-2, 3, (len(L), 1, 1, 1), generator=g, device="cuda").float())
        live = (torch.arange(T, device="cuda") < torch.tensor(L, device="cuda")[:, None])[:, None, :, None]
        for name, unit in (("K", True), ("V", False)):
            y = (_normal(g, len(L), hkv, T, d, unit=unit) * (1.0 if unit else size) * live).bfloat16()
            if case["bits"] == 8:
                y = _held(y.float().unflatten(2, (-1, BLOCK))).flatten(2, 3).bfloat16()
            x[name] = y
        out.append(x)
    return out


def prepare(case, seed):
    parts = _parts(case, seed)
    L = _lengths(case)[0]
    s = {"case": case, "parts": parts, "plan": _plan(case), "cursor": torch.tensor(L, device="cuda")}
    if case["kind"] == "round":
        T = _room(case)
        s["pos"] = torch.arange(T, device="cuda", dtype=torch.int32).expand(len(L), T).contiguous()
    if own:
        s.update(_handle(case, parts))
    torch.cuda.synchronize()
    return s


def _handle(case, parts):
    """The context that a user's program keeps, with its prefixes, and buffers for the answers."""
    from paper_2609_18935_gb300 import kvm
    L, N = _lengths(case)
    ctx = kvm.Context([kvm.LAYER_ATTN] * len(parts), case["hq"], case["hkv"], case["d"], case["rot"], THETA, 8, 64, 64,
                      [l + n + 1 for l, n in zip(L, N)], max(1, sum(N)), kv_bits=case["bits"])
    for i, (w, sinks) in enumerate(_windows(case)):
        if w:
            ctx.set_window(i, w, sinks)
    for b, l in enumerate(L):
        ctx.load_prefix(b, l, l, np.arange(l, dtype=np.int32))
        for i, x in enumerate(parts):
            if l:
                ctx.set_kv(i, b, x["K"][b, :, :l].contiguous(), x["V"][b, :, :l].contiguous())
    h = {"ctx": ctx, "out": [torch.empty_like(x["q"]) for x in parts], "cu": _cu(N)}
    if case["kind"] == "draft":
        ctx.draft_reserve(max(1, sum(N)))
        # a step's tree is announced once, for all its layers
        ctx.draft_begin(_cu(N), np.concatenate([np.array(t, np.int32) for t in _trees(case)]))
    if case["kind"] == "round":
        spans = _spans(case)
        flat = [x for t in spans for x in t]
        h["spans"] = (_cu([len(t) for t in spans]), np.array([a for a, _ in flat], np.int32), np.array([b for _, b in flat], np.int32))
        h["in"] = {i: {n: x[n] for n in "qkv"} for i, x in enumerate(parts)}
        h["outs"] = dict(enumerate(h["out"]))
    return h


# ---------------------------------------------------------------------------- the calls
def _run_own(s):
    case, ctx, out = s["case"], s["ctx"], s["out"]
    if case["kind"] == "round":
        ctx.update_round(*s["spans"], s["cu"], s["in"], s["outs"])
        chars, layers = range(case["chars"]), range(len(out))
        return {"out": out, "kv": [ctx.get_kv(i, b) for i in layers for b in chars], "pos": [ctx.get_positions(b) for b in chars]}
    x = s["parts"][0]
    if case["kind"] == "draft":
        ctx.draft_attn(0, x["q"], x["k"], x["v"], out[0])
    else:
        ctx.tail_attn_prefill(0, s["cu"], x["q"], x["k"], x["v"], out[0])
    return {"out": out[0]}


# ---------------------------------------------------------------------------- the plain form
def _turned(x, pos, rot):
    """Rows x [n][heads][d] rotated at pos [n]: pairs (i, i + rot/2); the angles in 64 bits."""
    half = rot // 2
    freq = THETA ** (-2.0 * torch.arange(half, device=x.device, dtype=torch.float64) / rot)
    ang = pos.double()[:, None, None] * freq
    c, s = ang.cos().float(), ang.sin().float()
    a, b = x[..., :half], x[..., half:rot]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., rot:]], -1)


def _append(case, x, plan, k):
    """The tail's rotated keys k and its values into the caches, in place."""
    for cache, rows in ((x["K"], k), (x["V"], x["v"].float())):
        if case["bits"] == 16:
            cache[plan["who"], :, plan["slot"]] = rows.bfloat16()
            continue
        view = cache.unflatten(2, (-1, BLOCK))
        b, at = plan["blk"][:, 0], plan["blk"][:, 1]
        blocks = view[b, :, at].float()                                # [blocks][hkv][64][d]
        blocks[plan["at"], :, plan["in"]] = rows
        view[b, :, at] = _held(blocks).bfloat16()


def _plain_attn(case, x, plan, window, sinks, cursor):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g, live, rows = hq // hkv, plan["live"], plan["row"]
    chars, n = rows.shape
    tree = case["kind"] == "draft"
    order = plan["anc"].sum(2) - 1 if tree else torch.arange(n, device="cuda").expand(chars, n)    # live index less L
    pos = (cursor[:, None] + order).flatten()[plan["flat"]]
    q, k = (_turned(x[t].float(), pos, case["rot"]) for t in "qk")
    _append(case, x, plan, k)
    K, V = x["K"].float(), x["V"].float()
    key = torch.arange(K.shape[2], device="cuda")
    at = (live[:, None] + order)[..., None]                            # [chars][n][1]
    if tree:
        node = key - live[:, None]                                     # [chars][keys]
        inside = (node >= 0) & (node < n)
        seen = torch.gather(plan["anc"], 2, node.clamp(0, n - 1)[:, None].expand(-1, n, -1)) & inside[:, None]
        seen = seen | (node < 0)[:, None]
    else:
        seen = key <= at
    if window:
        near = (key > at - window) | (key < sinks)
        seen = seen & (near | (node >= 0)[:, None] if tree else near)
    q = q[rows].view(chars, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(chars, hkv, n * g, d)
    w = (q @ K.transpose(2, 3)) * (1.0 / math.sqrt(d))
    w = w.masked_fill_(~seen.repeat_interleave(g, 1)[:, None], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True).clamp_(min=-3.0e38)).exp_()
    o = (w @ V) / w.sum(-1, keepdim=True).clamp_(min=1e-30)
    o = o.view(chars, hkv, n, g, d).permute(0, 2, 1, 3, 4).reshape(chars * n, hq, d)
    return o[plan["flat"]].bfloat16()


def _plain_removed(x, plan):
    """The survivors of the caches in their new places, the blocks from the first removed entry on formed anew."""
    b, at = plan["formed"][:, 0], plan["formed"][:, 1]
    for name in "KV":
        cache = x[name]
        to = plan["keep"][:, None, :, None].expand(-1, cache.shape[1], -1, cache.shape[3])
        cache = torch.gather(cache, 2, to) * plan["stay"][:, None, :, None]
        view = cache.unflatten(2, (-1, BLOCK))
        view[b, :, at] = _held(view[b, :, at].float()).bfloat16()
        x[name] = cache


def _run_plain(s):
    case, plan, parts = s["case"], s["plan"], s["parts"]
    if case["kind"] != "round":
        return {"out": _plain_attn(case, parts[0], plan, *_windows(case)[0], s["cursor"])}
    out = []
    for x, (w, sinks) in zip(parts, _windows(case)):
        _plain_removed(x, plan)
        out.append(_plain_attn(case, x, plan, w, sinks, s["cursor"]))
    pos = torch.gather(s["pos"], 1, plan["keep"])
    pos[plan["who"], plan["slot"]] = (s["cursor"][plan["who"]] + plan["slot"] - plan["live"][plan["who"]]).int()
    s["pos"], s["cursor"] = pos, s["cursor"] + plan["count"]
    L = _lengths(case)[0]
    return {"out": out, "kv": [(x["K"][b, :, :l].clone(), x["V"][b, :, :l].clone()) for x in parts for b, l in enumerate(L)],
            "pos": [pos[b, :l].clone() for b, l in enumerate(L)]}


def run(s):
    if own:
        return _run_own(s)
    return _run_plain(s)


# ---------------------------------------------------------------------------- work of a pass
def _attn_work(case, L, N, window, sinks):
    hq, hkv, d, per = case["hq"], case["hkv"], case["d"], case["bits"] // 8
    read = pairs = 0
    trees = _trees(case) if case["kind"] == "draft" else None
    for b, (l, m) in enumerate(zip(L, N)):
        if not m:
            continue
        lo = max(0, l - window + 1) if window else 0                   # the first token's window; later ones' begin later
        read += l - lo + min(sinks, lo)
        if trees:
            anc = _ancestors(trees[b])
            low = np.maximum(l + anc.sum(1) - window, 0)
            pairs += int(anc.sum()) + int((l - np.minimum(low, l) + np.minimum(np.minimum(sinks, low), l)).sum())
        else:
            x = l + np.arange(m, dtype=np.int64)
            low = np.maximum(x - window + 1, 0) if window else 0 * x
            pairs += int((x + 1 - low + np.minimum(sinks, low)).sum())
    m = sum(N)
    return read * hkv * d * 2 * per + m * (2 * hq + 2 * hkv) * d * 2 + m * hkv * d * 2 * per, 4 * d * hq * pairs


def work(case):
    L, N = _lengths(case)
    if case["kind"] != "round":
        b, f = _attn_work(case, L, N, case["window"], case["sinks"])
        return {"bytes": float(b), "flops": float(f)}
    b = f = 0
    # every survivor behind the first removed entry moves: read and written, and the caches are read out in 16 bits
    moved = sum(l - n - s[0][0] for l, n, s in zip(L, N, _spans(case)) if s)
    for w, sinks in _windows(case):
        x, y = _attn_work(case, [l - n for l, n in zip(L, N)], N, w, sinks)
        b, f = b + x + (2 * moved + 3 * sum(L)) * case["hkv"] * case["d"] * 2, f + y
    return {"bytes": float(b + 8 * (moved + sum(L))), "flops": float(f)}


# ---------------------------------------------------------------------------- the same in 64 bits
def _exact_held(rows):
    """rows [hkv][n][d] in 64 bits from a block's first row on, as 8 bits hold them."""
    out = torch.empty_like(rows)
    for lo in range(0, rows.shape[1], BLOCK):
        y = rows[:, lo:lo + BLOCK]
        top = y.abs().amax((1, 2), keepdim=True)
        e = torch.ceil(torch.log2(top / 448.0)).clamp(min=-117.0)
        e = torch.where(top <= 448.0 * 2.0 ** (e - 1), e - 1, torch.where(top > 448.0 * 2.0 ** e, e + 1, e)).clamp(min=-117.0)
        y = y / 2.0 ** e
        grid = 2.0 ** (torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, lo:lo + BLOCK] = torch.round(y / grid) * grid * 2.0 ** e
    return out


def _exact_layer(case, x, window, sinks, spans=None):
    """(outputs, per character its cache after the call, K and V [hkv][live][d])."""
    L, N = _lengths(case)
    g, rot = case["hq"] // case["hkv"], case["rot"]
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    freq = torch.exp(-math.log(THETA) * 2.0 * i / rot)
    outs, after, at = [], [], 0
    for b, (l, n) in enumerate(zip(L, N)):
        cache = [x[t][b, :, :l].double() for t in "KV"]
        if spans is not None:
            kept = torch.as_tensor(_kept(l, spans[b])).cuda()
            first = spans[b][0][0] // BLOCK * BLOCK if spans[b] else len(kept)
            cache = [y[:, kept] for y in cache]
            cache = [torch.cat([y[:, :first], _exact_held(y[:, first:])], 1) for y in cache]
        live = cache[0].shape[1]
        tree = _ancestors(_trees(case)[b]) if case["kind"] == "draft" else None
        depth = torch.as_tensor(tree.sum(1) - 1 if tree is not None else np.arange(n)).cuda()
        turn = torch.exp(1j * (l + depth).double()[:, None, None] * freq)

        def rotate(y):
            z = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * turn
            return torch.cat([z.real, z.imag, y[..., rot:]], -1)
        q = rotate(x["q"][at:at + n].double())
        new = [rotate(x["k"][at:at + n].double()), x["v"][at:at + n].double()]
        cache = [torch.cat([c, y.transpose(0, 1)], 1) for c, y in zip(cache, new)]
        if case["bits"] == 8 and n:
            lo = live // BLOCK * BLOCK
            cache = [torch.cat([c[:, :lo], _exact_held(c[:, lo:])], 1) for c in cache]
        K, V = cache
        after.append((K, V))
        at += n
        if not n:
            continue
        j = torch.arange(live + n, device="cuda")
        me = (live + depth)[:, None]
        if tree is not None:
            ok = torch.cat([(j[:live] > me - window) | (j[:live] < sinks), torch.as_tensor(tree).cuda()], 1)
        else:
            ok = j <= me
            if window:
                ok &= (j > me - window) | (j < sinks)
        bias = torch.where(ok, 0.0, -math.inf).double()
        o = torch.empty_like(q)
        for h in range(case["hkv"]):
            w = torch.softmax(torch.einsum("igd,jd->gij", q[:, h * g:(h + 1) * g], K[h]) / math.sqrt(case["d"]) + bias, -1)
            o[:, h * g:(h + 1) * g] = torch.einsum("gij,jd->igd", w, V[h])
        outs.append(o)
    return torch.cat(outs), after


def exact(case, seed):
    parts = _parts(case, seed)
    if case["kind"] != "round":
        return {"out": _exact_layer(case, parts[0], case["window"], case["sinks"])[0]}
    got = [_exact_layer(case, x, w, sinks, _spans(case)) for x, (w, sinks) in zip(parts, _windows(case))]
    return {"out": [o for o, _ in got], "kv": [kv for _, after in got for kv in after], "pos": [None] * case["chars"]}
