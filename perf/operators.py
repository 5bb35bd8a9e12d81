"""Drafting over a maintained state: trees of guessed tokens scored in one pass, judged, and the accepted path kept.

A draft model (or a lookup) guesses several continuations of a character at once.  They form a tree: node i of a character
follows its parent, a node of the same character with a smaller index, or the last live token (parent -1).  One step runs
all nodes through every layer, judges the guesses against the model's own probabilities, and commits one path from a root:

  attn     draft_attn: a node attends to the character's whole cache, to its ancestors and to itself, rotated at the
           position p + depth; its keys and values wait behind the live entries
  gdn      draft_gdn: a node's gated-delta-rule output from the carried state advanced along its ancestors and itself (with
           the short convolution over the same path), the state itself left alone
  verify   draft_verify: which path of the tree the target accepts, and the token that follows it, from given uniforms
  step     draft_begin, every layer's draft_attn or draft_gdn, and draft_commit of a path, as one decoding step makes them

Several characters are packed and ragged: `prefix` and `nodes` are upper ends, lengths are spread below them, and a character
may have no draft at all.  `width` is the most nodes on one level of a tree; 1 is a chain.  Value distributions: q, v ~ N(0, 1),
unit keys, alpha = sigmoid(N(3, 0.5)), beta = sigmoid(N(0, 1)), carried states N(0, 0.2^2).  Target and draft probabilities
are softmaxes of N(0, 3^2) logits, the target's with N(0, 1) added: the draft is right about two times in three.
"""
import math

import numpy as np
import torch

own = False

# the hybrid stack of the library's benchmark, a middle one, and the small test shape
HYBRID = {"hq": 16, "hkv": 2, "d": 256, "rot": 64, "h": 16, "dk": 128, "dv": 128}
MID = {"hq": 16, "hkv": 4, "d": 128, "rot": 128, "h": 8, "dk": 128, "dv": 64}
SMALL = {"hq": 8, "hkv": 2, "d": 64, "rot": 64, "h": 8, "dk": 64, "dv": 64}
THETA = 1.0e4


def _case(kind, shape, **kw):
    c = {"kind": kind, "chars": 1, "prefix": 0, "nodes": 1, "width": 1, "lens": 1}
    if kind in ("attn", "step"):
        c.update({k: shape[k] for k in ("hq", "hkv", "d", "rot")})
    if kind in ("gdn", "step"):
        c.update({k: shape[k] for k in ("h", "dk", "dv")})
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: a chain of five guesses after a short text
        _case("attn", SMALL, name="attn_small", prefix=512, nodes=5),
        # a game character's memory of 8K and a bushy tree of 16
        _case("attn", HYBRID, name="attn_npc", prefix=8192, nodes=16, width=4),
        # a long-lived character, the widest tree
        _case("attn", HYBRID, name="attn_long", prefix=32768, nodes=64, width=8),
        # a population decoding together, ragged memories and trees
        _case("attn", HYBRID, name="attn_population", chars=32, prefix=16384, nodes=24, width=4, lens=3),
        # the delta-rule layer of the same single character
        _case("gdn", HYBRID, name="gdn_npc", nodes=16, width=4, conv=False),
        # eight characters' chains of eight guesses, narrow heads
        _case("gdn", MID, name="gdn_chains", chars=8, nodes=8, lens=5, conv=False),
        # a population's delta-rule layer with its short convolution, trees of up to 64
        _case("gdn", HYBRID, name="gdn_population", chars=32, nodes=64, width=8, lens=3, conv=True),
        # one character's verdict over an odd vocabulary
        _case("verify", None, name="verify_one", nodes=16, width=4, vocab=50001, dtype="f32"),
        # a population's verdicts over a large vocabulary
        _case("verify", None, name="verify_population", chars=32, nodes=24, width=4, lens=3, vocab=131072, dtype="f32"),
        # probabilities that a sampler keeps in 16 bits, wide trees
        _case("verify", None, name="verify_bf16", chars=8, nodes=64, width=8, lens=7, vocab=32768, dtype="bf16"),
        # a whole decoding step of one character through four layers
        _case("step", HYBRID, name="step_npc", layers=4, prefix=8192, nodes=16, width=4, kv=True),
        # a population's step through eight layers
        _case("step", HYBRID, name="step_population", layers=8, chars=16, prefix=4096, nodes=32, width=4, lens=3, kv=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "gdn", "gdn", "gdn", "verify", "verify", "step", "step"])
    shape = rng.choice([HYBRID, HYBRID, MID, SMALL])
    chars = 1 if rng.random() < 0.4 else _log(rng, 2, 32)
    nodes = _log(rng, 1, 64)
    kw = {"chars": chars, "nodes": nodes, "width": rng.choice([1, 2, 3, 4, 8]), "lens": rng.randrange(1, 1 << 20)}
    if kind == "attn":
        # no more query-key pairs than the largest listed call
        prefix = _log(rng, 64, min(32768, max(2048, 12_000_000 // (nodes * chars))))
        return _case(kind, shape, prefix=prefix, **kw)
    if kind == "gdn":
        return _case(kind, shape, conv=rng.random() < 0.5, **kw)
    if kind == "verify":
        vocab = _log(rng, 300, min(131072, max(1000, 100_000_000 // (nodes * chars))))
        return _case(kind, None, vocab=vocab, dtype=rng.choice(["f32", "f32", "bf16"]), **kw)
    kw["chars"] = min(chars, 8)
    prefix = _log(rng, 64, 8192 if chars == 1 else 2048)
    return _case(kind, shape, layers=rng.choice([2, 4]), prefix=prefix, kv=kw["chars"] == 1, **kw)


# ---------------------------------------------------------------------------- sizes and trees of a case
def _lengths(case):
    """(live entries, nodes) per character."""
    n, hi_l, hi_n = case["chars"], case["prefix"], case["nodes"]
    if n == 1:
        return [hi_l], [hi_n]
    r = np.random.default_rng(case["lens"])
    L = [int(x) for x in r.integers(hi_l // 8, hi_l + 1, size=n)]
    return L, [hi_n] + [int(x) for x in r.integers(0, hi_n + 1, size=n - 1)]


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


def _paths(case):
    """Per character a path from its root: what a verdict may have accepted."""
    r = np.random.default_rng([case["lens"], 78])
    out = []
    for parent in _trees(case):
        path = []
        while len(path) < len(parent):
            nxt = [i for i, p in enumerate(parent) if p == (path[-1] if path else -1)]
            if not nxt or (path and r.random() < 0.2):
                break
            path.append(int(r.choice(nxt)))
        out.append(path)
    return out


def _kinds(layers):
    """Truth values: is the layer an attention layer?  Three delta-rule layers to one (one to one in a stack of two)."""
    return [i % 4 == 3 or (layers == 2 and i == 1) for i in range(layers)]


def _cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _plan(case):
    """The trees as index tables, padded to the largest: packed rows, truth values, depths, and for the convolution the rows
    (of three carried inputs and the nodes) that each node's four taps read."""
    L, N = _lengths(case)
    n = max(N)
    cu, trees = _cu(N), _trees(case)
    row = np.zeros((len(N), n), np.int64)
    real = np.zeros((len(N), n), bool)
    anc = np.zeros((len(N), n, n), bool)
    depth = np.zeros((len(N), n), np.int64)
    taps = np.zeros((len(N), n, 4), np.int64)
    par = np.full((len(N), n), -1, np.int64)
    rank = np.full((len(N), n), -1, np.int64)            # place among its siblings
    kids = np.zeros((len(N), n), np.int64)
    for b, parent in enumerate(trees):
        m = len(parent)
        row[b, :m] = cu[b] + np.arange(m)
        real[b, :m] = True
        anc[b, :m, :m] = _ancestors(parent)
        depth[b, :m] = anc[b, :m, :m].sum(1) - 1
        par[b, :m] = parent
        for i, p in enumerate(parent):
            taps[b, i, 3] = 3 + i
            taps[b, i, :3] = taps[b, p, 1:] if p >= 0 else [0, 1, 2]
            if p >= 0:
                rank[b, i] = kids[b, p]
                kids[b, p] += 1
    dev = lambda x: torch.as_tensor(x).cuda()
    return {"row": dev(row), "real": dev(real), "anc": dev(anc), "depth": dev(depth), "taps": dev(taps), "par": dev(par),
            "rank": dev(rank), "kids": dev(kids), "live": dev(np.array(L, np.int64)), "most": int(kids.max()),
            "flat": dev(np.flatnonzero(real.reshape(-1)))}


# ---------------------------------------------------------------------------- inputs
def _gen(seed, k):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + k)


def _normal(g, *shape, unit=False):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if unit:
        x = x / x.norm(dim=-1, keepdim=True)
    return x.to(torch.bfloat16)


def _attn_parts(case, g):
    """A layer's inputs and every character's cache, [chars][hkv][longest][d]."""
    L, N = _lengths(case)
    m, lmax, d = sum(N), max(L), case["d"]
    return {"q": _normal(g, m, case["hq"], d), "k": _normal(g, m, case["hkv"], d, unit=True),
            "v": _normal(g, m, case["hkv"], d), "K": _normal(g, len(L), case["hkv"], lmax, d, unit=True),
            "V": _normal(g, len(L), case["hkv"], lmax, d)}


def _gdn_parts(case, g, conv):
    N = _lengths(case)[1]
    m, h, dk, dv = sum(N), case["h"], case["dk"], case["dv"]
    gate = lambda mean, std: torch.sigmoid(mean + std * torch.randn((m, h), generator=g, device="cuda"))
    x = {"q": _normal(g, m, h, dk), "k": _normal(g, m, h, dk, unit=True), "v": _normal(g, m, h, dv),
         "alpha": gate(3.0, 0.5), "beta": gate(0.0, 1.0),
         "S": 0.2 * torch.randn((len(N), h, dv, dk), generator=g, device="cuda")}
    if conv:
        ch = h * (2 * dk + dv)
        x["w"] = 0.5 * torch.randn((ch, 4), generator=g, device="cuda")
        x["old"] = _normal(g, len(N), 3, ch)
    return x


def _verify_parts(case, g):
    """Probabilities after every node, the drafted tokens (each drawn from the draft's row of its parent), uniforms."""
    N, v = _lengths(case)[1], case["vocab"]
    m, cu, trees = sum(N), _cu(N), _trees(case)
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    logits = 3.0 * torch.randn((m, v), generator=g, device="cuda")
    draft = torch.softmax(logits, -1).to(dt)
    target = torch.softmax(logits.add_(torch.randn((m, v), generator=g, device="cuda")), -1).to(dt)
    parent_row = np.concatenate([np.maximum(np.array(t, np.int64), 0) + cu[b] for b, t in enumerate(trees) if t])
    want = torch.rand((m, 1), generator=g, device="cuda", dtype=torch.float64)
    cum = torch.cumsum(draft.double(), -1)[torch.as_tensor(parent_row).cuda()]
    tokens = torch.searchsorted(cum, want * cum[:, -1:]).clamp_(max=v - 1).to(torch.int32).reshape(-1)
    return {"target": target, "draft": draft, "tokens": tokens,
            "u": torch.rand((m,), generator=g, device="cuda"), "u_next": torch.rand((len(N),), generator=g, device="cuda")}


def _parts(case, seed):
    kind = case["kind"]
    if kind == "attn":
        return [_attn_parts(case, _gen(seed, 0))]
    if kind == "gdn":
        return [_gdn_parts(case, _gen(seed, 0), case["conv"])]
    if kind == "verify":
        return [_verify_parts(case, _gen(seed, 0))]
    return [_attn_parts(case, _gen(seed, i)) if a else _gdn_parts(case, _gen(seed, i), False)
            for i, a in enumerate(_kinds(case["layers"]))]


def prepare(case, seed):
    parts = _parts(case, seed)
    s = {"case": case, "parts": parts, "plan": _plan(case)}
    if case["kind"] == "step":
        L, N = _lengths(case)
        paths = _paths(case)
        on = np.zeros((len(N), max(N)), bool)
        for b, path in enumerate(paths):
            on[b, path] = True
        s["on"] = torch.as_tensor(on).cuda()
        s["accepted"] = torch.as_tensor([len(p) for p in paths]).cuda()
        s["cursor"] = torch.as_tensor(L).cuda()
        if case["kv"]:
            s["path"] = torch.as_tensor(paths[0], dtype=torch.int64).cuda()
            s["ids"] = torch.arange(L[0], device="cuda", dtype=torch.int32)
    if own:
        s.update(_handle(case, parts))
    torch.cuda.synchronize()
    return s


def _handle(case, parts):
    """The context that a user's program keeps, with its prefixes, and buffers for the answers."""
    from paper_2609_18935_gb300 import kvm
    L, N = _lengths(case)
    get = lambda k, alt: case.get(k, alt)
    kinds = {"attn": [True], "gdn": [False], "verify": [True]}.get(case["kind"]) or _kinds(case["layers"])
    ctx = kvm.Context([kvm.LAYER_ATTN if a else kvm.LAYER_GDN for a in kinds], get("hq", 8), get("hkv", 2), get("d", 64),
                      get("rot", 64), THETA, get("h", 8), get("dk", 64), get("dv", 64),
                      [l + n + 1 for l, n in zip(L, N)], max(1, sum(N)), conv_kernel=4 if get("conv", False) else 0)
    ctx.draft_reserve(sum(N))
    for b, l in enumerate(L):
        ctx.load_prefix(b, l, l, np.arange(l, dtype=np.int32))
    cu, parent = _cu(N), np.concatenate([np.array(t, np.int32) for t in _trees(case)])
    out = []
    for i, (a, x) in enumerate(zip(kinds, parts)):
        if case["kind"] == "verify":
            m = sum(N)
            out.append([torch.empty(n, dtype=torch.int32, device="cuda") for n in (m, len(N), len(N))])
        elif a:
            for b, l in enumerate(L):
                if l:
                    ctx.set_kv(i, b, x["K"][b, :, :l].contiguous(), x["V"][b, :, :l].contiguous())
            out.append(torch.empty_like(x["q"]))
        else:
            ctx.set_state(i, x["S"])
            if "w" in x:
                ctx.set_conv_weights(i, x["w"])
                ctx.set_conv_state(i, x["old"])
            out.append(torch.empty_like(x["v"]))
    h = {"ctx": ctx, "out": out, "tree": (cu, parent)}
    if case["kind"] == "step":
        paths = _paths(case)
        count = [len(p) for p in paths]
        h["commit"] = (_cu(count), np.concatenate([np.array(p, np.int32) for p in paths]))
        # the accepted entries, to be dropped again so that passes chain at one length
        h["drop"] = (_cu([1 if c else 0 for c in count]), np.array([l for l, c in zip(L, count) if c], np.int32),
                     np.array([l + c for l, c in zip(L, count) if c], np.int32))
    else:
        ctx.draft_begin(cu, parent)          # a step's tree is announced once, for all its layers
    return h


# ---------------------------------------------------------------------------- the calls
def _run_own(s):
    case, ctx, out, parts = s["case"], s["ctx"], s["out"], s["parts"]
    kind = case["kind"]
    if kind == "attn":
        x = parts[0]
        ctx.draft_attn(0, x["q"], x["k"], x["v"], out[0])
        return {"out": out[0]}
    if kind == "gdn":
        x = parts[0]
        ctx.draft_gdn(0, x["q"], x["k"], x["v"], x["alpha"], x["beta"], out[0])
        return {"out": out[0]}
    if kind == "verify":
        x = parts[0]
        ctx.draft_verify(x["tokens"], x["target"], x["draft"], x["u"], x["u_next"], *out[0])
        return {"path": out[0][0], "count": out[0][1], "next": out[0][2]}
    ctx.draft_begin(*s["tree"])
    for i, x in enumerate(parts):
        if "K" in x:
            ctx.draft_attn(i, x["q"], x["k"], x["v"], out[i])
        else:
            ctx.draft_gdn(i, x["q"], x["k"], x["v"], x["alpha"], x["beta"], out[i])
    ctx.draft_commit(*s["commit"])
    r = {"out": out, "state": [ctx.get_state(i) for i, x in enumerate(parts) if "S" in x]}
    if case["kv"]:
        r["kv"] = [ctx.get_kv(i, 0) for i, x in enumerate(parts) if "K" in x]
        r["pos"] = ctx.get_positions(0)
    ctx.kv_compact(*s["drop"])
    return r


# ---------------------------------------------------------------------------- the plain form
def _padded(x, plan):
    """Packed rows [sum n][...] as [chars][most nodes][...]; padding repeats some row."""
    return x[plan["row"]]


def _packed(x, plan):
    return x.flatten(0, 1)[plan["flat"]]


def _turned(x, pos, rot):
    """Rows x [chars][n][heads][d] rotated at pos [chars][n]: pairs (i, i + rot/2); the angles in 64 bits."""
    half = rot // 2
    freq = THETA ** (-2.0 * torch.arange(half, device=x.device, dtype=torch.float64) / rot)
    ang = pos.double()[..., None, None] * freq
    c, s = ang.cos().float(), ang.sin().float()
    a, b = x[..., :half], x[..., half:rot]
    return torch.cat([a * c - b * s, b * c + a * s, x[..., rot:]], -1)


def _plain_attn(case, x, plan, cursor):
    """(outputs in bf16, the nodes' rotated keys [chars][n][hkv][d])."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    pos = cursor[:, None] + plan["depth"]
    q = _turned(_padded(x["q"], plan).float(), pos, case["rot"])
    k = _turned(_padded(x["k"], plan).float(), pos, case["rot"])
    v = _padded(x["v"], plan).float()
    chars, n, lmax = q.shape[0], q.shape[1], x["K"].shape[2]
    K = torch.cat([x["K"].float(), k.transpose(1, 2)], 2)
    V = torch.cat([x["V"].float(), v.transpose(1, 2)], 2)
    q = q.view(chars, n, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(chars, hkv, -1, d)
    live = (torch.arange(lmax, device="cuda") < plan["live"][:, None])[:, None, :].expand(-1, n, -1)
    seen = torch.cat([live, plan["anc"]], 2).repeat_interleave(hq // hkv, 1)[:, None]
    w = (q @ K.transpose(2, 3)) * (1.0 / math.sqrt(d))
    w = w.masked_fill_(~seen, -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True).clamp_(min=-3.0e38)).exp_()
    o = (w @ V) / w.sum(-1, keepdim=True).clamp_(min=1e-30)
    o = o.view(chars, hkv, n, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(chars, n, hq, d)
    return _packed(o, plan).to(torch.bfloat16), k


def _plain_conv(case, x, plan):
    """(q, k, v) after the convolution along each node's path, SiLU, and the keys' norm."""
    flat = torch.cat([x[n].flatten(1) for n in ("q", "k", "v")], 1).float()
    rows = torch.cat([x["old"].float(), _padded(flat, plan)], 1)                   # [chars][3 + n][channels]
    at = plan["taps"][..., None].expand(-1, -1, -1, rows.shape[-1])
    near = torch.gather(rows[:, None].expand(-1, at.shape[1], -1, -1), 2, at)
    y = (near * x["w"].t()).sum(2)
    y = y / (1.0 + torch.exp(-y))
    h, dk, dv = case["h"], case["dk"], case["dv"]
    q, k, v = (t.unflatten(-1, (h, -1)) for t in y.split([h * dk, h * dk, h * dv], -1))
    return q, k / (k * k).sum(-1, keepdim=True).sqrt(), v


def _plain_gdn(case, x, plan):
    """(outputs in bf16, U [chars][h][n][dv], keys [chars][h][n][dk], decay from node j to node i [chars][h][n][n]).

    With G_i the product of alpha along the path to node i, R_ij = G_i / G_j for its ancestors j:
    u_i = beta_i (v_i - G_i S k_i - sum over strict ancestors R_ij (k_i . k_j) u_j), o_i = G_i S q_i + sum R_ij (q_i . k_j) u_j."""
    if "w" in x:
        q, k, v = _plain_conv(case, x, plan)
    else:
        q, k, v = (_padded(x[n], plan).float() for n in ("q", "k", "v"))
    q, k, v = (t.transpose(1, 2) for t in (q, k, v))                               # [chars][h][n][..]
    al, be = (_padded(x[n], plan).transpose(1, 2) for n in ("alpha", "beta"))      # [chars][h][n]
    anc = plan["anc"][:, None]
    g = (anc.double() @ al.double().log()[..., None])[..., 0]
    R = torch.where(anc, (g[..., :, None] - g[..., None, :]).exp(), 0.0).float()
    G = g.exp().float()[..., None]
    eye = torch.eye(R.shape[-1], device="cuda")
    A = -(be[..., None] * R * (k @ k.transpose(2, 3)) * (1.0 - eye))               # nilpotent
    rhs = be[..., None] * (v - G * (k @ x["S"].transpose(2, 3)))
    # (1 - A)^-1 = (1 + A)(1 + A^2)(1 + A^4) .. : A^64 = 0
    inv = eye + A
    for _ in range(5):
        A = A @ A
        inv = inv + A @ inv
    U = inv @ rhs
    o = G * (q @ x["S"].transpose(2, 3)) + (R * (q @ k.transpose(2, 3))) @ U
    return _packed(o.transpose(1, 2), plan).to(torch.bfloat16), U, k, R, G


def _plain_verify(case, x, plan):
    """Every node's judgement of its children, in their order: child j is taken where u q(t) Z_j < max(p(t) - c_j q(t), 0),
    Z_0 = 1, c_0 = 0; a child that is not taken leaves the residual max(p - c_{j+1} q, 0), c_1 = 1, c_{j+1} = c_j + Z_j."""
    chars, n = plan["par"].shape
    p, q = (_padded(x[k], plan).double() for k in ("target", "draft"))             # [chars][n][vocab]
    t = _padded(x["tokens"], plan).long()
    u = _padded(x["u"], plan).double()
    c = torch.zeros((chars, n, 1), dtype=torch.float64, device="cuda")
    Z = torch.ones_like(c)
    taken = torch.full((chars, n), -1, dtype=torch.int64, device="cuda")
    node = torch.arange(n, device="cuda")
    of = plan["real"][:, None, :] & (plan["par"][:, None, :] == node[:, None])     # [chars][parent][child]
    for j in range(plan["most"]):
        child = (of & (plan["rank"][:, None, :] == j)).long().argmax(-1)
        here = (plan["kids"] > j) & (taken < 0)
        tok = torch.gather(t, 1, child)[..., None]
        pt, qt = torch.gather(p, 2, tok), torch.gather(q, 2, tok)
        ok = torch.gather(u, 1, child)[..., None] * qt * Z < (pt - c * qt).clamp(min=0)
        taken = torch.where(here & ok[..., 0], child, taken)
        move = (here & (taken < 0))[..., None]
        c1 = torch.where(c == 0, torch.ones_like(c), c + Z)
        Z1 = (p - c1 * q).clamp(min=0).sum(-1, keepdim=True)
        c, Z = torch.where(move, c1, c), torch.where(move, Z1, Z)
    kept = (torch.gather(taken, 1, plan["par"].clamp(min=0)) == node) | (plan["par"] < 0)
    on = plan["real"] & (kept[:, None, :] | ~plan["anc"]).all(-1)                  # every ancestor was taken
    count = on.sum(1)
    order = torch.where(on, node, n).sort(1).values
    path = torch.where(order < n, order, -1)
    last = torch.where(on, node, 0).amax(1)[:, None, None]
    pl, ql = (torch.gather(a, 1, last.expand(-1, 1, a.shape[2]))[:, 0] for a in (p, q))
    w = (pl - torch.gather(c, 1, last)[:, 0] * ql).clamp(min=0)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, pl)
    cum = w.cumsum(-1)
    nxt = (cum <= x["u_next"].double()[:, None] * cum[:, -1:]).sum(-1)
    nxt = torch.where(count > 0, nxt, -1)
    return {"path": _packed(path, plan).int(), "count": count.int(), "next": nxt.int()}


def _run_plain(s):
    case, plan, parts = s["case"], s["plan"], s["parts"]
    kind = case["kind"]
    if kind == "attn":
        return {"out": _plain_attn(case, parts[0], plan, plan["live"])[0]}
    if kind == "gdn":
        return {"out": _plain_gdn(case, parts[0], plan)[0]}
    if kind == "verify":
        return _plain_verify(case, parts[0], plan)
    r = {"out": [], "state": [], "kv": []}
    leaf = (s["on"] * torch.arange(1, s["on"].shape[1] + 1, device="cuda")).amax(1)  # 1 + the path's last node, or 0
    for x in parts:
        if "K" in x:
            out, k = _plain_attn(case, x, plan, s["cursor"])
            if case["kv"]:
                new = (k[0, s["path"]].to(torch.bfloat16), _padded(x["v"], plan)[0, s["path"]])
                r["kv"].append(tuple(torch.cat([x[n][0], y.transpose(0, 1)], 1) for n, y in zip(("K", "V"), new)))
        else:
            out, U, k, R, G = _plain_gdn(case, x, plan)
            at = (leaf - 1).clamp(min=0)[:, None, None, None]
            w = torch.gather(R, 2, at.expand(-1, R.shape[1], 1, R.shape[3])).transpose(2, 3)   # [chars][h][n][1]
            w = w * s["on"][:, None, :, None]
            gl = torch.gather(G, 2, at.expand(-1, G.shape[1], 1, 1))
            gl = torch.where((leaf > 0)[:, None, None, None], gl, torch.ones_like(gl))
            x["S"] = gl * x["S"] + (w * U).transpose(2, 3) @ k
            r["state"].append(x["S"])
        r["out"].append(out)
    if case["kv"]:
        r["pos"] = torch.cat([s["ids"], (s["cursor"] + torch.arange(len(s["path"]), device="cuda")).int()])
    else:
        del r["kv"]
    s["cursor"] = s["cursor"] + s["accepted"]
    return r


def run(s):
    if own:
        return _run_own(s)
    return _run_plain(s)


# ---------------------------------------------------------------------------- work of a pass
def _attn_work(case):
    L, N = _lengths(case)
    m, hq, hkv, d = sum(N), case["hq"], case["hkv"], case["d"]
    pairs = sum(n * l for l, n in zip(L, N)) + sum(int(_ancestors(t).sum()) for t in _trees(case) if t)
    # the caches once, the nodes' q, k, v in, the outputs and the nodes' keys and values out
    return sum(l for l, n in zip(L, N) if n) * hkv * d * 4 + m * (2 * hq + 4 * hkv) * d * 2, 4 * d * hq * pairs


def _gdn_work(case, conv):
    N = _lengths(case)[1]
    m, act, h, dk, dv = sum(N), sum(1 for x in N if x), case["h"], case["dk"], case["dv"]
    pairs = sum(int(_ancestors(t).sum()) for t in _trees(case) if t)
    b = m * h * ((2 * dk + 2 * dv) * 2 + 8) + act * h * dv * dk * 4
    f = h * (4 * dk * dv * m + pairs * (4 * dk + 4 * dv))
    if conv:
        ch = h * (2 * dk + dv)
        b += ch * 16 + act * 3 * ch * 2
        f += 8 * ch * m
    return b, f


def work(case):
    kind = case["kind"]
    if kind == "attn":
        b, f = _attn_work(case)
    elif kind == "gdn":
        b, f = _gdn_work(case, case["conv"])
    elif kind == "verify":
        # whatever the verdict: the row that the next token is drawn from, and the draft's beside it where a guess failed
        N = _lengths(case)[1]
        act = sum(1 for x in N if x)
        b = act * 2 * case["vocab"] * (4 if case["dtype"] == "f32" else 2) + sum(N) * 16
        f = act * 4 * case["vocab"]
    else:
        kinds = _kinds(case["layers"])
        n_attn, n_gdn = sum(kinds), len(kinds) - sum(kinds)
        (ab, af), (gb, gf) = _attn_work(case), _gdn_work(case, False)
        paths = _paths(case)
        act, rows = sum(1 for p in paths if p), sum(len(p) for p in paths)
        state = case["h"] * case["dk"] * case["dv"]
        b = n_attn * ab + n_gdn * (gb + 4 * act * state)
        f = n_attn * af + n_gdn * (gf + 2 * rows * state)
    return {"bytes": float(b), "flops": float(f)}


# ---------------------------------------------------------------------------- the same in 64 bits
def _exact_attn(case, x, cursors):
    """Node by node groups of one character and KV head: (out, keys [hkv][live + n][d], values) per character."""
    L, N = _lengths(case)
    g, d, rot = case["hq"] // case["hkv"], case["d"], case["rot"]
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    freq = torch.exp(-math.log(THETA) * 2.0 * i / rot)
    outs, after, at = [], [], 0
    for b, (l, n, parent) in enumerate(zip(L, N, _trees(case))):
        if not n:
            after.append(None)
            continue
        anc = torch.as_tensor(_ancestors(parent)).cuda()
        turn = torch.polar(torch.ones_like(freq), 0 * freq) * torch.exp(1j * (cursors[b] + anc.sum(1) - 1)[:, None, None] * freq)

        def rotate(y):
            z = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * turn
            return torch.cat([z.real, z.imag, y[..., rot:]], -1)
        q, k = rotate(x["q"][at:at + n].double()), rotate(x["k"][at:at + n].double())
        K = torch.cat([x["K"][b, :, :l].double(), k.transpose(0, 1)], 1)
        V = torch.cat([x["V"][b, :, :l].double(), x["v"][at:at + n].double().transpose(0, 1)], 1)
        bias = torch.zeros((n, l + n), dtype=torch.float64, device="cuda")
        bias[:, l:][~anc] = -math.inf
        o = torch.empty_like(q)
        for h in range(case["hkv"]):
            w = torch.softmax(torch.einsum("igd,jd->gij", q[:, h * g:(h + 1) * g], K[h]) / math.sqrt(d) + bias, -1)
            o[:, h * g:(h + 1) * g] = torch.einsum("gij,jd->igd", w, V[h])
        outs.append(o)
        after.append((K, V))
        at += n
    return torch.cat(outs), after


def _exact_gdn(case, x, S, keep=None):
    """Every node's own state from its parent's: (out, the states after the paths `keep`, S where a path is empty)."""
    N = _lengths(case)[1]
    x = {n: y.double() for n, y in x.items()}
    after = S.double().clone()
    out, at = torch.empty_like(x["v"]), 0
    for b, parent in enumerate(_trees(case)):
        states, pasts = {-1: S[b].double()}, {-1: x["old"][b] if "old" in x else None}
        for i, p in enumerate(parent):
            r = at + i
            q, k, v = x["q"][r], x["k"][r], x["v"][r]
            if "w" in x:
                pasts[i] = torch.cat([pasts[p], torch.cat([q.flatten(), k.flatten(), v.flatten()])[None]])
                y = (pasts[i][-4:] * x["w"].t()).sum(0)
                y = y * torch.sigmoid(y)
                q, k, v = (t.view(u.shape) for t, u in zip(y.split([q.numel(), k.numel(), v.numel()]), (q, k, v)))
                k = k / k.norm(dim=-1, keepdim=True)
            a, be = x["alpha"][r][:, None], x["beta"][r][:, None]
            T = a[..., None] * states[p]
            T = T + (be * (v - (T @ k[..., None])[..., 0]))[..., None] * k[:, None, :]
            out[r] = (T @ q[..., None])[..., 0]
            states[i] = T
        if keep is not None and keep[b]:
            after[b] = states[keep[b][-1]]
        at += len(parent)
    return out, after


def _exact_verify(case, x):
    """The walk itself, a character at a time, on the host."""
    N = _lengths(case)[1]
    paths, counts, nexts, at = [], [], [], 0
    tok, u, last_u = (x[k].cpu().numpy().astype(np.float64) for k in ("tokens", "u", "u_next"))
    row = lambda y, i: y[at + i].double().cpu().numpy()
    for b, parent in enumerate(_trees(case)):
        path = [0] if parent else []
        while path:
            p, q, Z, step = row(x["target"], path[-1]), row(x["draft"], path[-1]), 1.0, None
            full = p
            for i in (j for j, up in enumerate(parent) if up == path[-1]):
                t = int(tok[at + i])
                if u[at + i] * q[t] < p[t] / Z:
                    step = i
                    break
                p = np.maximum(p / Z - q, 0.0) * Z          # the residual, in the first row's units
                Z = math.fsum(p)
                if Z <= 0.0:
                    break
            if step is None:
                w = p if math.fsum(p) > 0.0 else full
                cum = np.cumsum(w.astype(np.longdouble))
                nexts.append(int(np.searchsorted(cum, np.longdouble(last_u[b]) * cum[-1], side="right")))
                break
            path.append(step)
        if not path:
            nexts.append(-1)
        counts.append(len(path))
        paths += path + [-1] * (len(parent) - len(path))
        at += len(parent)
    whole = lambda y: torch.as_tensor(np.array(y, np.int32))
    return {"path": whole(paths), "count": whole(counts), "next": whole(nexts)}


def exact(case, seed):
    parts, kind = _parts(case, seed), case["kind"]
    L = _lengths(case)[0]
    if kind == "attn":
        return {"out": _exact_attn(case, parts[0], L)[0]}
    if kind == "gdn":
        return {"out": _exact_gdn(case, parts[0], parts[0]["S"])[0]}
    if kind == "verify":
        return _exact_verify(case, parts[0])
    paths = _paths(case)
    r = {"out": [], "state": [], "kv": []}
    for x in parts:
        if "K" in x:
            out, after = _exact_attn(case, x, L)
            if case["kv"]:
                rows = list(range(L[0])) + [L[0] + i for i in paths[0]]
                r["kv"].append(tuple(t[:, rows] for t in after[0]))
        else:
            out, S = _exact_gdn(case, x, x["S"], paths)
            r["state"].append(S)
        r["out"].append(out)
    if case["kv"]:
        r["pos"] = None
    else:
        del r["kv"]
    return r
