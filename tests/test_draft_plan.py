"""Drafted-token trees on the host: the library's planning and refusals, and the oracle's tree functions."""
import ctypes as C

import numpy as np
import pytest

from oracle import kvm_oracle as O


@pytest.fixture(scope="module")
def kvm():
    import os
    from paper_2609_18935_gb300 import build_lib, kvm
    if not os.path.exists(kvm.LIB_PATH):
        build_lib.build()
    kvm.load_library()
    return kvm


def _tree(r, n, roots=1):
    return [-1 if i < roots else int(r.integers(0, i)) for i in range(n)]


def test_ancestor_words_and_depths(kvm):
    r = np.random.default_rng(1)
    for _ in range(50):
        trees = [_tree(r, int(r.integers(0, 65)), int(r.integers(1, 4))) for _ in range(int(r.integers(1, 9)))]
        trees.append(list(range(-1, 63)))                       # a chain of 64
        cu = np.concatenate([[0], np.cumsum([len(t) for t in trees])])
        depth, anc = kvm.plan_draft(cu, sum(trees, []))
        for b, t in enumerate(trees):
            for i in range(len(t)):
                path = O.draft_path(t, i)
                assert depth[cu[b] + i] == len(path) - 1
                assert int(anc[cu[b] + i]) == sum(1 << j for j in path)


@pytest.mark.parametrize("cu,parent,code", [
    ([0, 2], [-1, 1], 1),              # its own parent
    ([0, 2], [-1, 2], 1),              # a later one
    ([0, 2], [-1, -2], 1),
    ([0, 1], [0], 1),
    ([1, 2], [-1, -1], 1),             # offsets do not start at 0
    ([0, 2, 1], [-1], 1),              # not monotone
    ([0, 65], [-1] * 65, 6),           # more nodes than a word has bits
    ([0, 1, 2], [-1, 0], 1),           # the second character's only node has a parent
])
def test_bad_trees_are_refused(kvm, cu, parent, code):
    with pytest.raises(kvm.KvmError) as ei:
        kvm.plan_draft(cu, parent)
    assert ei.value.code == code


@pytest.mark.parametrize("path_cu,path,ok", [
    ([0, 0, 0], [], True),
    ([0, 3, 3], [0, 1, 3], True),
    ([0, 1, 3], [2, 0, 1], True),      # the second root of the first tree; the whole second tree
    ([0, 2, 2], [0, 3], False),        # skips a generation
    ([0, 2, 2], [1, 3], False),        # does not start at a root
    ([0, 2, 2], [0, 0], False),
    ([0, 1, 1], [4], False),           # outside the tree
    ([0, 1, 1], [-1], False),
    ([0, 0, 3], [0, 1, 1], False),     # longer than the tree
    ([0, 2, 1], [0], False),
    ([1, 1, 1], [0], False),
])
def test_paths(kvm, path_cu, path, ok):
    cu, parent = [0, 4, 6], [-1, 0, -1, 1, -1, 0]
    if ok:
        kvm.plan_draft_path(cu, parent, path_cu, path)
    else:
        with pytest.raises(kvm.KvmError) as ei:
            kvm.plan_draft_path(cu, parent, path_cu, path)
        assert ei.value.code == kvm.KVM_E_INVAL


def test_null_arguments_are_refused(kvm):
    lib = kvm.load_library()
    one = (C.c_int32 * 2)(0, 1)
    assert lib.kvm_plan_draft(1, None, None, None, None) == kvm.KVM_E_INVAL
    assert lib.kvm_plan_draft(1, one, None, None, None) == kvm.KVM_E_INVAL
    assert lib.kvm_plan_draft(0, one, one, None, None) == kvm.KVM_E_INVAL
    assert lib.kvm_plan_draft_path(1, one, (C.c_int32 * 1)(-1), None, None) == kvm.KVM_E_INVAL
    assert lib.kvm_draft_reserve(None, 8) == kvm.KVM_E_INVAL
    assert lib.kvm_draft_begin(None, one, one, None) == kvm.KVM_E_INVAL
    assert lib.kvm_draft_attn(None, 0, None, None, None, None, None) == kvm.KVM_E_INVAL
    assert lib.kvm_draft_gdn(None, 0, None, None, None, None, None, None, None) == kvm.KVM_E_INVAL
    assert lib.kvm_draft_verify(None, 8, 0, None, None, None, None, None, None, None, None, None) == kvm.KVM_E_INVAL
    assert lib.kvm_draft_commit(None, one, one, None) == kvm.KVM_E_INVAL


# ---------------------------------------------------------------------------- the oracle's tree functions
def test_a_chain_is_a_tail():
    r = np.random.default_rng(2)
    n, L = 7, 5
    chain = list(range(-1, n - 1))
    cache = O.AttnCache(r.standard_normal((2, L, 8)), r.standard_normal((2, L, 8)), np.arange(L))
    q, k, v = r.standard_normal((n, 4, 8)), r.standard_normal((n, 2, 8)), r.standard_normal((n, 2, 8))
    tail = O.tail_attn_prefill(cache, q, k, v, L, 4, 1e4)[0]
    np.testing.assert_allclose(O.draft_attention(cache, q, k, v, chain, L, 4, 1e4), tail, rtol=1e-13, atol=1e-14)
    gq, gk, gv = r.standard_normal((n, 2, 4)), r.standard_normal((n, 2, 4)), r.standard_normal((n, 2, 3))
    a, b, S = r.random((n, 2)), r.random((n, 2)), r.standard_normal((2, 3, 4))
    o, last = O.gdn_recurrent(gq, gk, gv, a, b, S)
    out, states = O.draft_gdn(gq, gk, gv, a, b, S, chain)
    np.testing.assert_allclose(out, o, rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(states[-1], last, rtol=1e-12, atol=1e-13)


def test_the_tree_form_of_the_delta_rule():
    """u_i = beta_i (v_i - G_i S k_i - sum R_ij (k_i . k_j) u_j) over ancestors gives the nodes' outputs and states."""
    r = np.random.default_rng(3)
    n, dk, dv = 12, 6, 5
    parent = _tree(r, n, 2)
    q, k, v = r.standard_normal((n, 1, dk)), r.standard_normal((n, 1, dk)), r.standard_normal((n, 1, dv))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    a, b, S = r.random((n, 1)), r.random((n, 1)), r.standard_normal((1, dv, dk))
    out, states = O.draft_gdn(q, k, v, a, b, S, parent)
    u = np.zeros((n, dv))
    for i in range(n):
        path = O.draft_path(parent, i)
        G = np.prod(a[path, 0])
        R = {j: np.prod(a[path[x + 1:], 0]) for x, j in enumerate(path)}
        up = path[:-1]
        u[i] = b[i, 0] * (v[i, 0] - G * S[0] @ k[i, 0] - sum(R[j] * (k[i, 0] @ k[j, 0]) * u[j] for j in up))
        o = G * S[0] @ q[i, 0] + sum(R[j] * (q[i, 0] @ k[j, 0]) * u[j] for j in path)
        np.testing.assert_allclose(o, out[i, 0], rtol=1e-11, atol=1e-12)
        np.testing.assert_allclose(G * S[0] + sum(R[j] * np.outer(u[j], k[j, 0]) for j in path), states[i][0], rtol=1e-11,
                                   atol=1e-12)


def test_verdict_by_hand():
    p = np.array([[0.5, 0.3, 0.2], [1.0, 0.0, 0.0], [0.1, 0.2, 0.7]])
    q = np.array([[0.25, 0.5, 0.25], [1.0, 0.0, 0.0], [0.3, 0.3, 0.4]])
    par = [-1, 0, 0]
    # token 1: p / q = 0.6; u below it accepts, and the next token comes from that node's own row
    assert O.draft_verdict(par, [0, 1, 2], p, q, [0, 0.59, 0], 0.99) == ([0, 1], 0)
    # refused: residual (0.25, 0, 0); token 2 has nothing left, so token 0 follows
    assert O.draft_verdict(par, [0, 1, 2], p, q, [0, 0.61, 0], 0.5) == ([0], 0)
    # refused, then token 0 of the residual: 0.25 / 0.25 against q = 0.25: always accepted
    assert O.draft_verdict(par, [0, 1, 0], p, q, [0, 0.61, 0.999], 0.8) == ([0, 2], 2)
    # a leaf: inverse distribution of its row
    for un, x in ((0.0, 0), (0.09, 0), (0.11, 1), (0.31, 2), (0.999, 2)):
        assert O.draft_verdict(par, [0, 1, 0], p, q, [0, 0.61, 0.5], un)[1] == x
    # a row of zeros holds nothing
    assert O.draft_verdict([-1], [0], np.zeros((1, 3)), q[:1], [0], 0.5) == ([0], -1)


def test_verdict_keeps_the_targets_distribution():
    """By enumeration over tokens and uniforms: one root with two guesses drawn from q, five tokens; the first token that
    follows the root is distributed as p."""
    r = np.random.default_rng(4)
    V = 5
    p, q = r.random(V), r.random(V)
    p, q = p / p.sum(), q / q.sum()
    got = np.zeros(V)
    for x in range(V):
        a = min(1.0, p[x] / q[x])                       # accepted outright
        got[x] += q[x] * a
        if a == 1.0:
            continue
        w = np.maximum(p - q, 0)
        w = w / w.sum()
        for y in range(V):
            a2 = min(1.0, w[y] / q[y])
            got[y] += q[x] * (1 - a) * q[y] * a2
            w2 = np.maximum(w - q, 0)
            if a2 < 1.0:
                got += q[x] * (1 - a) * q[y] * (1 - a2) * (w2 / w2.sum() if w2.sum() > 0 else w)
    np.testing.assert_allclose(got, p, atol=1e-12)
    # and the verdict takes those steps: thresholds on both sides
    for x in range(V):
        for y in range(V):
            a = p[x] / q[x]
            rows = np.stack([p, p, p])
            qs = np.stack([q, q, q])
            if a < 1.0:
                assert O.draft_verdict([-1, 0, 0], [0, x, y], rows, qs, [0, a * (1 - 1e-9), 0], 0.5)[0] == [0, 1]
                assert 1 not in O.draft_verdict([-1, 0, 0], [0, x, y], rows, qs, [0, min(1, a * (1 + 1e-9)), 0.999999], 0.5)[0]
