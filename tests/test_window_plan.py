"""The partition of a windowed layer's attention (kvm_plan_attention_window), and the refusals that need no GPU."""
import numpy as np
import pytest

from paper_2609_18935_gb300 import kvm


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    from paper_2609_18935_gb300 import build_lib
    if not os.path.exists(kvm.LIB_PATH):
        build_lib.build()
    kvm.load_library()


def _key_tiles(L, tok0, tok1, window, sinks):
    """By the definition, key by key: the 64-key tiles that some token tok0 <= i < tok1 at live index L + i has a key in, and
    every tile from the first of those that are not sinks on (a row's window reaches to its own tile)."""
    want = set()
    for i in (tok0, tok1 - 1) if tok1 - tok0 > 1 else (tok0,):
        x = L + i
        lo = max(0, x - window + 1)
        want |= set(range(lo // 64, x // 64 + 1)) | set(range(0, -(-min(sinks, lo) // 64)))
    return want


def _mapped(L, tok0, nk, window, sinks):
    """The key tiles of a query tile's units, as kvm.h says."""
    f = max(0, L + tok0 + 1 - window) // 64
    s = min(-(-sinks // 64), f)
    return [u if u < s else u + f - s for u in range(nk)]


def _walk(live, tails, Hq, Hkv, window, sinks, G):
    """Per query tile the units that the blocks take, in order: as in kvm_plan_attention_launch."""
    cu = np.concatenate([[0], np.cumsum(tails)])
    plan = kvm.plan_attention_window(live, cu, Hq, Hkv, window, sinks, G)
    done = [[] for _ in range(plan["n_tiles"])]
    n, waves, tile, key = plan["n_blocks"], plan["n_waves"], plan["block_tile"], plan["block_key"]
    for c in range(n):
        for w in range(waves):
            done[w * n + (n - 1 - c if w & 1 else c)].append((0, None, c))
        (t0, k0), (t1, k1) = (tile[c], key[c]), (tile[c + 1], key[c + 1])
        for t in range(t0, t1 + (1 if k1 > 0 else 0)):
            done[t].append((k0 if t == t0 else 0, k1 if t == t1 else None, c))
    return plan, done


def test_windowed_plan_covers_every_tile_once():
    rng = np.random.default_rng(91)
    seen = {"gap": 0, "sinks": 0, "waves": 0, "split": 0, "whole": 0}
    for trial in range(300):
        B = int(rng.integers(1, 20))
        live = [int(rng.integers(0, [20000, 300, 5000][trial % 3])) for _ in range(B)]
        tails = [int(rng.integers(0, [300, 900, 3][trial % 3])) for _ in range(B)]
        tails[0] = max(tails[0], 1)
        window = int(rng.choice([1, 2, 63, 64, 65, 100, 1000, 4096, 2 ** 31 - 1]))
        sinks = int(rng.choice([0, 1, 4, 64, 65, 1000, 2 ** 31 - 1]))
        Hq, Hkv = [(16, 2), (8, 2), (8, 8), (64, 1)][trial % 4]
        G = int(rng.choice([1, 7, 152, 320]))
        plan, done = _walk(live, tails, Hq, Hkv, window, sinks, G)
        tpt, t, splits = 128 // (Hq // Hkv), 0, []
        for b in range(B):
            for h in range(Hkv):
                for tok0 in range(0, tails[b], tpt):
                    tok1 = min(tails[b], tok0 + tpt)
                    want = _key_tiles(live[b], tok0, tok1, window, sinks)
                    last = (live[b] + tok1 - 1) // 64
                    nk = last + 1 - (max(0, live[b] + tok0 + 1 - window) // 64 - min(-(-sinks // 64), max(0, live[b] + tok0 + 1 - window) // 64))
                    parts = sorted((a, nk if e is None else e, c) for a, e, c in done[t])
                    assert [p[0] for p in parts] == [0] + [p[1] for p in parts[:-1]] and parts[-1][1] == nk
                    tiles = _mapped(live[b], tok0, nk, window, sinks)
                    assert tiles == sorted(set(tiles)) and set(tiles) >= want and tiles[-1] == last
                    # nothing beyond what the first row sees and the sinks
                    assert all(x >= max(0, live[b] + tok0 + 1 - window) // 64 or 64 * x < sinks for x in tiles)
                    seen["gap"] += len(tiles) <= last
                    seen["sinks"] += 0 < sinks <= 64 and len(tiles) <= last
                    if len(parts) > 1:
                        splits.append(parts[1][2])
                    t += 1
        assert t == plan["n_tiles"] and sorted(plan["split_first_block"].tolist()) == splits
        seen["waves"] += plan["n_waves"] > 0
        seen["split"] += bool(splits)
        seen["whole"] += plan["n_blocks"] == plan["n_tiles"] and not splits
    assert min(seen.values()) >= 5, seen


def test_a_window_over_everything_is_the_whole_plan():
    live, cu = [7782, 300, 0], [0, 256, 300, 365]
    a = kvm.plan_attention_launch(live, cu, 16, 2, 152)
    b = kvm.plan_attention_window(live, cu, 16, 2, 10 ** 6, 0, 152)
    c = kvm.plan_attention_window(live, cu, 16, 2, 0, 0, 152)
    for x in (b, c):
        assert all(np.array_equal(a[k], x[k]) for k in a)


@pytest.mark.parametrize("window,sinks", [(-1, 0), (4, -1), (0, 4)])
def test_bad_windows_are_refused(window, sinks):
    with pytest.raises(kvm.KvmError) as e:
        kvm.plan_attention_window([100], [0, 5], 16, 2, window, sinks, 152)
    assert e.value.code == kvm.KVM_E_INVAL
    assert kvm.load_library().kvm_set_window(None, 0, 64, 0) == kvm.KVM_E_INVAL


@pytest.mark.parametrize("live,cu", [([2 ** 31 - 1], [0, 5]), ([2 ** 31 - 133], [0, 5]), ([0], [0, 2 ** 31 - 1]), ([5, 2 ** 31 - 130], [0, 7, 9])])
def test_lengths_past_32_bits_are_refused(live, cu):
    """A key list ends at live + tail, rounded up to whole tiles in 32 bits."""
    for call in (lambda: kvm.plan_attention(live, cu, 16, 2, 152), lambda: kvm.plan_attention_launch(live, cu, 16, 2, 152),
                 lambda: kvm.plan_attention_window(live, cu, 16, 2, 1000, 4, 152)):
        with pytest.raises(kvm.KvmError) as e:
            call()
        assert e.value.code == kvm.KVM_E_INVAL


def test_the_longest_lengths_are_planned():
    L, n = 2 ** 31 - 134, 5
    nk = -(-(L + n) // 64)
    plan = kvm.plan_attention_launch([L], [0, n], 16, 2, 152)
    assert plan["n_blocks"] == 152 and abs(plan["block_key"][1] - 2 * nk / 152) < 10
    # in a window's sight: its 64-key tiles and one of sinks
    f = (L + 1 - 1000) // 64
    plan = kvm.plan_attention_window([L], [0, n], 16, 2, 1000, 4, 152)
    assert plan["n_tiles"] == 2 and 1 <= plan["n_blocks"] <= 2 * (nk - f + 1) // 4


def test_tiles_past_32_bits_are_refused():
    with pytest.raises(kvm.KvmError) as e:
        kvm.plan_attention_launch([0], [0, 2 ** 31 - 129], 64 * 64, 64, 152)
    assert e.value.code == kvm.KVM_E_INVAL
