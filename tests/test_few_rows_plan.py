"""The partition of few rows over windowed layers and 8-bit caches (kvm_plan_attention_few), which one launch runs."""
import numpy as np
import pytest

from paper_2609_18935_gb300 import kvm

CASES = [(16, 2), (8, 2), (8, 8), (16, 1), (4, 4)]


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    from paper_2609_18935_gb300 import build_lib
    if not os.path.exists(kvm.LIB_PATH):
        build_lib.build()
    kvm.load_library()


def _units(L, n, window, sinks):
    """64-key tiles of n tokens behind L entries: those of the sinks, and those from the first token's oldest key on."""
    f = max(0, L + 1 - window) // 64 if window else 0
    return -(-(L + n) // 64) - f + min(-(-sinks // 64), f)


def _ranges(plan):
    """Per query tile the (first, last + 1 or None for all, block) that the blocks take, and per block its (units, segments)."""
    n, waves, tile, key = plan["n_blocks"], plan["n_waves"], plan["block_tile"], plan["block_key"]
    done = [[] for _ in range(plan["n_tiles"])]
    for c in range(n):
        for w in range(waves):
            done[w * n + (n - 1 - c if w & 1 else c)].append((0, None, c))
        (t0, k0), (t1, k1) = (tile[c], key[c]), (tile[c + 1], key[c + 1])
        for t in range(t0, t1 + (1 if k1 > 0 else 0)):
            a, e = (k0 if t == t0 else 0), (k1 if t == t1 else None)
            if (t0, k0) != (t1, k1):
                done[t].append((a, e, c))
    return done


@pytest.mark.parametrize("row_bytes", [64, 128, 256, 512])
@pytest.mark.parametrize("heads", CASES)
def test_every_unit_once(row_bytes, heads):
    rng = np.random.default_rng([row_bytes, *heads])
    seen = {"waves": 0, "split": 0, "whole": 0, "gap": 0, "two_new_blocks": 0}
    hq, hkv = heads
    most = 16 // (hq // hkv)
    for trial in range(60):
        B = int(rng.integers(1, [6, 40, 200][trial % 3]))
        live = [int(rng.integers(0, [60000, 5000, 200][trial % 3])) for _ in range(B)]
        tails = [int(rng.integers(0, most + 1)) for _ in range(B)]
        tails[0] = max(tails[0], 1)
        window, sinks = [(0, 0), (1, 0), (100, 4), (4096, 70), (2 ** 31 - 1, 0)][trial % 5]
        G = int(rng.choice([1, 7, 152, 320]))
        plan = kvm.plan_attention_few(live, np.concatenate([[0], np.cumsum(tails)]), hq, hkv, row_bytes, window, sinks, G)
        assert 1 <= plan["n_blocks"] <= G
        done, t, splits, load = _ranges(plan), 0, [], np.zeros(plan["n_blocks"])
        want = [_units(L, n, window, sinks) for L, n in zip(live, tails) if n for _ in range(hkv)]
        assert plan["n_tiles"] == len(want)
        for parts, nk in zip(done, want):
            parts = sorted((a, nk if e is None else e, c) for a, e, c in parts)
            assert [p[0] for p in parts] == [0] + [p[1] for p in parts[:-1]] and parts[-1][1] == nk
            assert all(a < e for a, e, _ in parts)
            # parts of a tile belong to blocks in a row: that is how the merge finds them
            assert [p[2] for p in parts] == list(range(parts[0][2], parts[0][2] + len(parts)))
            for a, e, c in parts:
                load[c] += e - a + 4096 / row_bytes
            if len(parts) > 1:
                splits.append(parts[1][2])
        assert sorted(plan["split_first_block"].tolist()) == splits
        whole = max(want) <= 1280 // row_bytes and len(want) <= G
        if whole:
            assert plan["n_blocks"] == len(want) and not splits
        else:
            assert plan["n_blocks"] == max(1, min(G, sum(want) // max(1, 512 // row_bytes)))
            # no block far over its share: a cut falls within a unit of the target, which all blocks' segments bound
            share = (sum(want) + 4096 / row_bytes * (len(want) + plan["n_blocks"])) / plan["n_blocks"]
            assert load.max() <= share + 2 * 4096 / row_bytes + 2 or plan["n_waves"]
        seen["waves"] += plan["n_waves"] > 0
        seen["split"] += bool(splits)
        seen["whole"] += whole
        seen["gap"] += window > 0 and any(L >= window + 64 for L in live)
        seen["two_new_blocks"] += any(n > 1 and L // 64 < (L + n - 1) // 64 for L, n in zip(live, tails))
    if most == 1:
        del seen["two_new_blocks"]
    assert min(seen.values()) >= 2, seen


def test_units_and_segments_weigh_by_a_rows_bytes():
    """One long character: a block has 512 bytes of rows at least; short lists stay whole up to 1280."""
    for row_bytes, live in ((64, 64 * 40), (128, 64 * 40), (256, 64 * 40), (512, 64 * 40)):
        plan = kvm.plan_attention_few([live], [0, 1], 8, 1, row_bytes, 0, 0, 152)
        assert plan["n_blocks"] == 41 // max(1, 512 // row_bytes)
        whole = 1280 // row_bytes
        assert kvm.plan_attention_few([64 * whole - 1], [0, 1], 8, 1, row_bytes, 0, 0, 152)["n_blocks"] == 1
        assert kvm.plan_attention_few([64 * whole], [0, 1], 8, 1, row_bytes, 0, 0, 152)["n_blocks"] == (whole + 1) // max(1, 512 // row_bytes)


def test_a_window_over_everything_is_no_window():
    live, cu = [7782, 300, 0], [0, 2, 3, 5]
    a = kvm.plan_attention_few(live, cu, 16, 2, 256, 0, 0, 152)
    b = kvm.plan_attention_few(live, cu, 16, 2, 256, 10 ** 6, 0, 152)
    assert all(np.array_equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("kw,code", [({"row_bytes": 96}, kvm.KVM_E_UNSUPPORTED), ({"row_bytes": 1024}, kvm.KVM_E_UNSUPPORTED),
                                     ({"cu": [0, 3]}, kvm.KVM_E_UNSUPPORTED), ({"hq": 64}, kvm.KVM_E_UNSUPPORTED),
                                     ({"window": -1}, kvm.KVM_E_INVAL), ({"sinks": 3}, kvm.KVM_E_INVAL), ({"cu": [0, -1]}, kvm.KVM_E_INVAL),
                                     ({"live": [2 ** 31 - 1]}, kvm.KVM_E_INVAL), ({"G": 0}, kvm.KVM_E_INVAL), ({"G": 321}, kvm.KVM_E_INVAL)])
def test_refusals(kw, code):
    a = {"live": [100], "cu": [0, 2], "hq": 16, "row_bytes": 256, "window": 0, "sinks": 0, "G": 152}
    a.update(kw)
    with pytest.raises(kvm.KvmError) as e:
        kvm.plan_attention_few(a["live"], a["cu"], a["hq"], 2, a["row_bytes"], a["window"], a["sinks"], a["G"])
    assert e.value.code == code
