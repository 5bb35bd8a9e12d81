// The attention's work list on the device: query tiles, the 64-key tiles of each, and
// the segments of them that a block walks.
#pragma once

#include "kvm_internal.cuh"

namespace kvm {

constexpr int kAttnKeys = 64;                  // keys of a unit

struct Tile {
    int b, kvh, qt, nk, tok0, tok_end;
    int sink, gap;                            // units below `sink` are the key tiles of their number, the others' lie `gap` further on
};

// Query tile t -> (character, KV head, tile within the head) and its number
// of 64-key tiles (every surviving entry plus the tail up to its last token, less
// those that a window leaves out).
template <bool WIN, bool TREE>
__device__ __forceinline__ Tile decode_tile(const AttnParams& p, int t) {
    int lo = 0, hi = p.n_chars - 1;               // last b with tile_off <= t
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.ch[mid].tile_off <= t) lo = mid; else hi = mid - 1;
    }
    Tile r;
    r.b = lo;
    const AttnChar& c = p.ch[lo];
    const int local = t - c.tile_off;
    r.kvh = local / c.n_qtiles;
    r.qt = local % c.n_qtiles;
    r.tok0 = r.qt * p.tok_per_tile;
    r.tok_end = min(c.M, r.tok0 + p.tok_per_tile);
    r.nk = (c.L_prev + r.tok_end + kAttnKeys - 1) / kAttnKeys;
    r.sink = r.gap = 0;
    if (WIN) {
        const WindowTiles w = window_tiles(c.L_prev + (TREE ? 0 : r.tok0), p.window, p.n_sink);
        r.sink = w.sink;
        r.gap = w.gap;
        r.nk -= w.gap;
    }
    return r;
}
template <bool WIN>
__device__ __forceinline__ int key_tile(const Tile& T, int unit) { return WIN && unit >= T.sink ? unit + T.gap : unit; }

}  // namespace kvm
