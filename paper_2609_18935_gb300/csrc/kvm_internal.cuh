// Internal declarations of the maintenance library (kernels + host runtime).
// Everything here is private to libkvm; the public ABI is include/kvm.h.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stdint.h>

namespace kvm {

// Programmatic dependent launch: every kernel of the library is launched so
// that it may start while the previous kernel of the stream finishes.  A
// kernel calls grid_dependency_wait() before its first global memory access
// (it returns once the previous grid has completed and its writes are
// visible), so stream order is kept; grid_dependents_launch() then lets the
// next kernel's blocks be scheduled and run their prologue early.
__device__ __forceinline__ void grid_dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_dependents_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename Params>
inline cudaError_t launch_pdl(void (*kernel)(Params), dim3 grid, dim3 block, size_t smem, cudaStream_t s,
                              const Params& p) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

constexpr int kMaxChars = 256;      // characters per context (per-round descriptors travel as kernel parameters)
constexpr int kMaxSpans = 1024;     // deletion spans per round, all characters together
constexpr int kMaxRotaryHalf = 128; // rotary_dim / 2
constexpr int kKv8Rows = 64;        // slots of a block of a cache in 8 bits

// Device error word bits (read by kvm_check).
constexpr int kErrBounds = 1;       // an index fell outside the buffers a kernel was given
constexpr int kErrWait = 2;         // a bounded wait expired
constexpr int kErrValue = 4;        // a draft's key, value or gate is not finite, or a number on its way into an 8-bit cache

// ----------------------------------------------------------------------------
// kv_compact
// ----------------------------------------------------------------------------
constexpr int kCompactThreads = 256;
constexpr int kCompactVecPerThread = 8;            // 16-byte vectors held per thread (1.5 GB in 48 slabs: 4 293 us, 8 260, 16 257 but half the resident blocks beside other kernels)
constexpr int kCompactVecPerChunk = kCompactThreads * kCompactVecPerThread;
constexpr int kCompactWaitLimit = 1 << 22;        // default polls of a read flag (~0.3-1 s with the back-off)

struct CompactChar {
    int32_t L_new;        // live length after removal
    int32_t first;        // first removed live index (= first moved destination)
    int32_t seg_off;      // offset of this character's segments in seg_start/seg_shift
    int32_t n_seg;        // number of spans (= moved segments)
    int32_t cap_off;      // slot offset of the character inside every slab
    int32_t chunks_kv;    // chunks per KV slab
    int32_t chunks_pos;   // chunks of the position slab
    int32_t blk_off;      // first block of this character
    int32_t flag_off;     // first read-flag of this character
};

struct CompactParams {
    int32_t n_chars;
    int32_t n_kv_slabs;   // 2 * n_attn * n_kv_heads  (K slabs, then V slabs)
    int32_t vec_per_row;  // 16-byte vectors per KV row (head_dim * 2 / 16)
    int32_t rows_kv;      // rows per KV chunk
    int32_t rows_pos;     // rows per position chunk
    int32_t total_blocks;
    uint32_t epoch;
    int64_t slab_rows;    // rows per (layer, head) slab = total capacity
    uint4* K;
    uint4* V;
    float* K_scale;       // of caches in 8 bits: per 64 rows; else null
    float* V_scale;
    int32_t* pos;
    int32_t* tickets;     // [n_chars][n_kv_slabs + 1]
    uint32_t* flags;      // read flag of chunk i at flags[i * flag_stride]
    int32_t flag_stride;  // 32 keeps every flag in its own 128-byte line (no line shared by pollers)
    int32_t* err;
    int32_t wait_limit;   // polls of a read flag before the wait gives up (kErrWait)
    // failure-detection test only: when set, every block also waits on this
    // word, which nothing ever sets, so its wait expires after wait_limit polls
    const uint32_t* never_set;
    CompactChar ch[kMaxChars];
    // segment k of a character: survivors whose new index is >= seg_start[k]
    // (and below the next segment's start) come from new index + seg_shift[k]
    int32_t seg_start[kMaxSpans];
    int32_t seg_shift[kMaxSpans];
};

void launch_kv_compact(const CompactParams& p, cudaStream_t s);

struct GatherParams {
    int32_t n_chars;
    int32_t total;        // sum of L_new
    int32_t out_off[kMaxChars + 1];
    int32_t first[kMaxChars];
    int32_t seg_off[kMaxChars];
    int32_t n_seg[kMaxChars];
    int32_t* out;
    int32_t seg_start[kMaxSpans];
    int32_t seg_shift[kMaxSpans];
};
void launch_gather_map(const GatherParams& p, cudaStream_t s);

// Copies of the state accessors: rows x bytes (a multiple of 4) of up to two
// arrays, every row 16-byte aligned on both sides.
struct CopyParams {
    int32_t n, rows, num_sms;
    uint8_t* dst[2];
    const uint8_t* src[2];
    int64_t dpitch, spitch, bytes;
};
void launch_copy(const CopyParams& p, cudaStream_t s);

// ----------------------------------------------------------------------------
// tail attention
// ----------------------------------------------------------------------------
struct AttnChar {
    int32_t L_prev;       // surviving live entries (L')
    int32_t M;            // tail tokens
    int32_t tail_off;     // first packed tail row
    int32_t cap_off;      // slot offset of the character in the slabs
    int64_t p;            // cursor: position of tail token 0
    int32_t n_qtiles;     // query tiles per KV head
    int32_t tile_off;     // first query tile of this character (tiles ordered character, KV head, tile)
};

// The attention's work is the list of (query tile, 64-key tile) units, query
// tiles in order and each tile's key tiles in order.  The first waves * n_ctas
// query tiles are dealt whole, one per block and wave (odd waves in reverse
// block order); of the rest, persistent block c processes units
// [start_c, start_{c+1}), given as (query tile, key tile).
constexpr int kMaxAttnCtas = 320;

// The key tiles of a query tile whose first row is at live index x0, under a window:
// `sink` tiles from the first on, then, `gap` tiles further, all up to its last key.
// A row at x sees keys j <= x with j > x - window or j < n_sink.
struct WindowTiles { int sink, gap; };
__host__ __device__ inline WindowTiles window_tiles(int x0, int window, int n_sink) {
    const int oldest = x0 + 1 - window, first = oldest > 0 ? oldest / 64 : 0;
    const int sinks = n_sink / 64 + (n_sink % 64 > 0);
    const int sink = sinks < first ? sinks : first;
    return {sink, first - sink};
}

struct AttnParams {
    // TMA maps: every layer's K / V slabs as rows of D (box 64 x 64), 128-byte swizzle
    CUtensorMap tmap_k;
    CUtensorMap tmap_v;
    int32_t attn_layer;   // index among attention layers
    int32_t n_chars;
    int32_t Hq, Hkv, D, R, g;
    int32_t n_tiles;      // query tiles over all characters and KV heads
    int32_t n_ctas;       // persistent attention blocks
    int32_t waves;        // whole query tiles dealt to every block first
    int32_t tok_per_tile; // tail tokens per 128-row query tile (128 / g)
    float scale_log2;     // log2(e) / sqrt(D)
    int64_t slab_rows;    // rows per (layer, head) slab
    const __nv_bfloat16* q;       // caller's unrotated q  [sum M][Hq][D]
    const __nv_bfloat16* k_new;   // [sum M][Hkv][D]
    const __nv_bfloat16* v_new;
    __nv_bfloat16* q_rot;         // workspace [sum M][Hq][D]
    __nv_bfloat16* K;             // this layer's K slabs [Hkv][slab_rows][D]
    __nv_bfloat16* V;
    int32_t* pos;                 // [slab_rows]
    __nv_bfloat16* out;           // [sum M][Hq][D]
    const int32_t* tail_pos;      // device [sum M] position of each tail token, or null: p + i
    float* part_o;                // [2 n_ctas][D / 32][8][128][4]: partial O of a block's first / last segment
    float* part_ml;               // [2 n_ctas][128][2]: (reference max in log2 units, sum) of a partial
    int32_t* err;
    int32_t* diag;                // first expired wait: block + 1, tag, parity
    const uint64_t* anc;          // device [sum M]: a draft's ancestor bits (DraftTreeParams), or null: a causal tail
    const float2* turn;           // of a draft: (cos, sin) [sum M][R / 2], with which the attention rotates q itself; or null
    int32_t window, n_sink;       // a row sees its `window` newest keys and the first n_sink; window 0: all
    int32_t widened;              // the kernel before wrote all keys and values, not the tail's alone
    int32_t append;               // of a draft: the attention puts the nodes' keys and values into the caches itself
    double inv_freq[kMaxRotaryHalf];
    int32_t cta_tile[kMaxAttnCtas + 1];
    int32_t cta_k[kMaxAttnCtas + 1];
    AttnChar ch[kMaxChars];
};

// A query tile shared by several attention blocks: its parts are in slot0 and
// in slots 2 (block0 + q), 0 < q < n_parts; its real rows (token-major, then
// the group's heads) are output rows of tokens token0 .. and heads head0 ..
struct SplitTile {
    int32_t slot0;
    int32_t token0;
    int32_t head0;
    int16_t block0, n_parts, rows;
};
struct CombineParams {
    int32_t Hq, D, g;
    int32_t n_split_tiles;
    int32_t many_parts;           // of a draft or over 8-bit caches: parts side by side while there is room
    const float* part_o;          // as in AttnParams
    const float* part_ml;
    __nv_bfloat16* out;           // [sum M][Hq][D]
    SplitTile tile[kMaxAttnCtas];
};

void launch_rope_append(const AttnParams& p, int total_tokens, cudaStream_t s);

// Key re-rotation (tail-and-relocate, §5.2): rotate stored keys of live slots
// [slot0, slot0 + n) in every attention layer by (new_pos - pos), then set pos.
struct RerotateParams {
    int32_t n;            // entries
    int32_t n_attn, Hkv, D, R;
    int64_t slot0;        // first slot (character offset + live index)
    int64_t slab_rows;
    __nv_bfloat16* K;     // all layers' K slabs [n_attn][Hkv][slab_rows][D]
    int32_t* pos;         // [slab_rows]
    const int32_t* new_pos;   // device [n]
    int32_t* err;
    double inv_freq[kMaxRotaryHalf];
};
void launch_rerotate(const RerotateParams& p, cudaStream_t s);
void launch_tail_attention(const AttnParams& p, cudaStream_t s);
void launch_window_attention(const AttnParams& p, cudaStream_t s);      // of which p.window > 0 is this
void launch_attn_combine(const CombineParams& p, cudaStream_t s);

// ----------------------------------------------------------------------------
// caches in 8 bits: e4m3 numbers times a power of two for each block of 64 slots
// and KV head, K and V apart (see kv8.cuh)
// ----------------------------------------------------------------------------
// One layer's slabs [Hkv][slab_rows][D] and scales [Hkv][slab_rows / 64].
struct Kv8Layer {
    uint8_t* K;
    uint8_t* V;
    float* Ks;
    float* Vs;
};

// A character's `rows` rows between its 8-bit blocks and bf16 rows, at row0 on of
// slabs [Hkv][other_rows][D].  pack: into the blocks, the rest of the last becomes 0.
// widen: out of them, rows at or past `rows` are left alone.
struct Kv8CopyParams {
    Kv8Layer cache;
    int32_t Hkv, D, rows;
    int32_t sides;                // 2: keys and values, 1: keys
    int64_t slab_rows, other_rows;
    int64_t cap_off, row0;
    __nv_bfloat16* K;
    __nv_bfloat16* V;
    int32_t* err;
};
void launch_kv8_pack(const Kv8CopyParams& p, cudaStream_t s);
void launch_kv8_widen(const Kv8CopyParams& p, cudaStream_t s);

// A tail's rotated keys and its values into the blocks behind the live entries, and
// its rotated queries into q_rot; those blocks and the older ones in sight as bf16 rows
// of K and V.
struct Kv8AppendChar {
    int32_t cap_off;      // slot offset of the character in the slabs
    int32_t L, M;         // live entries, tail tokens
    int32_t tail_off;     // first packed tail token
    int32_t blk_off;      // first item (block, head, K or V) of its new blocks, those from L / 64 on
    int32_t old_off;      // first item (kv8_widen_blocks blocks, head, K or V) of its older ones in sight
    int32_t n_old;        // those blocks; of them the ones from `sink` on lie `gap` further
    int32_t sink, gap;
    int64_t p;            // cursor
};
struct Kv8AppendParams {
    Kv8Layer to;
    __nv_bfloat16* K;             // [Hkv][slab_rows][D]
    __nv_bfloat16* V;
    const __nv_bfloat16* q;       // [sum M][Hq][D]
    const __nv_bfloat16* k_new;   // [sum M][Hkv][D]
    const __nv_bfloat16* v_new;
    __nv_bfloat16* q_rot;
    int32_t* pos;                 // [slab_rows]
    const int32_t* tail_pos;      // as in AttnParams
    const uint64_t* turn;         // device [R / 2]: a position's turn of each pair, in 2^-64 of a whole one
    int32_t* err;
    int64_t slab_rows;
    int32_t n_chars, Hq, Hkv, D, R, n_items, n_widen, total;
    Kv8AppendChar ch[kMaxChars];
};
void launch_kv8_append(const Kv8AppendParams& p, cudaStream_t s);
constexpr int kv8_widen_blocks(int D) { return 1024 / D; }   // of an item of `old`: 64 KB

// Attention of a few rows a KV head straight from the cache, under the same partition
// and with the same partials as launch_tail_attention.  It rotates the tail's queries
// and puts its keys and values into the cache itself.
constexpr int kDecodeRows = 16;   // most rows (tail tokens of a character x group)
struct DecodeParams {
    AttnParams a;
    Kv8Layer from;                // of a cache in 8 bits; null: a.K and a.V
    int32_t rows;                 // most rows of a query tile
    const uint64_t* turn;         // as in Kv8AppendParams
};
void launch_decode_attention(const DecodeParams& p, cudaStream_t s);
int attention_ctas_per_sm(int head_dim);
constexpr int kAttnRows = 128;   // query rows per attention tile

// ----------------------------------------------------------------------------
// attention-probe diagnostics (§5.3, Appendix C)
// ----------------------------------------------------------------------------
constexpr int kProbeMaxQueries = 16;   // probe queries per call (the paper averages the last 8)
constexpr int kProbeKeys = 64;         // keys per score tile
constexpr int kProbeRows = 64;         // query rows per score tile

struct ProbeParams {
    int32_t L;            // live entries of the character
    int32_t n_q;          // probe queries: the last n_q live entries
    int32_t Hq, Hkv, D, R, g;
    int32_t n_groups;
    int32_t window, n_sink;   // of the layer (window 0: none)
    float scale;          // 1 / sqrt(D)
    int64_t slab_rows;
    int64_t slot0;        // the character's first slot
    const __nv_bfloat16* q;   // caller's unrotated probe queries [n_q][Hq][D]
    float* q_rot;             // workspace [n_q][Hq][D] fp32
    const __nv_bfloat16* K;   // this layer's K slabs [Hkv][slab_rows][D]
    const int32_t* pos;       // [slab_rows]
    float* scores;            // workspace [n_row_blocks * 64][pitch]
    int64_t scores_cap;       // its floats; at least 64 rows of any character
    int32_t pitch;            // L rounded up to 4
    int32_t row_block0, n_row_blocks;   // 64-row blocks of this pass (each within one KV head)
    int32_t last;             // the last pass
    float* row_ms;            // workspace [n_row_blocks * 64][2]: per query row (max, 1 / sum)
    float* probs;             // out [L]
    const int32_t* group_of;  // [L] or null
    float* group_mass;        // out [n_groups]
    int32_t* err;
    double inv_freq[kMaxRotaryHalf];
};
int probe_row_blocks(int n_q, int Hkv, int g);
int launch_attn_probe(ProbeParams p, cudaStream_t s);   // returns the number of launches

// ----------------------------------------------------------------------------
// gated delta rule
// ----------------------------------------------------------------------------
struct GdnChar {
    int32_t M;
    int32_t tail_off;
    int32_t chunk_off;        // first 64-token chunk of this character (all characters' chunks numbered in order)
};

struct GdnParams {
    int32_t n_chars, H, dk, dv;
    int32_t dv_slice;         // rows of S per block (a multiple of 16, <= 128, dividing dv)
    int32_t num_sms;
    int32_t prep_parts;       // prep blocks per (chunk, head): 1, or 2 (one writes [W; Q'] and K, one U | A U)
    const __nv_bfloat16* q;   // [sum M][H][dk]
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;   // [sum M][H][dv]
    const float* alpha;       // [sum M][H]
    const float* beta;
    __nv_bfloat16* out;       // [sum M][H][dv]
    float* S;                 // this layer's state [n_chars][H][dv][dk]
    uint8_t* work;            // per (chunk, head) records written by the prep pass, read by the scan
    int64_t rec_bytes;        // bytes per record
    int32_t total_chunks;     // sum over characters of ceil(M / 64)
    int32_t* err;
    int32_t* diag;            // first expired wait: block + 1, tag, parity
    // fused launches (launch_gdn_fused): the first n_scan blocks are scan
    // items, the rest prep workers; record r is published by flags[32 r] = epoch
    int32_t n_scan;
    uint32_t epoch;
    uint32_t* flags;
    // v2: the state entering each chunk, per (chunk, head), as the output pass reads it
    uint8_t* snap;
    int64_t snap_bytes;
    GdnChar ch[kMaxChars];
    // characters by decreasing tail: a population's longest chains start first
    // (32 characters of 64 .. 512 tokens, 16 heads: 107 -> 94 us)
    int16_t order[kMaxChars];
};

// Short convolution (width 4) + SiLU of a delta-rule layer's q/k/v with the
// carried conv state; k is L2-normalised per head afterwards.
struct ConvParams {
    int32_t n_chars, H, dk, dv, channels;     // channels = H (2 d_k + d_v)
    int32_t total;                            // sum M
    int32_t strip, n_strips;                  // packed tokens a thread walks; ceil(total / strip)
    int32_t aligned;                          // xq, xk, xv on 16 bytes
    int32_t tail_cu[kMaxChars + 1];
    const __nv_bfloat16* xq;                  // caller's pre-conv inputs [sum M][H][d_k]
    const __nv_bfloat16* xk;
    const __nv_bfloat16* xv;                  // [sum M][H][d_v]
    const float* w;                           // [channels][4]
    const __nv_bfloat16* state_in;            // [n_chars][3][channels]: the last 3 inputs before the tail
    __nv_bfloat16* state_out;                 // [n_chars][3][channels]: the last 3 inputs after it
    __nv_bfloat16* yq;                        // outputs, laid out like the inputs
    __nv_bfloat16* yk;
    __nv_bfloat16* yv;
    int32_t* err;
};
void launch_gdn_conv(const ConvParams& p, cudaStream_t s);

// Token-by-token form of a delta-rule layer for short tails, with the short
// convolution (w non-null) in the same launch.
constexpr int kRecurMaxTail = 48;             // most tokens staged at once
struct RecurParams {
    int32_t n_chars, H, dk, dv, channels;     // channels: of the conv state
    int32_t tile;                             // tokens staged at a time
    int32_t tail_cu[kMaxChars + 1];
    const __nv_bfloat16* q;                   // [sum M][H][d_k] (pre-convolution with w)
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;                   // [sum M][H][d_v]
    const float* alpha;                       // [sum M][H]
    const float* beta;
    __nv_bfloat16* out;                       // [sum M][H][d_v]
    float* S;                                 // this layer's state [n_chars][H][d_v][d_k]
    const float* w;                           // [channels][4], or null: no convolution
    const __nv_bfloat16* state_in;            // [n_chars][3][channels], as in ConvParams
    __nv_bfloat16* state_out;
};
// nr: rows of S per eight lanes (1, 2 or 4); 16 nr divides d_v.
void launch_gdn_recur(const RecurParams& p, int nr, cudaStream_t s);

// ----------------------------------------------------------------------------
// drafts: trees of guessed tokens behind the live entries (kvm_draft_*)
// ----------------------------------------------------------------------------
constexpr int kDraftNodes = 64;               // nodes a character: a node's ancestors are the bits of one word
constexpr int kMaxDraftNodes = kMaxChars * kDraftNodes;
constexpr int kMaxDraftLayers = 1024;         // delta-rule layers of a context that drafts

// Writes each node's ancestor word (bit j: node j is the node itself or an
// ancestor; so its depth is the number of bits less one, and its parent,
// grandparent, .. are its bits from the highest below its own down) and its
// position, cursor + depth.
struct DraftTreeParams {
    int32_t n_chars;
    int32_t cu[kMaxChars + 1];
    int64_t cursor[kMaxChars];
    int8_t parent[kMaxDraftNodes];            // packed; -1: a root
    int32_t slot0[kMaxChars];                 // slot of the character's first node: slot offset + live length
    uint64_t* anc;                            // device [sum n]
    int32_t* pos;                             // device [sum n]
    int32_t* slot;                            // device [sum n]: the node's cache slot
    float2* turn;                             // device [sum n][R / 2]: (cos, sin) of each node's rotary angles
    int32_t R, most;                          // rotary dims; nodes of the largest tree
    double inv_freq[kMaxRotaryHalf];
};
void launch_draft_tree(const DraftTreeParams& p, cudaStream_t s);
// Keys and values of a draft's nodes to their slots (R a multiple of 16).
struct DraftAppendParams {
    int32_t nodes, Hkv, D, R;
    int64_t slab_rows;
    const __nv_bfloat16* k_new;               // [sum n][Hkv][D]
    const __nv_bfloat16* v_new;
    __nv_bfloat16* K;                         // this layer's slabs [Hkv][slab_rows][D]
    __nv_bfloat16* V;
    int32_t* cache_pos;                       // [slab_rows]
    const int32_t* pos;                       // as the tree kernel left them
    const int32_t* slot;
    const float2* turn;
    int32_t* err;
};
void launch_draft_append(const DraftAppendParams& p, cudaStream_t s);

// The delta rule over a draft's nodes, and what a commit needs of each: its
// update u, its key, its decay and, with the convolution, its raw inputs.
struct DraftGdnParams {
    int32_t n_chars, H, dk, dv, channels;
    int32_t cu[kMaxChars + 1];
    const uint64_t* anc;                      // [sum n]
    const __nv_bfloat16* q;                   // [sum n][H][d_k] (pre-convolution with w)
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;                   // [sum n][H][d_v]
    const float* alpha;                       // [sum n][H]
    const float* beta;
    __nv_bfloat16* out;                       // [sum n][H][d_v]
    const float* S;                           // this layer's state [n_chars][H][d_v][d_k]
    const float* w;                           // [channels][4], or null: no convolution
    const __nv_bfloat16* state_in;            // [n_chars][3][channels]
    float* rec_u;                             // [sum n][H][d_v]
    __nv_bfloat16* rec_k;                     // [sum n][H][d_k]
    float* rec_a;                             // [sum n][H]
    __nv_bfloat16* rec_x;                     // [sum n][channels] (with w)
    int32_t most;                             // nodes of the largest tree
    int32_t wide;                             // both halves of S in shared memory at once
    int32_t* err;
    int32_t* diag;                            // first expired wait: block + 1, tag, parity
    int16_t order[kMaxChars];                 // characters by decreasing number of nodes
};
void launch_draft_gdn(const DraftGdnParams& p, cudaStream_t s);

// The verdict over a draft: the path that the target's probabilities accept and
// the token after it (see draft_verify.cu).
struct DraftVerifyParams {
    int32_t n_chars, vocab;
    int32_t cu[kMaxChars + 1];
    const uint64_t* anc;                      // [sum n]
    const int32_t* tokens;                    // [sum n]
    const void* target;                       // [sum n][vocab]
    const void* draft;
    const float* u;                           // [sum n]
    const float* u_next;                      // [n_chars]
    int32_t* path;                            // [sum n]
    int32_t* count;                           // [n_chars]
    int32_t* next;                            // [n_chars]
    int32_t* err;
    int32_t* diag;                            // first expired wait: block + 1, tag, parity
};
void launch_draft_verify(const DraftVerifyParams& p, bool bf16, int num_sms, cudaStream_t s);

// Keeps one path of every character's draft: its keys and values move to the
// live end, the delta-rule states advance along it.
struct DraftCommitParams {
    int32_t n_chars, n_attn, Hkv, D;
    int32_t n_gdn, H, dk, dv, channels;       // channels: of the convolution, 0 without
    int32_t rec_nodes;                        // nodes a layer's records have room for
    int64_t slab_rows;
    __nv_bfloat16* K;                         // [n_attn][Hkv][slab_rows][D]
    __nv_bfloat16* V;
    int32_t* pos;                             // [slab_rows]
    float* S;                                 // [n_gdn][n_chars][H][d_v][d_k]
    const float* rec_u;                       // [n_gdn][rec_nodes][H][d_v]
    const __nv_bfloat16* rec_k;
    const float* rec_a;
    const __nv_bfloat16* rec_x;               // [n_gdn][rec_nodes][channels]
    __nv_bfloat16* conv_state;                // [2][n_gdn][n_chars][3][channels]
    uint32_t conv_par[kMaxDraftLayers / 32];  // bit g: the current buffer of layer g
    int32_t node0[kMaxChars];                 // the character's first packed node
    int32_t slot[kMaxChars];                  // slot of its first node: slot offset + live length
    int32_t first_pos[kMaxChars];             // its cursor
    int32_t path_cu[kMaxChars + 1];
    int8_t path[kMaxDraftNodes];              // the accepted nodes' indices, packed
};
void launch_draft_commit(const DraftCommitParams& p, cudaStream_t s);

// Bytes of one (chunk, head) record of the delta-rule workspace.
int64_t gdn_record_bytes(int dk, int dv);
void launch_gdn_chunk_prep(const GdnParams& p, cudaStream_t s);   // state-independent chunk products
void launch_gdn_chunk_scan(const GdnParams& p, cudaStream_t s);   // chunks in order, state in TMEM
// Both in one launch of `grid` blocks (one per SM at most); returns the
// launch's error (the caller falls back to the two launches).
cudaError_t launch_gdn_fused(const GdnParams& p, int grid, cudaStream_t s);
// v2 (d_k = 128, 32-row slices): prep, state chain and output pass (or, with
// fused_grid > 0, prep and chain in one launch of fused_grid blocks, then the
// output pass).  Returns a refused launch's error before enqueuing anything else.
int64_t gdn_snapshot_bytes(int dk, int dv);
cudaError_t launch_gdn_v2(const GdnParams& p, int fused_grid, cudaStream_t s);

// Set the text returned by kvm_last_error() and return `code`.
int report_error(int code, const char* msg);

}  // namespace kvm
