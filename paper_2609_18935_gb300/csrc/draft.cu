// Drafts: a tree of guessed tokens behind each character's live entries, and
// the commit of one of its paths (kvm_draft_begin, kvm_draft_commit).
//
//  draft_tree   : each node's ancestors as the bits of one word, its position,
//                 cursor + depth, and the cosines and sines of its rotary angles.
//                 Once a step, for every layer.
//  draft_append : an attention layer's keys (rotated) and values of the nodes to
//                 the slots behind the live entries, where the attention does
//                 not do it itself.
//  draft_commit : one launch for every layer.  The nodes of a path are the
//                 character's next tokens:
//                 * attention caches: the path's key and value rows move from
//                   live + node to live + rank.  A path's indices increase, so
//                   rank <= node, and a block that reads the rows of its slab in
//                   pieces, each before it is written, moves them in place;
//                 * states: S <- G S + sum_r w_r u_r k_r^T, with G the product
//                   of alpha along the path and w_r that of the nodes after r.
//                   u_r, the delta rule's update at node r, depends on the
//                   node's ancestors only and was kept by the draft's layer
//                   (draft_gdn.cu), so nothing is solved again and the sum has
//                   no chain over the tokens;
//                 * convolution states: the last three of the carried inputs
//                   and the path's raw ones.
//                 Bound by reading and writing S once (128 KB a head of 128 x
//                 128); a block holds 32 rows of it in registers.  Six
//                 delta-rule layers of 16 characters (16 heads): 201 MB in 34 us,
//                 5.9 TB/s.
#include "draft_rows.cuh"
#include "kvm_internal.cuh"

namespace kvm {
namespace {

constexpr double kTwoPi = 6.283185307179586476925286766559;
constexpr int kTreeNodes = 8;                // nodes a block of the tree kernel

// grid (n_chars, ceil(most / kTreeNodes))
__global__ void __launch_bounds__(256) draft_tree_kernel(const __grid_constant__ DraftTreeParams p) {
    grid_dependency_wait();
    grid_dependents_launch();
    const int b = blockIdx.x, i0 = blockIdx.y * kTreeNodes, n0 = p.cu[b];
    const int n = min(kTreeNodes, p.cu[b + 1] - n0 - i0);
    __shared__ int depth[kTreeNodes];
    if ((int)threadIdx.x < n) {
        const int i = i0 + threadIdx.x;
        uint64_t anc = 0;
        for (int j = i; j >= 0; j = p.parent[n0 + j]) anc |= 1ull << j;   // parents have smaller indices (checked on the host)
        p.anc[n0 + i] = anc;
        depth[threadIdx.x] = __popcll(anc) - 1;
        p.pos[n0 + i] = (int32_t)(p.cursor[b] + depth[threadIdx.x]);
        p.slot[n0 + i] = p.slot0[b] + i;
    }
    __syncthreads();
    const int half = p.R / 2;
    for (int e = threadIdx.x; e < n * half; e += blockDim.x) {
        const int x = e / half, d = e % half;
        // formed and reduced in 64 bits: positions far beyond the live length stay exact
        const double ang = (double)(p.cursor[b] + depth[x]) * p.inv_freq[d];
        const double r = fma(-rint(ang * (1.0 / kTwoPi)), kTwoPi, ang);
        float2 t;
        sincosf((float)r, &t.y, &t.x);
        p.turn[(int64_t)(n0 + i0 + x) * half + d] = t;
    }
}

// A block a node, a thread eight elements of a key or value row, those of a rotary
// pair (i, i + R / 2) together: the attention that follows rotates q itself and
// waits for this kernel only where it reads the nodes' rows.
__global__ void __launch_bounds__(128) draft_append_kernel(const __grid_constant__ DraftAppendParams p) {
    grid_dependency_wait();
    grid_dependents_launch();
    const int n = blockIdx.x;
    const int64_t slot = p.slot[n];
    const int D = p.D, half = p.R / 2, rot = half / 8, per = D / 8, keys = p.Hkv * (per - rot);
    for (int e = threadIdx.x; e < keys + p.Hkv * per; e += blockDim.x) {
        const bool is_v = e >= keys;
        const int x = is_v ? e - keys : e, pieces = is_v ? per : per - rot, h = x / pieces, g = x % pieces;
        const bool turned = !is_v && g < rot;
        const int d = 8 * (is_v || turned ? g : g + rot);            // past the pairs' second halves
        const __nv_bfloat16* src = (is_v ? p.v_new : p.k_new) + ((int64_t)n * p.Hkv + h) * D + d;
        __nv_bfloat16* dst = (is_v ? p.V : p.K) + ((int64_t)h * p.slab_rows + slot) * D + d;
        bool bad;
        if (turned) {
            TurnedNode x;
            x.load(src, half, p.turn + (int64_t)n * half + d);
            bad = x.store(dst, half);
        } else {
            uint4 v = *reinterpret_cast<const uint4*>(src);
            bad = clear_not_finite(v);
            *reinterpret_cast<uint4*>(dst) = v;
        }
        if (bad) atomicOr(p.err, kErrValue);
    }
    if (threadIdx.x == 0) p.cache_pos[slot] = p.pos[n];
}

constexpr int kThreads = 128;
constexpr int kStateRows = 32;               // rows of S a block
constexpr int kTile = 16;                    // path nodes staged at a time
constexpr int kMoveVec = 4;                  // 16-byte pieces a thread moves at a time

// Blocks of one character (blockIdx.y), in blockIdx.x order: states [layer][head][32-row slice], cache slabs
// [K, V][layer][KV head], convolution states [layer][1024-channel piece], position ids.
struct Parts {
    int state, kv, conv;
};
__host__ __device__ inline Parts parts_of(const DraftCommitParams& p) {
    Parts x;
    x.state = p.n_gdn * p.H * (p.dv / kStateRows);
    x.kv = 2 * p.n_attn * p.Hkv;
    x.conv = p.n_gdn * ((p.channels + 8 * kThreads - 1) / (8 * kThreads));
    return x;
}

template <int DK>
__device__ void commit_state(const DraftCommitParams& p, int b, int item, const int8_t* path, int d) {
    constexpr int NP = DK / 32;
    __shared__ __align__(16) float ks[kTile][DK];
    __shared__ float us[kTile][kStateRows];
    __shared__ float al[kDraftNodes], wt[kDraftNodes + 1];
    const int slices = p.dv / kStateRows;
    const int sl = item % slices, h = item / slices % p.H, g = item / slices / p.H;
    const int tid = threadIdx.x, j = tid & 7, row = tid >> 3;   // this thread: rows 2 row, 2 row + 1; float4 groups j, j + 8, ..
    const int64_t node0 = (int64_t)g * p.rec_nodes + p.node0[b];
    float* S = p.S + ((((int64_t)g * p.n_chars + b) * p.H + h) * p.dv + sl * kStateRows + 2 * row) * DK + 4 * j;
    float4 s[2][NP];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < NP; ++i) s[r][i] = *reinterpret_cast<const float4*>(S + r * DK + 32 * i);
    if (tid < d) al[tid] = p.rec_a[(node0 + path[tid]) * p.H + h];
    __syncthreads();
    if (tid <= d) {                                  // wt[r]: product of alpha after the r-th node of the path; wt[d] == G at r = -1
        float w = 1.f;
        for (int t = tid == d ? 0 : tid + 1; t < d; ++t) w *= al[t];
        wt[tid] = w;
    }
    __syncthreads();
    const float G = wt[d];
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < NP; ++i) { s[r][i].x *= G; s[r][i].y *= G; s[r][i].z *= G; s[r][i].w *= G; }
    for (int t0 = 0; t0 < d; t0 += kTile) {
        const int nt = min(kTile, d - t0);
        if (t0 > 0) __syncthreads();
        for (int e = tid; e < nt * (DK / 2); e += kThreads) {
            const int t = e / (DK / 2), c = e % (DK / 2);
            const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(
                p.rec_k + ((node0 + path[t0 + t]) * p.H + h) * DK + 2 * c);
            *reinterpret_cast<float2*>(&ks[t][2 * c]) = __bfloat1622float2(x);
        }
        for (int e = tid; e < nt * kStateRows; e += kThreads) {
            const int t = e / kStateRows, r = e % kStateRows;
            us[t][r] = wt[t0 + t] * p.rec_u[((node0 + path[t0 + t]) * p.H + h) * p.dv + sl * kStateRows + r];
        }
        __syncthreads();
        for (int t = 0; t < nt; ++t) {
            const float u0 = us[t][2 * row], u1 = us[t][2 * row + 1];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const float4 k = *reinterpret_cast<const float4*>(&ks[t][4 * j + 32 * i]);
                s[0][i].x = fmaf(u0, k.x, s[0][i].x); s[0][i].y = fmaf(u0, k.y, s[0][i].y);
                s[0][i].z = fmaf(u0, k.z, s[0][i].z); s[0][i].w = fmaf(u0, k.w, s[0][i].w);
                s[1][i].x = fmaf(u1, k.x, s[1][i].x); s[1][i].y = fmaf(u1, k.y, s[1][i].y);
                s[1][i].z = fmaf(u1, k.z, s[1][i].z); s[1][i].w = fmaf(u1, k.w, s[1][i].w);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int i = 0; i < NP; ++i) *reinterpret_cast<float4*>(S + r * DK + 32 * i) = s[r][i];
}

__device__ void commit_kv(const DraftCommitParams& p, int b, int item, const int8_t* path, int d) {
    bool moves = false;
    for (int r = 0; r < d; ++r) moves |= path[r] != r;
    if (!moves) return;                              // uniform
    const int slabs = p.n_attn * p.Hkv;
    const int slab = item % slabs;
    uint4* rows = reinterpret_cast<uint4*>((item < slabs ? p.K : p.V) + ((int64_t)slab * p.slab_rows + p.slot[b]) * p.D);
    // In pieces from the first row on: a row comes from its own place or a later one,
    // so no piece overwrites what a later piece reads.
    const int vec = p.D / 8, n = d * vec;
    for (int x0 = 0; x0 < n; x0 += kMoveVec * kThreads) {
        uint4 v[kMoveVec];
#pragma unroll
        for (int e = 0; e < kMoveVec; ++e) {
            const int x = x0 + threadIdx.x + e * kThreads;
            if (x < n) v[e] = rows[path[x / vec] * vec + x % vec];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kMoveVec; ++e) {
            const int x = x0 + threadIdx.x + e * kThreads;
            if (x < n) rows[x] = v[e];
        }
    }
}

__device__ void commit_conv(const DraftCommitParams& p, int b, int item, const int8_t* path, int d) {
    const int pieces = (p.channels + 8 * kThreads - 1) / (8 * kThreads);
    const int g = item / pieces, c = 8 * (item % pieces * kThreads + (int)threadIdx.x);
    if (c >= p.channels) return;
    const int cur = p.conv_par[g >> 5] >> (g & 31) & 1;
    __nv_bfloat16* st = p.conv_state + (((int64_t)cur * p.n_gdn + g) * p.n_chars + b) * 3 * p.channels + c;
    const __nv_bfloat16* x = p.rec_x + ((int64_t)g * p.rec_nodes + p.node0[b]) * p.channels + c;
    uint4 v[3];
#pragma unroll
    for (int r = 0; r < 3; ++r) {
        const int t = d - 3 + r;                     // place in the path; negative: the carried row t + 3
        v[r] = *reinterpret_cast<const uint4*>(t >= 0 ? x + (int64_t)path[t] * p.channels : st + (int64_t)(t + 3) * p.channels);
    }
#pragma unroll
    for (int r = 0; r < 3; ++r) *reinterpret_cast<uint4*>(st + (int64_t)r * p.channels) = v[r];
}

__global__ void __launch_bounds__(kThreads) draft_commit_kernel(const __grid_constant__ DraftCommitParams p) {
    grid_dependency_wait();
    grid_dependents_launch();
    const int b = blockIdx.y;
    const int d = p.path_cu[b + 1] - p.path_cu[b];
    if (d <= 0) return;
    __shared__ int8_t path[kDraftNodes];
    if ((int)threadIdx.x < d) path[threadIdx.x] = p.path[p.path_cu[b] + threadIdx.x];
    __syncthreads();
    const Parts n = parts_of(p);
    int x = blockIdx.x;
    if (x < n.state) {
        if (p.dk == 64) commit_state<64>(p, b, x, path, d);
        else commit_state<128>(p, b, x, path, d);
        return;
    }
    x -= n.state;
    if (x < n.kv) return commit_kv(p, b, x, path, d);
    x -= n.kv;
    if (x < n.conv) return commit_conv(p, b, x, path, d);
    if (p.pos && (int)threadIdx.x < d) p.pos[p.slot[b] + threadIdx.x] = p.first_pos[b] + threadIdx.x;
}

}  // namespace

void launch_draft_tree(const DraftTreeParams& p, cudaStream_t s) {
    launch_pdl(draft_tree_kernel, dim3(p.n_chars, (p.most + kTreeNodes - 1) / kTreeNodes), dim3(256), 0, s, p);
}

void launch_draft_append(const DraftAppendParams& p, cudaStream_t s) {
    launch_pdl(draft_append_kernel, dim3(p.nodes), dim3(128), 0, s, p);
}

void launch_draft_commit(const DraftCommitParams& p, cudaStream_t s) {
    const Parts n = parts_of(p);
    launch_pdl(draft_commit_kernel, dim3(n.state + n.kv + n.conv + 1, p.n_chars), dim3(kThreads), 0, s, p);
}

}  // namespace kvm
