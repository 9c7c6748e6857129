// Queries, keys and values of new tokens on their way to the attention: norm of every query and key head, rotation by the
// token's position, K and V rows into the cache, in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * w            (per head, w of the queries or of the keys; without weights y = x)
//   (a, b) -> (a cos t - b sin t, b cos t + a sin t)   for the pairs of the first rope_dim elements, t of the token's position
//
// All of it in fp32, rounded once to bf16.  The position of node i is pos_off + ctx_len + its depth in the tree, or + i in a run of
// prompt tokens (parent == NULL).
//
// What bounds it: a row of 256 bytes in, one out, and some 60 instructions for 16 bytes: HBM in long calls (two prompts of 6001 tokens, 40
// heads: 128 us, 5.78 TB/s), the instructions with norm and half-split pairs (8192 tokens, 32 heads over 8: 59 us, 3.5 TB/s; without norm 47; eight shuffles
// a lane and row, the weights unpacked for every row, 12 to 32 bytes of spill in the streaming forms), the chain
// ctx_len -> table row -> store in short ones (a token: 3.9 us), with node counts n_nodes in front of it, and parent -> depths beside it (16 trees
// of 64 nodes: 8.0).  16 lanes have a row (8 elements, one 16-byte load a lane), so that the norm is four
// shuffles and the partner of a half-split pair another lane's element of the same place; a group of 16 lanes takes
// kRows rows of one token at a time, whose loads are all in flight together, and keeps the token's cosines and sines in registers.
#include "goose_internal.cuh"

namespace goose {

constexpr int kAppendThreads = 256;
constexpr int kAppendGroups = kAppendThreads / 16;   // rows a block works on at once
constexpr int kRows = 4;                             // rows of a group in flight

__device__ __forceinline__ void unpack8(const uint4& p, float (&x)[8]) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Depth of every node of a tree of nn <= kMaxB nodes, by all threads of the block: up to the root in steps that double, so a
// chain of 128 takes seven rounds.  Returns false, the same in every thread, for a parent[] that is no tree.
__device__ __forceinline__ bool tree_depths(const int32_t* __restrict__ parent, int nn, int* s_up, int* s_depth) {
    const int i = threadIdx.x;
    const bool node = i < nn;
    int up = node ? parent[i] : 0, depth = node && i > 0;
    const bool bad = node && (i == 0 ? up != -1 : (up < 0 || up >= i));
    if (i == 0) up = 0;
    if (__syncthreads_or(bad)) return false;
    for (int reach = 1; reach < kMaxB; reach *= 2) {
        if (node) { s_up[i] = up; s_depth[i] = depth; }
        if (!__syncthreads_or(node && up != 0)) break;
        if (node) { depth += s_depth[up]; up = s_up[up]; }
        __syncthreads();
    }
    if (node) s_depth[i] = depth;
    __syncthreads();
    return true;
}

// kTree: positions by the depth in a tree, else by the place in a run of tokens.  kPaged: the rows lie in pages (a run of tokens), and every
// new row gets its position and a weight of zero.  kStream: the next rows are on their way while a group's
// rows are worked on (two prompts of 6001 tokens, 40 heads, in blocks of 16 tokens: 137 -> 132 us; 16 trees of 64 nodes, two rounds a group: 8.0 -> 8.8)
template <bool kTree, bool kStream, bool kPaged>
__global__ void __launch_bounds__(kAppendThreads, 3)
append_kv_kernel(const AppendKv a, int groups_log2 /* groups of 16 lanes a token */) {
    __shared__ int s_up[kMaxB], s_depth[kMaxB];
    const int s = blockIdx.y, lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int per_token = 1 << groups_log2;
    const int first = blockIdx.x * (kAppendGroups >> groups_log2);
    const int i = first + (group >> groups_log2);              // token of this group
    const int H = a.H, Hkv = a.Hkv, rows = H + 2 * Hkv;
    const size_t tok = (size_t)s * a.B + i;
    pdl_wait();
    pdl_trigger();
    // rows r, r + per_token, ... of the token; they depend on no length, so the first leave ahead of everything
    auto load = [&](int r0, uint4 (&x)[kRows]) {
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int r = r0 + u * per_token;
            if (r < rows) {
                const __nv_bfloat16* from = r < H ? a.q + tok * a.ldq + r * kHeadDim
                                          : r < H + Hkv ? a.k + tok * a.ldk + (r - H) * kHeadDim
                                                        : a.v + tok * a.ldv + (r - H - Hkv) * kHeadDim;
                x[u] = reinterpret_cast<const uint4*>(from)[lane];
            }
        }
    };
    uint4 x[kRows];
    const int r_first = group & (per_token - 1);
    if (i < a.B) load(r_first, x);
    const int nn = nodes_of(a.n_nodes, s, a.B);
    if (blockIdx.x == 0 && threadIdx.x == 0 && nodes_bad(a.n_nodes, s, a.B)) atomicOr(&a.status[s], GOOSE_ST_BAD_NODES);
    if (first >= nn) return;
    const int ctx = a.ctx_len[s];
    const int64_t row0 = kPaged ? 0 : a.row_off[s];
    const int64_t pos0 = (int64_t)(a.pos_off ? a.pos_off[s] : 0) + ctx;
    int flaw = rows_outside(row0, ctx, nn, kPaged ? a.pages.room(a.ldw) : a.kv_rows) ? GOOSE_ST_BAD_ROWS : 0;
    int depth = i;
    if (kTree) {
        if (!tree_depths(a.parent + (size_t)s * a.B, nn, s_up, s_depth)) flaw |= GOOSE_ST_BAD_PARENT;
        else if (i < nn) depth = s_depth[i];
    }
    const bool live = i < nn;
    if (!kPaged && !live) return;                              // (whole groups: the shuffles below name their 16 lanes)
    const int64_t pos = pos0 + depth;
    if (a.rope_dim && (pos < 0 || pos >= a.rope_rows)) flaw |= GOOSE_ST_BAD_POS;
    int64_t place = row0 + ctx + i;                            // row of the caches
    if (kPaged && live && !flaw) {
        place = a.pages.row(s, ctx + i);
        if (place < 0) flaw |= GOOSE_ST_BAD_ROWS;
        if (a.row_pos && (pos < 0 || pos > INT32_MAX)) flaw |= GOOSE_ST_BAD_POS;
    }
    if (flaw && live && lane == 0 && r_first == 0) atomicOr(&a.status[s], flaw);

    const int half = a.rope_dim >> 1;
    // cosines and sines of this lane's elements, and the lane that has their partners (half-split pairs)
    float cs[8], sn[8];
    int partner = lane;
    const bool turns = 8 * lane < a.rope_dim;
    if (turns && !flaw) {
        const float* t = a.rope + pos * a.rope_dim;
        if (a.interleaved) {
            const float4 c4 = *reinterpret_cast<const float4*>(t + 4 * lane), s4 = *reinterpret_cast<const float4*>(t + half + 4 * lane);
            const float c[4] = {c4.x, c4.y, c4.z, c4.w}, v[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) { cs[e] = c[e >> 1]; sn[e] = (e & 1) ? v[e >> 1] : -v[e >> 1]; }
        } else {
            const bool upper = 8 * lane >= half;               // y = own * cos -+ partner * sin
            partner = upper ? lane - (half >> 3) : lane + (half >> 3);
            const int j = 8 * (upper ? partner : lane);
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const float4 c4 = *reinterpret_cast<const float4*>(t + j + e), s4 = *reinterpret_cast<const float4*>(t + half + j + e);
                cs[e] = c4.x; cs[e + 1] = c4.y; cs[e + 2] = c4.z; cs[e + 3] = c4.w;
                sn[e] = upper ? s4.x : -s4.x; sn[e + 1] = upper ? s4.y : -s4.y; sn[e + 2] = upper ? s4.z : -s4.z; sn[e + 3] = upper ? s4.w : -s4.w;
            }
        }
    }
    const uint32_t mask = 0xFFFFu << (threadIdx.x & 16);
    const size_t cache_row = (size_t)place * Hkv;
    for (int r0 = kPaged && !live ? rows : r_first; r0 < rows; r0 += kRows * per_token) {
        uint4 next[kRows];
        if (kStream) load(r0 + kRows * per_token, next);
        else if (r0 != r_first) load(r0, x);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int r = r0 + u * per_token;
            if (r >= rows) break;
            uint4* to = r < H ? reinterpret_cast<uint4*>(a.q_out + (tok * H + r) * kHeadDim)
                      : r < H + Hkv ? reinterpret_cast<uint4*>(a.k_cache + (cache_row + r - H) * kHeadDim)
                                    : reinterpret_cast<uint4*>(a.v_cache + (cache_row + r - H - Hkv) * kHeadDim);
            const bool is_q = r < H;
            if (flaw) {                                        // queries of zeros, no row of the cache touched
                if (is_q) to[lane] = make_uint4(0, 0, 0, 0);
                continue;
            }
            if (r < H + Hkv) {
                float y[8];
                unpack8(x[u], y);
                const __nv_bfloat16* weight = is_q ? a.q_weight : a.k_weight;
                if (weight) {
                    float ss = 0.f, w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o, 16);
                    const float inv = rsqrtf(ss * (1.f / kHeadDim) + a.eps);
                    unpack8(reinterpret_cast<const uint4*>(weight)[lane], w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = y[e] * inv * w[e];
                }
                if (a.rope_dim) {
                    float z[8];
                    if (a.interleaved) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = y[e ^ 1];
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = __shfl_sync(mask, y[e], partner, 16);
                    }
                    if (turns) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = fmaf(z[e], sn[e], y[e] * cs[e]);
                    }
                }
                x[u] = pack8(y);
            }
            to[lane] = x[u];
        }
        if (kStream)
#pragma unroll
            for (int u = 0; u < kRows; ++u) x[u] = next[u];
    }
    if (kPaged && (a.row_weight || a.row_pos)) {
        // the new rows' weights and positions, a head's neighbouring tokens side by side (each token's by itself, two prompts of 6001 tokens, 40 heads: 135 -> 150 us)
        __shared__ int s_pos[kAppendGroups];
        const int tokens_log2 = 4 - groups_log2;
        if (lane == 0 && r_first == 0) s_pos[group >> groups_log2] = live && !flaw ? a.row_pos ? (int)pos : 0 : -1;
        __syncthreads();
        for (int e = threadIdx.x; e < Hkv << tokens_log2; e += kAppendThreads) {
            const int t = e & ((1 << tokens_log2) - 1), p = s_pos[t];
            if (p < 0) continue;
            const size_t at = ((size_t)s * Hkv + (e >> tokens_log2)) * a.ldw + ctx + first + t;
            if (a.row_weight) a.row_weight[at] = 0.f;
            if (a.row_pos) a.row_pos[at] = p;
        }
    }
}

cudaError_t launch_append_kv(goose_ctx* c, AppendKv a, int S, cudaStream_t st) {
    if (S == 0) return cudaSuccess;
    a.status = c->status;
    // groups a token: as few as give every SM three blocks (a token's lengths, tree and table row are then looked up for more rows),
    // at most as many as leave each kRows rows, and a block of one token; more, up to sixteen blocks an SM, where each keeps four rounds of rows:
    // the last blocks then end together (64 trees of 128 nodes, 40 heads: 153 -> 118 us; with two rounds left to each, 157)
    const int rows = a.H + 2 * a.Hkv;
    int lg = 0;
    while ((1 << lg) < kAppendGroups && (kRows << lg) < rows && (((long long)S * a.B) << lg) < 3LL * kAppendGroups * c->num_sms) ++lg;
    while ((1 << lg) < kAppendGroups && (8 * kRows << lg) <= rows && (((long long)S * a.B) << lg) < 16LL * kAppendGroups * c->num_sms) ++lg;
    const int per_block = kAppendGroups >> lg;
    const dim3 grid((a.B + per_block - 1) / per_block, S);
    const bool stream = rows >= (4 * kRows << lg);            // four rounds a group and more
    auto kernel = a.pages.table ? (stream ? append_kv_kernel<false, true, true> : append_kv_kernel<false, false, true>)
                : a.parent ? (stream ? append_kv_kernel<true, true, false> : append_kv_kernel<true, false, false>)
                           : (stream ? append_kv_kernel<false, true, false> : append_kv_kernel<false, false, false>);
    cudaError_t e = launch_pdl(kernel, grid, dim3(kAppendThreads), 0, st, a, lg);
    c->launches++;
    return e;
}

// The accepted path's tokens behind a sequence's history: hist[s][hist_len[s] + j] = draft_tok[s][path[s][j]], j = 0..accept_len[s].
// A launch and two dependent loads (1.4 us for a sequence, 1.9 for 64): a block a sequence, a thread a node of the path.
__global__ void __launch_bounds__(kMaxB)
append_tokens_kernel(const int32_t* __restrict__ draft_tok, const int32_t* __restrict__ path, const int32_t* __restrict__ accept_len,
                     const int32_t* __restrict__ n_nodes, int B, int32_t* __restrict__ hist, int64_t ldh,
                     const int32_t* __restrict__ hist_len, int32_t* __restrict__ new_len, int32_t* __restrict__ status) {
    __shared__ int s_path[kMaxB];
    const int s = blockIdx.x, j = threadIdx.x;
    pdl_wait();
    pdl_trigger();
    const int p = j < B ? path[(size_t)s * B + j] : -1;
    const int L = accept_len[s], len = hist_len[s], nn = nodes_of(n_nodes, s, B);
    s_path[j] = p;
    __syncthreads();
    int flaw = nodes_bad(n_nodes, s, B) ? GOOSE_ST_BAD_NODES : 0;
    if (nn > 0) {
        const bool off_path = j <= L && (p < j || p >= nn || (j == 0 ? p != 0 : p <= s_path[j - 1]));
        if (__syncthreads_or(off_path || L < 0 || L >= nn)) flaw = GOOSE_ST_BAD_PATH;
        else if (len < 0 || (int64_t)len + L + 1 > ldh) flaw = GOOSE_ST_BAD_ROWS;
        else if (j <= L) hist[(size_t)s * ldh + len + j] = draft_tok[(size_t)s * B + p];
    }
    if (j == 0) {
        new_len[s] = nn > 0 && !flaw ? len + L + 1 : len;
        if (flaw) atomicOr(&status[s], flaw);
    }
}

cudaError_t launch_append_tokens(goose_ctx* c, const int32_t* draft_tok, const int32_t* path, const int32_t* accept_len,
                                 const int32_t* n_nodes, int S, int B, int32_t* hist, int64_t ldh, const int32_t* hist_len,
                                 int32_t* new_len, cudaStream_t st) {
    if (S == 0) return cudaSuccess;
    cudaError_t e = launch_pdl(append_tokens_kernel, dim3(S), dim3(kMaxB), 0, st, draft_tok, path, accept_len, n_nodes, B, hist, ldh,
                               hist_len, new_len, c->status);
    c->launches++;
    return e;
}

cudaError_t init_append_kernels() {
    return load_kernels({(const void*)append_kv_kernel<true, false, false>, (const void*)append_kv_kernel<true, true, false>,
                         (const void*)append_kv_kernel<false, false, false>, (const void*)append_kv_kernel<false, true, false>,
                         (const void*)append_tokens_kernel, (const void*)append_kv_kernel<false, false, true>,
                         (const void*)append_kv_kernel<false, true, true>});
}

}  // namespace goose
