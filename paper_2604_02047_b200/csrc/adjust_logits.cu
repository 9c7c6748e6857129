// Logits of a tree's nodes ahead of the top-k: penalties for tokens that occurred, bias, grammar mask.
//
//   n  = occurrences of token v in the generated part of the sequence and on the node's path, root to node
//   x' = x, or, where v occurs anywhere in the sequence or on the path, x / rep for x > 0 and x * rep otherwise
//   x' = x' - freq * n - pres * (n > 0) + bias[v];   tokens whose mask bit is 0: -inf
//
// in fp32, rounded once.  What a tree makes different is the path: every row of logits has counts of its own, which differ from its
// sequence's in the few tokens of its ancestors.
//
// What bounds it: 2 bytes in and 2 out for every logit, and an eighth for its mask.  A block has kVocab tokens of one sequence and
// walks a share of its nodes: it counts the history once, into shared memory (each block reads the whole history, of which the
// tokens outside its piece of the vocabulary fall through), and keeps what that makes of 8 tokens in a thread's registers for all of its
// rows.  The path is a 128-bit set of nodes for each thread, those whose token is one of the thread's 8, which a row
// intersects with its ancestors: nearly always empty.
#include "goose_internal.cuh"

namespace goose {

constexpr int kAdjustThreads = 256;
constexpr int kVocab = 8 * kAdjustThreads;           // tokens of a block
constexpr int kAdjustRows = 4;                       // rows in flight
constexpr uint32_t kInPrompt = 0x80000000u;          // of a token's word: it occurs in the prompt; below: its count behind it

__global__ void __launch_bounds__(kAdjustThreads)
adjust_logits_kernel(const AdjustLogits a, int rows_per_block) {
    __shared__ uint32_t s_count[kVocab];
    __shared__ uint32_t s_nodes[4][kAdjustThreads];  // nodes whose token is one of thread t's
    __shared__ uint4 s_path[kMaxB];                  // ancestors of a node, itself included
    __shared__ int s_up[kMaxB], s_tok[kMaxB];
    const int s = blockIdx.z, tid = threadIdx.x, base = blockIdx.x * kVocab;
    pdl_wait();
    pdl_trigger();
    const int nn = nodes_of(a.n_nodes, s, a.B);
    if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0 && nodes_bad(a.n_nodes, s, a.B)) atomicOr(&a.status[s], GOOSE_ST_BAD_NODES);
    const int i0 = blockIdx.y * rows_per_block, i1 = min(i0 + rows_per_block, nn);
    if (i0 >= nn) return;

    // ---- the sequence's tokens
#pragma unroll
    for (int e = 0; e < 8; e += 4) reinterpret_cast<uint4*>(s_count)[tid * 2 + e / 4] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int w = 0; w < 4; ++w) s_nodes[w][tid] = 0;
    int len = a.hist ? a.hist_len[s] : 0;
    const int prompt = a.n_prompt ? a.n_prompt[s] : 0;
    const bool bad_len = len < 0 || len > a.ldh;
    if (bad_len) len = 0;
    const bool node = tid < nn;
    const int32_t* par = a.parent + (size_t)s * a.B;
    int up = node ? par[tid] : 0;
    const int tok = node && a.draft_tok ? a.draft_tok[(size_t)s * a.B + tid] - base : -1;
    const bool no_tree = node && (tid == 0 ? up != -1 : (up < 0 || up >= tid));
    if (tid == 0) up = 0;
    uint4 path = make_uint4(0, 0, 0, 0);
    if (node) {
        const uint32_t bit = 1u << (tid & 31);
        (tid < 32 ? path.x : tid < 64 ? path.y : tid < 96 ? path.z : path.w) = bit;
        s_tok[tid] = tok;
    }
    const bool bad = __syncthreads_or(no_tree);
    if (tid == 0 && blockIdx.x == 0 && blockIdx.y == 0 && (bad || bad_len))
        atomicOr(&a.status[s], (bad ? GOOSE_ST_BAD_PARENT : 0) | (bad_len ? GOOSE_ST_BAD_ROWS : 0));
    const int32_t* hist = a.hist + (size_t)s * a.ldh;
#pragma unroll 8
    for (int j = tid; j < len; j += kAdjustThreads) {
        const uint32_t u = (uint32_t)(hist[j] - base);
        if (u < (uint32_t)kVocab) {
            if (j < prompt) atomicOr(&s_count[u], kInPrompt);
            else atomicAdd(&s_count[u], 1u);
        }
    }
    if (!bad) {
        if (node && (uint32_t)tok < (uint32_t)kVocab) atomicOr(&s_nodes[tid >> 5][tok >> 3], 1u << (tid & 31));
        // ancestors, in steps up the tree that double
        for (int reach = 1; reach < kMaxB; reach *= 2) {
            if (node) { s_path[tid] = path; s_up[tid] = up; }
            if (!__syncthreads_or(node && up != 0)) break;
            if (node) {
                const uint4 more = s_path[up];
                path.x |= more.x; path.y |= more.y; path.z |= more.z; path.w |= more.w;
                up = s_up[up];
            }
            __syncthreads();
        }
        if (node) { path.x |= 1u; s_path[tid] = path; }    // (the root is on every path)
    }
    __syncthreads();

    // ---- this thread's tokens
    const int v0 = base + 8 * tid, n_v = min(8, a.V - v0);
    if (n_v <= 0) return;
    const float rep = a.repetition ? a.repetition[s] : 1.f, freq = a.frequency ? a.frequency[s] : 0.f, pres = a.presence ? a.presence[s] : 0.f;
    const float inv_rep = 1.f / rep;
    const float* bias = a.bias ? a.bias + (size_t)s * a.bias_stride + v0 : nullptr;
    float add[8];
    uint32_t seen = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t word = s_count[8 * tid + e], n = word & ~kInPrompt;
        if (word) seen |= 1u << e;
        add[e] = bias && e < n_v ? bias[e] : 0.f;
        if (n) add[e] += -freq * (float)n - pres;
    }
    uint32_t mine[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) mine[w] = s_nodes[w][tid];

    for (int i = i0; i < i1; i += kAdjustRows) {
        uint4 x[kAdjustRows];
        uint32_t open[kAdjustRows];
#pragma unroll
        for (int u = 0; u < kAdjustRows; ++u) {
            if (i + u < i1) {
                const size_t r = (size_t)s * a.B + i + u;
                x[u] = *reinterpret_cast<const uint4*>(a.logits + r * a.ldl + v0);
                open[u] = a.mask ? reinterpret_cast<const unsigned char*>(a.mask + r * a.ldm)[v0 >> 3] : 0xFFu;
            }
        }
#pragma unroll
        for (int u = 0; u < kAdjustRows; ++u) {
            if (i + u >= i1) break;
            const size_t r = (size_t)s * a.B + i + u;
            const uint32_t in[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
            const uint4 anc = s_path[i + u];
            const uint32_t hit[4] = {anc.x & mine[0], anc.y & mine[1], anc.z & mine[2], anc.w & mine[3]};
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float l = (e & 1) ? __uint_as_float(in[e >> 1] & 0xFFFF0000u) : __uint_as_float(in[e >> 1] << 16);
                y[e] = ((seen >> e) & 1u) ? (l > 0.f ? l * inv_rep : l * rep) : l;
                y[e] += add[e];
            }
            if (hit[0] | hit[1] | hit[2] | hit[3]) {           // tokens of this path among the thread's eight
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    uint32_t more = 0;
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        for (uint32_t h = hit[w]; h; h &= h - 1) more += s_tok[32 * w + __ffs(h) - 1] == 8 * tid + e;
                    if (more) {
                        const uint32_t n = (s_count[8 * tid + e] & ~kInPrompt) + more;
                        const float l = (e & 1) ? __uint_as_float(in[e >> 1] & 0xFFFF0000u) : __uint_as_float(in[e >> 1] << 16);
                        y[e] = (l > 0.f ? l * inv_rep : l * rep) - freq * (float)n - pres + (bias && e < n_v ? bias[e] : 0.f);
                    }
                }
            }
            uint32_t out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float lo = (open[u] >> (2 * e)) & 1u ? y[2 * e] : -INFINITY, hi = (open[u] >> (2 * e + 1)) & 1u ? y[2 * e + 1] : -INFINITY;
                const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
                out[e] = bad ? 0u : *reinterpret_cast<const uint32_t*>(&b);
            }
            __nv_bfloat16* to = a.out + r * a.ldo + v0;
            if (n_v == 8) *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[2], out[3]);
            else
                for (int e = 0; e < n_v; ++e) reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(out[e >> 1] >> (16 * (e & 1)));
        }
    }
}

cudaError_t launch_adjust_logits(goose_ctx* c, AdjustLogits a, int S, cudaStream_t st) {
    if (S == 0) return cudaSuccess;
    a.status = c->status;
    const int pieces = (a.V + kVocab - 1) / kVocab;
    // about four blocks an SM, where the rows allow it
    const long long blocks = 4LL * c->num_sms, per = ((long long)S * pieces * a.B + blocks - 1) / blocks;
    const int rows = (int)(per > a.B ? a.B : per);
    const dim3 grid(pieces, (a.B + rows - 1) / rows, S);
    cudaError_t e = launch_pdl(adjust_logits_kernel, grid, dim3(kAdjustThreads), 0, st, a, rows);
    c->launches++;
    return e;
}

cudaError_t init_adjust_kernel() { return load_kernels({(const void*)adjust_logits_kernel}); }

}  // namespace goose
