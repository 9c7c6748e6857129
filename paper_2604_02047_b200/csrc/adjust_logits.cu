// Logits of a tree's nodes ahead of the top-k: penalties for tokens that occurred, bias, grammar mask.
//
//   n  = occurrences of token v in the generated part of the sequence and on the node's path, root to node
//   x' = x, or, where v occurs anywhere in the sequence or on the path, x / rep for x > 0 and x * rep otherwise
//   x' = x' - freq * n - pres * (n > 0) + bias[v];   tokens whose mask bit is 0: -inf
//
// in fp32, rounded once.  What a tree makes different is the path: every row of logits has counts of its own, which differ from its
// sequence's in the few tokens of its ancestors.
//
// What bounds it: 2 bytes in and 2 out for every logit, and an eighth for its mask: HBM.  A block has kVocab tokens of one sequence and
// a share of its nodes.  It counts the history into shared memory (every block reads the whole history, from L2; tokens outside its
// piece of the vocabulary fall through) and keeps what that makes of 8 tokens in a thread's registers for all of its rows, which then stream
// past.  Tokens of the path are put right behind the stream, a thread a (row, node of the path) pair: where the tokens are those of text,
// most of a tree's lie in the first few of the vocabulary, and whatever thread has those in the stream would do the others' work.
#include "goose_internal.cuh"

namespace goose {

constexpr int kAdjustColumns = 256;                  // threads beside one another, 8 tokens each
constexpr int kAdjustThreads = 2 * kAdjustColumns;   // two rows at a time
constexpr int kVocab = 8 * kAdjustColumns;           // tokens of a block
constexpr int kAdjustRows = 4;                       // rows of a thread in flight
constexpr int kPathTasks = 2;                        // (row, node) pairs of a thread in a batch of rows
constexpr uint32_t kInPrompt = 0x80000000u;          // of a token's word: it occurs in the prompt; below: its count behind it

__device__ __forceinline__ uint32_t common(const uint4& a, const uint4& b, int w) {
    return w == 0 ? a.x & b.x : w == 1 ? a.y & b.y : w == 2 ? a.z & b.z : a.w & b.w;
}

__global__ void __launch_bounds__(kAdjustThreads, 2)
adjust_logits_kernel(const AdjustLogits a, int rows_per_block) {
    __shared__ uint32_t s_count[kVocab];
    __shared__ uint4 s_path[kMaxB];                  // a node's path, as a set of nodes
    __shared__ uint4 s_same[kMaxB];                  // of the list below: the nodes that have the same token
    __shared__ int s_up[kMaxB], s_tok[kMaxB];        // s_tok: relative to this piece of the vocabulary
    __shared__ unsigned char s_list[kMaxB];          // nodes whose token lies in it
    __shared__ int s_listed;
    const int s = blockIdx.z, tid = threadIdx.x, base = blockIdx.x * kVocab;
    pdl_wait();
    pdl_trigger();
    const int nn = nodes_of(a.n_nodes, s, a.B);
    if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0 && nodes_bad(a.n_nodes, s, a.B)) atomicOr(&a.status[s], GOOSE_ST_BAD_NODES);
    const int i0 = blockIdx.y * rows_per_block, i1 = min(i0 + rows_per_block, nn);
    if (i0 >= nn) return;

    // ---- the sequence's tokens
    static_assert(kVocab == 4 * kAdjustThreads, "one store a thread");
    reinterpret_cast<uint4*>(s_count)[tid] = make_uint4(0, 0, 0, 0);
    if (tid == 0) s_listed = 0;
    int len = a.hist ? a.hist_len[s] : 0;
    const int prompt = a.n_prompt ? a.n_prompt[s] : 0;
    const bool bad_len = len < 0 || len > a.ldh;
    if (bad_len) len = 0;
    const bool node = tid < nn;
    int up = node ? a.parent[(size_t)s * a.B + tid] : 0;
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
    auto count = [&](int t, int j) {
        const uint32_t u = (uint32_t)(t - base);
        if (u < (uint32_t)kVocab) {
            if (j < prompt) atomicOr(&s_count[u], kInPrompt);
            else atomicAdd(&s_count[u], 1u);
        }
    };
    if (len > 0) {
        const int32_t* hist = a.hist + (size_t)s * a.ldh;
        const int head = min(len, (int)((16 - (reinterpret_cast<uintptr_t>(hist) & 15)) >> 2) & 3);   // up to a 16-byte boundary
        if (tid < head) count(hist[tid], tid);
        const int4* h4 = reinterpret_cast<const int4*>(hist + head);
        const int quads = (len - head) >> 2;
#pragma unroll 4
        for (int j = tid; j < quads; j += kAdjustThreads) {
            const int4 t = h4[j];
            const int at = head + 4 * j;
            count(t.x, at); count(t.y, at + 1); count(t.z, at + 2); count(t.w, at + 3);
        }
        const int tail = head + 4 * quads;
        if (tid < len - tail) count(hist[tail + tid], tail + tid);
    }
    if (!bad) {
        if (node && (uint32_t)tok < (uint32_t)kVocab) {
            uint4 same = make_uint4(0, 0, 0, 0);
            for (int j = 0; j < nn; ++j) {
                const uint32_t bit = s_tok[j] == tok ? 1u << (j & 31) : 0;
                (j < 32 ? same.x : j < 64 ? same.y : j < 96 ? same.z : same.w) |= bit;
            }
            s_same[tid] = same;
            s_list[atomicAdd(&s_listed, 1)] = (unsigned char)tid;   // (in any order: each pair writes an element of its own)
        }
        // paths, in steps up the tree that double
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
    const int column = tid & (kAdjustColumns - 1), v0 = base + 8 * column, n_v = min(8, a.V - v0);
    const float rep = a.repetition ? a.repetition[s] : 1.f, freq = a.frequency ? a.frequency[s] : 0.f, pres = a.presence ? a.presence[s] : 0.f;
    const float inv_rep = 1.f / rep;
    const float* bias = a.bias ? a.bias + (size_t)s * a.bias_stride : nullptr;
    float add[8];
    uint32_t seen = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t word = s_count[8 * column + e], n = word & ~kInPrompt;
        if (word) seen |= 1u << e;
        add[e] = bias && e < n_v ? bias[v0 + e] : 0.f;
        if (n) add[e] += -freq * (float)n - pres;
    }

    // ---- rows, in batches of as many as a batch's pairs allow
    const int listed = s_listed, batch = listed ? max(1, kPathTasks * kAdjustThreads / listed) : i1 - i0;
    const size_t row0 = (size_t)s * a.B;
    for (int b0 = i0; b0 < i1; b0 += batch) {
        const int b1 = min(b0 + batch, i1);
        // what the pairs make of their logits, read ahead of the stream, which may write them in place
        float fixed[kPathTasks];
        int fixed_row[kPathTasks], fixed_tok[kPathTasks];
#pragma unroll
        for (int u = 0; u < kPathTasks; ++u) {
            const int task = tid + u * kAdjustThreads, of_row = listed ? task / listed : 0, i = b0 + of_row;
            fixed_row[u] = -1;
            if (listed && i < b1) {
                const int j = s_list[task - of_row * listed], t = s_tok[j], v = base + t;
                const uint4 anc = s_path[i], same = s_same[j];
                uint32_t n = 0;
                int first = kMaxB;
#pragma unroll
                for (int w = 3; w >= 0; --w) {
                    const uint32_t here = common(anc, same, w);
                    n += __popc(here);
                    if (here) first = 32 * w + __ffs(here) - 1;
                }
                // of a path's nodes with one token the first has the pair
                if (first == j && v < a.V && !(a.mask && !((a.mask[(row0 + i) * a.ldm + (v >> 5)] >> (v & 31)) & 1u))) {
                    const float l = __bfloat162float(a.logits[(row0 + i) * a.ldl + v]);
                    n += s_count[t] & ~kInPrompt;
                    fixed[u] = (l > 0.f ? l * inv_rep : l * rep) + ((bias ? bias[v] : 0.f) + (-freq * (float)n - pres));
                    fixed_row[u] = i;
                    fixed_tok[u] = v;
                }
            }
        }
        if (listed) __syncthreads();
        if (n_v > 0) {
            for (int i = b0 + (tid >= kAdjustColumns); i < b1; i += 2 * kAdjustRows) {
                uint4 x[kAdjustRows];
                uint32_t open[kAdjustRows];
#pragma unroll
                for (int u = 0; u < kAdjustRows; ++u) {
                    if (i + 2 * u < b1) {
                        const size_t r = row0 + i + 2 * u;
                        x[u] = *reinterpret_cast<const uint4*>(a.logits + r * a.ldl + v0);
                        open[u] = a.mask ? reinterpret_cast<const unsigned char*>(a.mask + r * a.ldm)[v0 >> 3] : 0xFFu;
                    }
                }
#pragma unroll
                for (int u = 0; u < kAdjustRows; ++u) {
                    if (i + 2 * u >= b1) break;
                    const uint32_t in[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
                    uint32_t out[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float y[2] = {__uint_as_float(in[e] << 16), __uint_as_float(in[e] & 0xFFFF0000u)};
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if ((seen >> (2 * e + h)) & 1u) y[h] = y[h] > 0.f ? y[h] * inv_rep : y[h] * rep;
                            y[h] += add[2 * e + h];
                            if (!((open[u] >> (2 * e + h)) & 1u)) y[h] = -INFINITY;
                        }
                        const __nv_bfloat162 b2 = __floats2bfloat162_rn(y[0], y[1]);
                        out[e] = bad ? 0u : *reinterpret_cast<const uint32_t*>(&b2);
                    }
                    __nv_bfloat16* to = a.out + (row0 + i + 2 * u) * a.ldo + v0;
                    if (n_v == 8) *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[2], out[3]);
                    else
#pragma unroll
                        for (int e = 0; e < 7; ++e)
                            if (e < n_v) reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(out[e >> 1] >> (16 * (e & 1)));
                }
            }
        }
        if (listed) {
            __syncthreads();                           // the stream's stores are in front of these
#pragma unroll
            for (int u = 0; u < kPathTasks; ++u)
                if (fixed_row[u] >= 0) a.out[(row0 + fixed_row[u]) * a.ldo + fixed_tok[u]] = __float2bfloat16_rn(fixed[u]);
        }
    }
}

cudaError_t launch_adjust_logits(goose_ctx* c, AdjustLogits a, int S, cudaStream_t st) {
    if (S == 0) return cudaSuccess;
    a.status = c->status;
    const int pieces = (a.V + kVocab - 1) / kVocab;
    // Blocks share a sequence's rows as ends earliest by this count: waves of two blocks an SM, each as long as its rows and what stands in
    // front of them, worth about seven rows.
    long long best = 0;
    int groups = 1;
    for (int n = 1; n <= a.B; ++n) {
        const long long waves = ((long long)S * pieces * n + 2 * c->num_sms - 1) / (2 * c->num_sms), cost = waves * ((a.B + n - 1) / n + 7);
        if (n == 1 || cost < best) { best = cost; groups = n; }
    }
    const int rows = (a.B + groups - 1) / groups;
    const dim3 grid(pieces, (a.B + rows - 1) / rows, S);
    cudaError_t e = launch_pdl(adjust_logits_kernel, grid, dim3(kAdjustThreads), 0, st, a, rows);
    c->launches++;
    return e;
}

cudaError_t init_adjust_kernel() { return load_kernels({(const void*)adjust_logits_kernel}); }

}  // namespace goose
