// Logits of a tree's nodes ahead of the top-k: penalties for tokens that occurred, bias, grammar mask.
//
//   n  = occurrences of token v in the generated part of the sequence and on the node's path, root to node, where that is no longer the prompt
//   x' = x, or, where v occurs anywhere in the sequence or on the path, x / rep for x > 0 and x * rep otherwise
//   x' = x' - freq * n - pres * (n > 0) + bias[v];   tokens whose mask bit is 0: -inf
//
// in fp32, rounded once.  What a tree makes different is the path: every row of logits has counts of its own, which differ from its
// sequence's in the few tokens of its ancestors.
//
// What bounds it: 2 bytes in and 2 out for every logit, and an eighth for its mask: HBM.  Two kernels.  The first makes of each
// sequence's history a word per token of the vocabulary, of its tree the nodes' paths and which nodes have the same token.  In the second
// a block has kVocab tokens and a few rows: a thread reads the words of its 8 tokens once and the rows stream past.  The blocks are many and
// short, since trees differ in size and sequences leave; the first rows are on their way before the first kernel has ended.  Tokens of the
// path are put right behind the stream, a thread a (row, node of the path) pair: where the tokens are those of text, most of a tree's
// lie in the first few of the vocabulary, and whatever thread has those in the stream would do the others' work.
// Measured: 16 trees of 64 nodes, 32000 tokens, everything on 22.7 us (82 MB, 3.6 TB/s; an elementwise addition of as many bytes 14.2); 4 trees of
// 32 nodes, 128256 tokens 18.1 us; 16 nodes, 32000 tokens, penalties alone 4.9 us: two launches and the history's latency.
#include "goose_internal.cuh"

namespace goose {

constexpr int kAdjustThreads = 256;
constexpr int kVocab = 8 * kAdjustThreads;           // tokens of a block
constexpr int kBlockRows = 8;                        // rows of a block, at most
constexpr int kCountThreads = 1024;
constexpr int kCountVocab = 4 * kCountThreads;       // tokens of a block of the first kernel
static_assert(kCountVocab % kVocab == 0, "the second kernel's pieces lie in the first's");
constexpr uint32_t kInPrompt = 0x80000000u;          // of a token's word: it occurs in the prompt; below: its count behind it

// what the first kernel leaves of a sequence
struct AdjustTree {
    uint4 path[kMaxB];                               // a node's path, as a set of nodes
    uint4 same[kMaxB];                               // the nodes that have its token
    uint32_t made[kMaxB / 32];                       // the nodes that are no tokens of the prompt
    int bad;                                         // parent[] is no tree
    int pad[3];
};

// Of a path's nodes that have the token of node j (same): is j the first?  n: how many of them are generated (made).
__device__ __forceinline__ bool first_of_path(const uint4& path, const uint4& same, const uint4& made, int j, uint32_t& n) {
    const uint32_t both[4] = {path.x & same.x, path.y & same.y, path.z & same.z, path.w & same.w}, generated[4] = {made.x, made.y, made.z, made.w};
    int first = kMaxB;
    n = 0;
#pragma unroll
    for (int w = 3; w >= 0; --w) {
        n += __popc(both[w] & generated[w]);
        if (both[w]) first = 32 * w + __ffs(both[w]) - 1;
    }
    return first == j;
}

// the words of kCountVocab tokens (blocks 0 .. pieces - 1), the tree (the last block) of a sequence
__global__ void __launch_bounds__(kCountThreads)
adjust_tables_kernel(const AdjustLogits a, int pieces, int64_t ldw, uint32_t* __restrict__ words, AdjustTree* __restrict__ trees) {
    __shared__ uint32_t s_count[kCountVocab];
    __shared__ uint4 s_path[kMaxB];
    __shared__ int s_up[kMaxB], s_tok[kMaxB];
    const int s = blockIdx.y, tid = threadIdx.x;
    pdl_wait();
    pdl_trigger();
    const int nn = nodes_of(a.n_nodes, s, a.B);
    if ((int)blockIdx.x == pieces) {
        const bool node = tid < nn;
        int up = node ? a.parent[(size_t)s * a.B + tid] : 0;
        const int tok = node && a.draft_tok ? a.draft_tok[(size_t)s * a.B + tid] : -1;
        const bool no_tree = node && (tid == 0 ? up != -1 : (up < 0 || up >= tid));
        const bool bad_len = a.hist && nn > 0 && (a.hist_len[s] < 0 || a.hist_len[s] > a.ldh);
        if (tid == 0) up = 0;
        uint4 path = make_uint4(0, 0, 0, 0), same = path;
        if (node) {
            const uint32_t bit = 1u << (tid & 31);
            (tid < 32 ? path.x : tid < 64 ? path.y : tid < 96 ? path.z : path.w) = bit;
            s_tok[tid] = tok;
        }
        const bool bad = __syncthreads_or(no_tree);
        if (tid == 0) {
            trees[s].bad = bad;
            const int flaws = (bad ? GOOSE_ST_BAD_PARENT : 0) | (bad_len ? GOOSE_ST_BAD_ROWS : 0) | (nodes_bad(a.n_nodes, s, a.B) ? GOOSE_ST_BAD_NODES : 0);
            if (flaws) atomicOr(&a.status[s], flaws);
        }
        if (bad) return;
        // in steps up the tree that double
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
        path.x |= 1u;                                          // (the root is on every path)
        // The node at depth d stands at position hist_len + d: a token of the prompt where that is in front of n_prompt.
        const long long left = a.hist && a.n_prompt && nn > 0 && !bad_len ? (long long)a.n_prompt[s] - a.hist_len[s] : 0;
        const int in_prompt = left > 0 && left <= a.B ? (int)left : 0;   // (a prompt that no node is the end of: goose.h)
        const uint32_t made = __ballot_sync(0xFFFFFFFFu, __popc(path.x) + __popc(path.y) + __popc(path.z) + __popc(path.w) > in_prompt);
        if (tid < kMaxB && (tid & 31) == 0) trees[s].made[tid >> 5] = made;
        if (!node) return;
        for (int j = 0; j < nn; ++j) {
            const uint32_t bit = s_tok[j] == tok ? 1u << (j & 31) : 0;
            (j < 32 ? same.x : j < 64 ? same.y : j < 96 ? same.z : same.w) |= bit;
        }
        trees[s].path[tid] = path;
        trees[s].same[tid] = same;
        return;
    }
    if (nn == 0) return;
    const int base = blockIdx.x * kCountVocab;
    reinterpret_cast<uint4*>(s_count)[tid] = make_uint4(0, 0, 0, 0);
    int len = a.hist_len[s];
    const int prompt = a.n_prompt ? a.n_prompt[s] : 0;
    if (len < 0 || len > a.ldh) len = 0;
    __syncthreads();
    auto count = [&](int t, int j) {
        const uint32_t u = (uint32_t)t - (uint32_t)base;
        if (u < (uint32_t)kCountVocab) {
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
        for (int j = tid; j < quads; j += kCountThreads) {
            const int4 t = h4[j];
            const int at = head + 4 * j;
            count(t.x, at); count(t.y, at + 1); count(t.z, at + 2); count(t.w, at + 3);
        }
        const int tail = head + 4 * quads;
        if (tid < len - tail) count(hist[tail + tid], tail + tid);
    }
    __syncthreads();
    reinterpret_cast<uint4*>(words + (size_t)s * ldw + base)[tid] = reinterpret_cast<const uint4*>(s_count)[tid];
}

// bulk copy into shared memory: size a multiple of 16, both addresses too
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, unsigned long long* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(bytes), "r"((uint32_t)__cvta_generic_to_shared(bar)) : "memory");
}

// kMask: 0 none, 1 its bytes loaded by the threads, 2 its rows lie on 16 bytes and come with the logits
template <int kMask>
__global__ void __launch_bounds__(kAdjustThreads, 4)
adjust_logits_kernel(const AdjustLogits a, int rows_per_block, int64_t ldw, const uint32_t* __restrict__ words,
                     const AdjustTree* __restrict__ trees) {
    __shared__ __align__(128) uint4 s_row[kBlockRows][kAdjustThreads];   // the block's logits as they were
    __shared__ __align__(16) unsigned char s_mask[kMask == 2 ? kBlockRows : 1][kMask == 2 ? kAdjustThreads : 1];
    __shared__ uint4 s_keep[kMask ? kAdjustThreads : 1];      // a mask byte as 16 bits a token: eight selects less a row
    __shared__ unsigned long long s_full;
    __shared__ volatile int s_abort;
    __shared__ int s_listed;
    __shared__ short s_tok[kMaxB];                             // nodes whose token lies in this piece of the vocabulary: where
    __shared__ unsigned char s_list[kMaxB];                    // and which
    const int s = blockIdx.z, tid = threadIdx.x, base = blockIdx.x * kVocab;
    const int v0 = base + 8 * tid, n_v = min(8, a.V - v0);
    // The first kernel has waited for all that is in front of it and writes none of the inputs: they are read ahead of the wait.
    const int nn = nodes_of(a.n_nodes, s, a.B);
    const int i0 = blockIdx.y * rows_per_block, rows = min(rows_per_block, nn - i0);
    const size_t row0 = (size_t)s * a.B + i0;
    if (tid == 0) {
        s_listed = 0;
        s_abort = 0;
        if (rows > 0) {
            const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&s_full), bytes = 16u * ((min(kVocab, a.V - base) + 7) / 8);
            const uint32_t mask_bytes = kMask == 2 ? (uint32_t)min((int64_t)kAdjustThreads, 4 * a.ldm - base / 8) : 0;   // (ldm * 4 is a multiple of 16)
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar));
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((bytes + mask_bytes) * rows) : "memory");
            for (int u = 0; u < rows; ++u) {
                bulk_load(s_row[u], a.logits + (row0 + u) * a.ldl + base, bytes, &s_full);
                if (kMask == 2) bulk_load(s_mask[u], reinterpret_cast<const unsigned char*>(a.mask + (row0 + u) * a.ldm) + base / 8, mask_bytes, &s_full);
            }
        }
    }
    if (kMask) {
        static_assert(kAdjustThreads == 256, "an entry a thread");
        uint32_t keep[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) keep[e] = ((tid >> (2 * e)) & 1 ? 0xFFFFu : 0u) | ((tid >> (2 * e + 1)) & 1 ? 0xFFFF0000u : 0u);
        s_keep[tid] = make_uint4(keep[0], keep[1], keep[2], keep[3]);
    }
    uint32_t open[2] = {0, 0};                                 // a byte a row
    if (kMask == 1 && n_v > 0) {
        const unsigned char* at = reinterpret_cast<const unsigned char*>(a.mask + row0 * a.ldm) + (v0 >> 3);
#pragma unroll
        for (int u = 0; u < kBlockRows; ++u)
            if (u < rows) open[u >> 2] |= (uint32_t)at[(size_t)u * 4 * a.ldm] << (8 * (u & 3));
    }
    const uint32_t tok = tid < nn && rows > 0 && a.draft_tok ? (uint32_t)a.draft_tok[(size_t)s * a.B + tid] - (uint32_t)base : ~0u;
    const float rep = a.repetition ? a.repetition[s] : 1.f, freq = a.frequency ? a.frequency[s] : 0.f, pres = a.presence ? a.presence[s] : 0.f;
    const float inv_rep = 1.f / rep;
    const float* bias = a.bias ? a.bias + (size_t)s * a.bias_stride + base : nullptr;
    // x' = x * (x > 0 ? up : down) + add
    float add[8], m_up[8], m_down[8];
    if (bias && n_v == 8 && (reinterpret_cast<uintptr_t>(bias) & 15) == 0) {
        *reinterpret_cast<float4*>(add) = reinterpret_cast<const float4*>(bias)[2 * tid];
        *reinterpret_cast<float4*>(add + 4) = reinterpret_cast<const float4*>(bias)[2 * tid + 1];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) add[e] = bias && e < n_v ? bias[8 * tid + e] : 0.f;
    }
    __syncthreads();
    if (tok < (uint32_t)kVocab) {
        const int k = atomicAdd(&s_listed, 1);                 // (in any order: each pair writes an element of its own)
        s_list[k] = (unsigned char)tid;
        s_tok[k] = (short)tok;
    }
    pdl_wait();
    pdl_trigger();
    if (rows <= 0) return;
    const AdjustTree& tree = trees[s];
    const bool bad = tree.bad != 0;
    const uint32_t* w = words ? words + (size_t)s * ldw + base : nullptr;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
        const uint4 w4 = w ? *reinterpret_cast<const uint4*>(w + 8 * tid + e) : make_uint4(0, 0, 0, 0);
        const uint32_t word[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int f = 0; f < 4; ++f) {
            const uint32_t n = word[f] & ~kInPrompt;
            m_up[e + f] = word[f] ? inv_rep : 1.f;
            m_down[e + f] = word[f] ? rep : 1.f;
            if (n) add[e + f] += -freq * (float)n - pres;
        }
    }
    constexpr long long kWaitCycles = 2000000000ll;            // about one second of SM clock
    if (mbar_wait_bounded(&s_full, 0, kWaitCycles, &s_abort) == 2) {   // (nothing raises the flag: every thread finds out for itself)
        atomicOr(&a.status[s], GOOSE_ST_TIMEOUT);
        mbar_wait_bounded(&s_full, 0, kWaitCycles, &s_abort);  // copies still in flight land before the block ends
        return;
    }
    if (n_v > 0) {
        __nv_bfloat16* to = a.out + row0 * a.ldo + v0;
#pragma unroll 2
        for (int u = 0; u < rows; ++u, to += a.ldo) {
            const uint4 x = s_row[u][tid];
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
            const uint4 keep4 = kMask ? s_keep[kMask == 2 ? s_mask[u][tid] : ((u < 4 ? open[0] : open[1]) >> (8 * (u & 3))) & 0xFF] : make_uint4(0, 0, 0, 0);
            const uint32_t keep[4] = {keep4.x, keep4.y, keep4.z, keep4.w};
            uint32_t out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y0 = __uint_as_float(in[e] << 16), y1 = __uint_as_float(in[e] & 0xFFFF0000u);
                y0 = fmaf(y0, y0 > 0.f ? m_up[2 * e] : m_down[2 * e], add[2 * e]);
                y1 = fmaf(y1, y1 > 0.f ? m_up[2 * e + 1] : m_down[2 * e + 1], add[2 * e + 1]);
                const __nv_bfloat162 b2 = __floats2bfloat162_rn(y0, y1);
                out[e] = *reinterpret_cast<const uint32_t*>(&b2);
                if (kMask) out[e] = (out[e] & keep[e]) | (0xFF80FF80u & ~keep[e]);   // -inf
            }
            if (bad) out[0] = out[1] = out[2] = out[3] = 0;
            if (n_v == 8) *reinterpret_cast<uint4*>(to) = make_uint4(out[0], out[1], out[2], out[3]);
            else
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < n_v) reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(out[e >> 1] >> (16 * (e & 1)));
        }
    }
    __syncthreads();                                           // the list is complete, the stream's stores are in front of these
    const int listed = bad ? 0 : s_listed, pairs = rows * listed;
    const uint4 made = *reinterpret_cast<const uint4*>(tree.made);
    for (int k = tid; k < pairs; k += kAdjustThreads) {
        const int of_row = k / listed, l = k - of_row * listed, j = s_list[l], t = s_tok[l], v = base + t;
        const size_t r = row0 + of_row;
        uint32_t n;
        if (v >= a.V || !first_of_path(tree.path[i0 + of_row], tree.same[j], made, j, n)) continue;
        if (kMask && !((a.mask[r * a.ldm + (v >> 5)] >> (v & 31)) & 1u)) continue;
        if (w) n += w[t] & ~kInPrompt;
        const float x1 = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(s_row[of_row])[t]);
        a.out[r * a.ldo + v] = __float2bfloat16_rn((x1 > 0.f ? x1 * inv_rep : x1 * rep) + ((bias ? bias[t] : 0.f) + (n ? -freq * (float)n - pres : 0.f)));
    }
}

cudaError_t launch_adjust_logits(goose_ctx* c, AdjustLogits a, int S, cudaStream_t st) {
    if (S == 0) return cudaSuccess;
    a.status = c->status;
    const int pieces = (a.V + kVocab - 1) / kVocab, count_pieces = (a.V + kCountVocab - 1) / kCountVocab;
    const bool counts = a.hist && (a.repetition || a.frequency || a.presence);
    const int64_t ldw = counts ? (int64_t)count_pieces * kCountVocab : 0;
    const size_t tree_bytes = sizeof(AdjustTree) * (size_t)S, need = tree_bytes + sizeof(uint32_t) * (size_t)ldw * S;
    if (cudaError_t e = grow(c, &c->adjust_tables, &c->adjust_bytes, need)) return e;
    AdjustTree* trees = static_cast<AdjustTree*>(c->adjust_tables);
    uint32_t* words = counts ? reinterpret_cast<uint32_t*>(static_cast<char*>(c->adjust_tables) + tree_bytes) : nullptr;
    cudaError_t e = launch_pdl(adjust_tables_kernel, dim3((counts ? count_pieces : 0) + 1, S), dim3(kCountThreads), 0, st, a, counts ? count_pieces : 0, ldw, words, trees);
    c->launches++;
    if (e != cudaSuccess) return e;
    // rows of a block: kBlockRows, fewer where there would not be two blocks an SM
    const long long all = (long long)S * pieces * a.B / (2LL * c->num_sms);
    const int rows = all >= kBlockRows ? kBlockRows : all < 1 ? 1 : (int)all;
    const bool on_16 = ((reinterpret_cast<uintptr_t>(a.mask) | (uintptr_t)(4 * a.ldm)) & 15) == 0;
    auto kernel = !a.mask ? adjust_logits_kernel<0> : on_16 ? adjust_logits_kernel<2> : adjust_logits_kernel<1>;
    e = launch_pdl(kernel, dim3(pieces, (a.B + rows - 1) / rows, S), dim3(kAdjustThreads), 0, st, a, rows, ldw, words, trees);
    c->launches++;
    return e;
}

cudaError_t init_adjust_kernel() { return load_kernels({(const void*)adjust_tables_kernel, (const void*)adjust_logits_kernel<0>, (const void*)adjust_logits_kernel<1>,
                         (const void*)adjust_logits_kernel<2>}); }

}  // namespace goose
