// Attention of a chunk of new tokens over the pages of its sequence: out_i = sum_j p_ij v_j, p_ij = exp(x_ij - lse_i), x_ij = scale q_i . k_j,
// lse_i = log sum_j exp(x_ij), over the rows j <= ctx + i.  One pass over the rows with the running maximum m and sum l of every query row
// (base 2); what several CTAs have of a row is joined by  out = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p.
//
// Persistent, one CTA an SM, tcgen05 with TMEM accumulators, TMA loads, mbarrier pipeline; work list: chunk_work.cuh.  A segment has two lanes with
// a softmax warpgroup and accumulators each: the two M tiles of a pair over the same key tiles, or, with a single M tile, every other key tile.
// Roles (384 threads), barriers and waits are those of the shared-prefix attention (tree_attn_shared.cu):
//   warp 0            TMA producer: the queries of a segment, then K and V tiles, a box a page, into a ring of 32 KB stages.  Its lanes look the
//                     pages up, a tile ahead; rows behind the last page are a box outside the cache, which arrives as zeros
//   warps 1, 3        MMA issuers of lane 0 and of lane 1: S = Q K^T, O += P V
//   warp 2            planner: walks the work list and puts the segments' descriptions into a ring; checks the segments' pages behind that
//   warps 4..7, 8..11 softmax of lane 0 and of lane 1: one query row a thread; at the segment's end the results.  The lanes of a single M tile are
//                     joined through tensor memory, by the one that has the last tile.  An item that is the CTA's alone is written out; of any other
//                     the CTA leaves a partial result, and the warp that completes a count joins the 32 rows of all CTAs, in the order of the keys
//                     whoever comes last.
// What bounds it.  Long chunks: a lane's chain (scores, exponentials, product), 3080 cycles a pair of tiles of which the exponentials are 2048 and the
// products 2048 (4096 tokens behind 8192, 32 heads over 8: 546 us, 1.26 PFLOP/s in bursts; under the power cap 622).  Short ones: changes of item, some
// 10000 cycles with the first tile behind them (5 prompts of 500 to 1500 tokens, 52 heads: 145 us), and the causal edge
// (with heads of their own lane 0 of a pair has a tile that is masked for all of its tokens).  A token a sequence: HBM, and the TMA boxes of
// pages of 16 rows, some 100 cycles each (64 sequences of 500 to 8192 rows, 32 over 8: 235 us, 5.1 TB/s; pages of 128 rows and equal lengths 5.8).  One token: serial latency
// (511 rows: 10.3 to 12 us).
// Every wait is bounded: one that runs out raises the CTA's abort flag and GOOSE_ST_TIMEOUT, and every role unwinds.
#include <stddef.h>

#include "chunk_work.cuh"
#include "goose_internal.cuh"
#include "tcgen05.cuh"
#include "tree_attn_combine.cuh"

namespace goose {

namespace {

constexpr int kStages = 5;
constexpr int kStageBytes = kChunkTile * kHeadDim * 2;       // 32 KB: one K or one V tile
constexpr int kHalfBytes = kChunkTile * 128;                 // 16 KB: 128 rows x 64 bf16 (one swizzle-atom column)
constexpr int kQBytes = 2 * kHalfBytes;
constexpr int kHeaderBytes = 2048;
constexpr int kChunkSmem = 1008 /*alignment slack*/ + 2 * kQBytes + kStages * kStageBytes + kHeaderBytes;
constexpr int kChunkThreads = 384;
// registers: 168 a thread at launch; the warps of the loads and products give 96 each to the others (72 + 2 x 216 = 3 x 168)
constexpr int kRegsFew = 72, kRegsMany = 216;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleThreshold = 8.0f;                    // rescale O only when the running max grew by > 2^8
constexpr long long kWaitCycles = 2000000000ll;              // bound of every wait: about one second of SM clock

// Partial result of an M tile: 33 words of 16 bytes a row, words of neighbouring rows next to one another: O in fp32, 4 columns a word, as it was summed (rounded
// to fewer bits, parts that nearly cancel would leave the error of the larger ones), then (m, l).  l < 0: rows that cannot be computed.
// A CTA has four places: of its segment that does not begin an item (at most one, its first) and of the one that begins an item and does not end it
// (its last), two M tiles each.
constexpr int kPartSums = kHeadDim / 4, kPartWords = kPartSums + 1;
constexpr uint32_t kPartBlock = kPartWords * kChunkTile;

// a segment, as the planner describes it
struct Segment {
    int n;                                                   // key tiles; 0: the end
    int t_first;
    int ctx, n_keys;                                         // rows in front of the chunk, and all
    int single, whole;                                       // one M tile; the CTA has all of the item
    int s, hk;
    int token;                                               // the sequence's token of the first M tile's first row
    int rows[2];                                             // query rows of the M tiles
    int c0, parts;                                           // CTAs that have a part of the item: the first, how many
    int again;                                               // the rows are read for other items too
    int bad;                                                 // when it has been checked
    int pad;
};
constexpr int kSegments = 6;

struct Header {
    Segment seg[kSegments];
    float2 other[kChunkTile];                                // (m, l) of the lane that does not have a single M tile's last key tile
    // Full: of the key tiles of single M tiles lane by lane (0, 1), of pairs (2).  A parity tells two phases apart, not three: nobody may wait
    // for a phase of a barrier whose phases it has not all followed, and a lane does not follow the tiles of the other one.
    unsigned long long kv_full[3][kStages];
    unsigned long long kv_empty[kStages];
    unsigned long long seg_full[kSegments], seg_empty[kSegments], seg_checked[kSegments];
    // The two places of query tiles.  A pair has both, each lane its own; single M tiles have them in turn.
    unsigned long long pair_full[2], pair_empty[2], single_full[2], single_empty[2];
    unsigned long long s_full[2], v_there[2], o_full[2], o_free[2];
    unsigned long long p_ready[2][2];                        // of a lane, P of either half of a tile's keys
    unsigned long long other_full;                           // `other`, and the product behind it
    uint32_t tmem_base;
    volatile int abort_flag;
};
static_assert(sizeof(Header) <= kHeaderBytes, "header");
static_assert(kChunkSmem <= 232448, "shared memory of a block");

template <typename Int>
struct ChunkArgs {
    ChunkWork<Int> wk;
    Pages pages;
    int g, H;                                                // query heads per key/value head, query heads
    int nb;                                                  // tokens of a box of queries
    int box_log2;                                            // rows of a box of keys
    int wide;                                                // out is aligned for 32-byte stores
    float scale_log2;
    uint4* parts;
    int32_t* counters;                                       // [CTA][M tile][warp], zero between launches
    int32_t* status;
    __nv_bfloat16* out;
    float* lse;
};

__device__ __forceinline__ bool wait_for(Header* hd, unsigned long long* bar, uint32_t parity, int32_t* status) {
    const int r = mbar_wait_bounded(bar, parity, kWaitCycles, &hd->abort_flag);
    if (r == 2) {
        hd->abort_flag = 1;
        atomicOr(status, GOOSE_ST_TIMEOUT);
    }
    return r == 0;
}
__device__ __forceinline__ bool mbar_done(unsigned long long* bar, uint32_t parity) {   // a look, no wait
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ void drain(unsigned long long* bar, uint32_t parity) {   // after an abort
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, parity) && clock64() - t0 < kWaitCycles) {}
}

// a place in a ring of n and its phase
struct Ring {
    uint32_t at, phase;
    __device__ __forceinline__ void next(uint32_t n) {
        if (++at == n) { at = 0; phase ^= 1; }
    }
};

template <typename Int>
__device__ __forceinline__ Int warp_sum(Int v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// the list's length and a place in it, by a whole warp (lane = sequence); false: the CTA has no range
template <typename Int>
__device__ __forceinline__ bool locate(ChunkWork<Int>& wk, ChunkCursor<Int>& cu, ChunkSeq<Int>& q, Int& from, Int& to, int cta, int lane) {
    Int sum = 0;
    bool several = false;
    for (int s0 = 0; s0 < wk.S; s0 += 32)
        if (s0 + lane < wk.S) {
            const ChunkSeq<Int> x = wk.seq(s0 + lane);
            sum += x.before(x.pairs);
            several |= x.n > wk.t;
        }
    wk.set(warp_sum(sum), __any_sync(0xFFFFFFFFu, several));
    from = wk.start(cta);
    to = wk.start(cta + 1);
    if (from >= to) return false;
    Int begin = 0;
    for (int s0 = 0; s0 < wk.S; s0 += 32) {
        Int own = 0;
        if (s0 + lane < wk.S) {
            const ChunkSeq<Int> x = wk.seq(s0 + lane);
            own = wk.Hkv * x.before(x.pairs);
        }
        Int upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const Int u = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += u;
        }
        const uint32_t here = __ballot_sync(0xFFFFFFFFu, begin + upto > from);
        if (here) {
            const int l = __ffs(here) - 1;
            cu.s = s0 + l;
            q = wk.seq(cu.s);
            cu.enter(q, begin + __shfl_sync(0xFFFFFFFFu, upto - own, l), from);
            return true;
        }
        begin += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    return false;
}

// The same wait for the softmax warps, which have few registers to spare: 32-bit addresses and clock.
__device__ __forceinline__ bool wait_at(uint32_t bar, uint32_t parity, uint32_t abort_flag, int32_t* status) {
    auto done = [&]() {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        return ok != 0;
    };
    if (done()) return true;
    const uint32_t t0 = (uint32_t)clock();
    for (;;) {
        if (done()) return true;
        uint32_t raised;
        asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(raised) : "r"(abort_flag) : "memory");
        if (raised) return false;
        if ((uint32_t)clock() - t0 > (uint32_t)kWaitCycles) break;
    }
    asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(abort_flag), "r"(1) : "memory");
    atomicOr(status, GOOSE_ST_TIMEOUT);
    return false;
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Joins the partial results of 32 rows (row0 on) of M tile l of an item that the CTAs c0 .. c0 + n - 1 have, by one warp: lanes <-> rows, and where the
// rows are fewer, several lanes share a row's columns.  kCols columns a time, kRound parts in flight.
template <int kCols, int kRound, typename Int>
__device__ __forceinline__ void join_parts(const ChunkArgs<Int>& a, int c0, int n, int l, int row0, int rows, int lane, size_t out_row /* of this lane's row */,
                                           int width, bool write_lse) {
    const int r = lane & (width - 1);
    for (int c = lane / width * kCols; c < kHeadDim; c += 32 / width * kCols) {
        float M = -INFINITY, L = 0.f, acc[kCols];
        bool bad = false;
#pragma unroll
        for (int e = 0; e < kCols; ++e) acc[e] = 0.f;
        for (int k0 = 0; k0 < n; k0 += kRound) {
            float2 ml[kRound];
            float4 x[kRound][kCols / 4];
#pragma unroll
            for (int u = 0; u < kRound; ++u) {
                const int k = k0 + u;
                ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int w = 0; w < kCols / 4; ++w) x[u][w] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < n && row0 + r < rows) {
                    const uint4* part = a.parts + (size_t)(4 * (c0 + k) + (k == 0 ? 2 : 0) + l) * kPartBlock + row0 + r;
                    ml[u] = __ldcg(reinterpret_cast<const float2*>(part + kPartSums * kChunkTile));
#pragma unroll
                    for (int w = 0; w < kCols / 4; ++w) x[u][w] = __ldcg(reinterpret_cast<const float4*>(part + (c / 4 + w) * kChunkTile));
                }
            }
#pragma unroll
            for (int u = 0; u < kRound; ++u) {
                bad |= ml[u].y < 0.f;
                if (ml[u].x == -INFINITY && ml[u].y == 0.f) continue;   // no key of the part is visible to the row
                const float M_new = fmaxf(M, ml[u].x), old = M == -INFINITY ? 0.f : ex2(M - M_new);
                const float w = ml[u].x == -INFINITY ? 1.f : ex2(ml[u].x - M_new);   // (NaN alone: it stays one)
                M = M_new;
                L = __fmaf_rn(w, ml[u].y, __fmul_rn(L, old));
#pragma unroll
                for (int v = 0; v < kCols / 4; ++v) {
                    float* o = acc + 4 * v;
                    o[0] = __fmaf_rn(w, x[u][v].x, __fmul_rn(o[0], old));
                    o[1] = __fmaf_rn(w, x[u][v].y, __fmul_rn(o[1], old));
                    o[2] = __fmaf_rn(w, x[u][v].z, __fmul_rn(o[2], old));
                    o[3] = __fmaf_rn(w, x[u][v].w, __fmul_rn(o[3], old));
                }
            }
        }
        if (row0 + r < rows) {
            const float inv = bad ? 0.f : 1.f / L;
            uint4* dst = reinterpret_cast<uint4*>(a.out + out_row * kHeadDim + c);
#pragma unroll
            for (int e = 0; e < kCols; e += 8)
                dst[e / 8] = bad ? make_uint4(0, 0, 0, 0)
                                 : make_uint4(pack_bf16x2(acc[e] * inv, acc[e + 1] * inv), pack_bf16x2(acc[e + 2] * inv, acc[e + 3] * inv),
                                              pack_bf16x2(acc[e + 4] * inv, acc[e + 5] * inv), pack_bf16x2(acc[e + 6] * inv, acc[e + 7] * inv));
            if (write_lse && c == 0) a.lse[out_row] = bad ? kNoLse : (M + log2f(L)) * kLn2;
        }
    }
}

template <typename Int>
__global__ void __launch_bounds__(kChunkThreads, 1)
chunk_attn_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ ChunkArgs<Int> a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* q_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* kv_smem = q_smem + 2 * kQBytes;
    Header* hd = reinterpret_cast<Header*>(kv_smem + kStages * kStageBytes);
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { for (int u = 0; u < 3; ++u) mbar_init(&hd->kv_full[u][i], 1); mbar_init(&hd->kv_empty[i], 2); }
        for (int i = 0; i < kSegments; ++i) { mbar_init(&hd->seg_full[i], 1); mbar_init(&hd->seg_empty[i], 3 + 8); mbar_init(&hd->seg_checked[i], 1); }
        for (int l = 0; l < 2; ++l) {
            mbar_init(&hd->pair_full[l], 1); mbar_init(&hd->pair_empty[l], 1); mbar_init(&hd->single_full[l], 1); mbar_init(&hd->single_empty[l], 2);
            mbar_init(&hd->s_full[l], 1); mbar_init(&hd->v_there[l], 1); mbar_init(&hd->p_ready[l][0], 4); mbar_init(&hd->p_ready[l][1], 4); mbar_init(&hd->o_full[l], 1); mbar_init(&hd->o_free[l], 4);
        }
        mbar_init(&hd->other_full, 4);
        hd->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&tmap_q); prefetch_tmap(&tmap_k); prefetch_tmap(&tmap_v);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&hd->tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, hd->tmem_base, 0);
    pdl_wait();
    pdl_trigger();

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
        if (warp == 2) {
            // =========================================================== planner
            ChunkWork<Int> wk = a.wk;
            if (wk.n_new && blockIdx.x == 0)
                for (int s = lane; s < wk.S; s += 32)
                    if (nodes_bad(wk.n_new, s, wk.B)) atomicOr(&a.status[s], GOOSE_ST_BAD_NODES);
            ChunkCursor<Int> cu{};
            ChunkSeq<Int> q{};
            Int from, to;
            bool live = locate(wk, cu, q, from, to, blockIdx.x, lane);
            auto advance = [&]() {
                if (cu.next(wk, q)) return;
                do {
                    if (++cu.s < wk.S) q = wk.seq(cu.s);
                } while (cu.s < wk.S && q.pairs == 0);
                cu.hk = cu.p = 0;
                live = cu.s < wk.S;
            };
            Ring ring{0, 0};
            for (;;) {
                bool any = false;
                while (live && cu.w0 < to) {
                    cu.look(wk, q, blockIdx.x, from, to);
                    any = cu.t1 > cu.t0;
                    if (any) break;
                    advance();
                }
                if (!wait_for(hd, &hd->seg_empty[ring.at], ring.phase ^ 1, a.status)) break;
                Segment* sg = &hd->seg[ring.at];
                if (lane == 0) {
                    sg->n = any ? cu.t1 - cu.t0 : 0;
                    if (any) {
                        const int left = q.n - cu.p * q.step, here = min(left, q.step);   // tokens of the item
                        sg->t_first = cu.t0; sg->ctx = q.ctx; sg->n_keys = q.ctx + q.n;
                        sg->single = here <= wk.t; sg->whole = cu.c0 == cu.c1;
                        sg->s = cu.s; sg->hk = cu.hk; sg->token = cu.p * q.step;
                        sg->rows[0] = min(here, wk.t) * a.g;
                        sg->rows[1] = max(here - wk.t, 0) * a.g;
                        sg->c0 = cu.c0; sg->parts = cu.c1 - cu.c0 + 1;
                        sg->again = q.pairs > 1;
                    }
                    mbar_arrive(&hd->seg_full[ring.at]);
                }
                __syncwarp();
                if (!any) break;
                // the segment's pages: who needs to know asks at its end
                bool bad = q.bad;
                if (!bad) {
                    const int lg = a.pages.size_log2;
                    const int p1 = (min(cu.t1 * kChunkTile, q.ctx + q.n) - 1) >> lg;
                    for (int p = ((cu.t0 * kChunkTile) >> lg) + lane; p <= p1; p += 32) {
                        const int page = a.pages.table[cu.s * a.pages.ldt + p];
                        bad |= page < 0 || page >= a.pages.n;
                    }
                }
                bad = __any_sync(0xFFFFFFFFu, bad);
                if (lane == 0) {
                    sg->bad = bad;
                    if (bad) atomicOr(&a.status[cu.s], GOOSE_ST_BAD_ROWS);
                    mbar_arrive(&hd->seg_checked[ring.at]);
                }
                __syncwarp();
                ring.next(kSegments);
                advance();
            }
        } else if (warp == 0) {
            // =========================================================== TMA producer (the warp runs converged)
            const bool leader = elect_leader();
            const unsigned long long pol_once = l2_policy_evict_first(), pol_again = l2_policy_evict_last();
            const uint32_t kv_addr = smem_u32(kv_smem);
            const int boxes = kChunkTile >> a.box_log2, outside = a.pages.n << a.pages.size_log2;
            uint32_t pairs = 0, singles = 0, tile0 = 0;      // segments of either kind, tiles in front of this segment
            uint32_t phases = 0, users = 0;                  // a bit a kv_full barrier; two bits a stage: who has it, 3: nobody yet
            for (int i = 0; i < kStages; ++i) users |= 3u << 2 * i;
            Ring st{0, 0}, ring{0, 0};
            bool ok = true;
            Segment sg{};
            uint32_t asked = 0;                              // query tiles of the segment that still wait for their place
            auto all = [](bool x) { return __all_sync(0xFFFFFFFFu, x) != 0; };
            auto load_q = [&](int b) {
                const int first = sg.s * a.wk.B + sg.token + (sg.single ? 0 : b) * a.wk.t;
                unsigned long long* full = sg.single ? &hd->single_full[b] : &hd->pair_full[b];
                if (leader) {
                    mbar_expect_tx(full, (uint32_t)(a.nb * a.g) * 256u);
                    tma_load_4d(q_smem + b * kQBytes, &tmap_q, full, 0, 0, sg.hk, first);
                    tma_load_4d(q_smem + b * kQBytes + kHalfBytes, &tmap_q, full, 64, 0, sg.hk, first);
                }
                __syncwarp();
                asked &= ~(1u << b);
            };
            // place b is free when the last pair and the last single M tile that had it are done
            auto pair_parity = [&]() { return (pairs & 1) ^ 1; };
            auto single_parity = [&](int b) { return ((singles + 1 - b) >> 1 & 1) ^ 1; };
            // The key tiles do not wait for the queries' place: a pair's is free only when the products of the segment in front
            // are done, and the ring would run dry meanwhile.
            auto stage_free = [&]() {
                const long long t0 = clock64();
                while (asked) {
                    for (int b = 0; b < 2; ++b)
                        if ((asked >> b & 1) && all(mbar_done(&hd->pair_empty[b], pair_parity()) && mbar_done(&hd->single_empty[b], single_parity(b)))) load_q(b);
                    if (all(mbar_done(&hd->kv_empty[st.at], st.phase ^ 1))) return true;
                    if (!all(!(hd->abort_flag || clock64() - t0 > kWaitCycles))) break;   // (the wait below says so)
                }
                return all(wait_for(hd, &hd->kv_empty[st.at], st.phase ^ 1, a.status));
            };
            // the cache row of this lane's box of tile t: no page behind the sequence's last row is looked up
            auto box_row = [&](int t) {
                const int j = (t << 7) + (lane << a.box_log2), page = j >> a.pages.size_log2;
                if (lane >= boxes || j >= sg.n_keys || page >= a.pages.ldt) return outside;
                const int at = a.pages.table[sg.s * a.pages.ldt + page];
                return at < 0 || at >= a.pages.n ? outside : (at << a.pages.size_log2) + (j & ((1 << a.pages.size_log2) - 1));
            };
            while (ok) {
                for (int b = 0; b < 2 && ok; ++b)            // of the segment in front
                    if (asked >> b & 1) {
                        ok = all(wait_for(hd, &hd->pair_empty[b], pair_parity(), a.status) && wait_for(hd, &hd->single_empty[b], single_parity(b), a.status));
                        if (ok) load_q(b);
                    }
                if (ok && sg.n > 0) { if (sg.single) ++singles; else ++pairs; sg.n = 0; }
                ok = ok && all(wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status));
                if (!ok) break;
                sg = hd->seg[ring.at];
                __syncwarp();
                if (leader) mbar_arrive(&hd->seg_empty[ring.at]);
                ring.next(kSegments);
                if (sg.n == 0) break;
                asked = sg.single ? 1u << (singles & 1) : 3u;
                const unsigned long long pol = sg.again ? pol_again : pol_once;
                int row = box_row(sg.t_first);
                for (int i = 0; i < sg.n && ok; ++i) {
                    const int ahead = i + 1 < sg.n ? box_row(sg.t_first + i + 1) : outside;
                    const uint32_t user = sg.single ? (tile0 + i) & 1 : 2;
                    for (int kv = 0; kv < 2 && ok; ++kv) {
                        ok = stage_free();
                        if (!ok) break;
                        unsigned long long* full = &hd->kv_full[user][st.at];
                        if (leader) mbar_expect_tx(full, kStageBytes);
                        __syncwarp();
                        const CUtensorMap* mp = kv ? &tmap_v : &tmap_k;
                        const uint32_t dst = kv_addr + st.at * kStageBytes;
                        int from[8];                         // (all of them ahead of the copies: a copy behind a shuffle waits for it)
#pragma unroll
                        for (int b = 0; b < 8; ++b) from[b] = __shfl_sync(0xFFFFFFFFu, row, b);
#pragma unroll
                        for (int b = 0; b < 8; ++b) {
                            if (b >= boxes) break;
                            const uint32_t to = dst + ((uint32_t)b << (a.box_log2 + 7));
                            tma_load_3d_hint_by(leader, to, mp, full, 0, sg.hk, from[b], pol);
                            tma_load_3d_hint_by(leader, to + kHalfBytes, mp, full, 64, sg.hk, from[b], pol);
                        }
                        phases ^= 1u << (user * kStages + st.at);
                        users = (users & ~(3u << 2 * st.at)) | user << 2 * st.at;
                        st.next(kStages);
                    }
                    row = ahead;
                }
                tile0 += sg.n;
            }
            // The products' arrivals have landed, too, before the CTA ends: those that free stages and queries' places are behind the one
            // that the epilogue waits for.
            for (int i = 0; i < kStages && ok; ++i, st.next(kStages)) ok = all(wait_for(hd, &hd->kv_empty[st.at], st.phase ^ 1, a.status));
            for (int b = 0; b < 2 && ok; ++b)
                ok = all(wait_for(hd, &hd->pair_empty[b], pair_parity(), a.status) && wait_for(hd, &hd->single_empty[b], single_parity(b), a.status));
            if (!ok) {                                       // copies still in flight land before the CTA ends
                for (int i = 0; i < kStages; ++i) {
                    const uint32_t user = users >> 2 * i & 3;
                    if (user < 3) drain(&hd->kv_full[user][i], (phases >> (user * kStages + i) & 1) ^ 1);
                }
                if (sg.n > 0 && sg.single && !asked) ++singles;   // (only copies that began)
                for (int b = 0; b < 2; ++b) {
                    const uint32_t of_pairs = pairs + (sg.n > 0 && !sg.single && !(asked >> b & 1)), of_singles = (singles + 1 - b) >> 1;
                    if (of_pairs > 0) drain(&hd->pair_full[b], (of_pairs - 1) & 1);
                    if (of_singles > 0) drain(&hd->single_full[b], (of_singles - 1) & 1);
                }
            }
        } else {
            // =========================================================== MMA issuers: warp 1 for lane 0, warp 3 for lane 1
            const bool leader = elect_leader();              // the warp runs converged, this lane acts
            const uint32_t l = warp >> 1;
            const uint32_t q_addr = smem_u32(q_smem), kv_addr = smem_u32(kv_smem);
            const uint32_t s_tmem = tmem + kColS + l * 128, o_tmem = tmem + kColO + l * 128;
            constexpr uint32_t idesc_qk = instr_desc(false), idesc_pv = instr_desc(true);
            uint32_t ops = 0, segs = 0, tile0 = 0;           // products, segments of this lane; tiles of the CTA
            uint32_t pairs = 0, singles = 0;                 // segments of the CTA
            Ring ring{0, 0};
            bool ok = true;
            uint32_t phases = 0;                             // a bit a kv_full barrier of this lane and, kStages further, of pairs
            bool single = false;
            // K of tile i of the CTA is load 2 i, V load 2 i + 1; once a load
            auto stage_full = [&](uint32_t load) {
                const uint32_t at = load % kStages, bit = single ? at : kStages + at;
                const uint32_t parity = phases >> bit & 1;
                phases ^= 1u << bit;
                return wait_for(hd, &hd->kv_full[single ? l : 2][at], parity, a.status);
            };
            while (ok) {
                ok = wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status);
                if (!ok) break;
                const int n = __shfl_sync(0xFFFFFFFFu, hd->seg[ring.at].n, 0);   // (uniform registers)
                single = __shfl_sync(0xFFFFFFFFu, hd->seg[ring.at].single, 0) != 0;
                __syncwarp();
                if (leader) mbar_arrive(&hd->seg_empty[ring.at]);
                ring.next(kSegments);
                if (n == 0) break;
                const uint32_t place = single ? singles & 1 : l;
                unsigned long long* const q_full = single ? &hd->single_full[place] : &hd->pair_full[l];
                unsigned long long* const q_empty = single ? &hd->single_empty[place] : &hd->pair_empty[l];
                ok = wait_for(hd, q_full, (single ? singles >> 1 : pairs) & 1, a.status);
                if (!ok) break;
                const uint32_t q_lo = smem_desc_lo(q_addr + place * kQBytes, 16);
                const uint32_t step = single ? 2 : 1, end = tile0 + n;
                auto release = [&](uint32_t load) {          // every stage has two arrivals
                    umma_commit_by(leader, &hd->kv_empty[load % kStages]);
                    if (single && leader) mbar_arrive(&hd->kv_empty[load % kStages]);
                };
                auto scores = [&](uint32_t t) {
                    tc_fence_after();
                    const uint32_t k_lo = smem_desc_lo(kv_addr + (2 * t % kStages) * kStageBytes, 16);
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {         // 16 of the 128 head dims per instruction
                        const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
                        umma_f16_by(leader, s_tmem, smem_desc(q_lo + off), smem_desc(k_lo + off), idesc_qk, kk > 0 ? 1u : 0u);
                    }
                    umma_commit_by(leader, &hd->s_full[l]);             // (and with it the product in front of it)
                };
                uint32_t t = tile0 + (single ? (tile0 ^ l) & 1 : 0);
                const bool any = t < end;
                if (any) {
                    ok = stage_full(2 * t);
                    if (!ok) break;
                    scores(t);
                    release(2 * t);
                }
                if (t + step >= end) {                       // the lane's last Q K^T of the segment
                    if (any) umma_commit_by(leader, q_empty);
                    else if (leader) mbar_arrive(q_empty);
                }
                if (any && segs > 0) ok = wait_for(hd, &hd->o_free[l], (segs - 1) & 1, a.status);
                for (bool first = true; t < end && ok; t += step, first = false) {
                    const bool more = t + step < end;
                    // A look at a barrier takes some 150 cycles beside the tensor cores' reads of shared memory: those at the tiles come
                    // first, while P is still being made.  (The next K of a single M tile may only be on its way behind the other
                    // lane's product.)
                    if (!(ok = stage_full(2 * t + 1))) break;
                    if (leader) mbar_arrive(&hd->v_there[l]);
                    if (more && !single && !(ok = stage_full(2 * (t + step)))) break;
                    const uint32_t v_lo = smem_desc_lo(kv_addr + ((2 * t + 1) % kStages) * kStageBytes, kHalfBytes);   // MN-major: LBO = next 64 d
                    // the product with the first half's P runs beside the exponentials of the second
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!(ok = wait_for(hd, &hd->p_ready[l][h], ops & 1, a.status))) break;
                        tc_fence_after();
#pragma unroll
                        for (int kk = 4 * h; kk < 4 * h + 4; ++kk)   // 16 keys per instruction
                            umma_f16_ts_by(leader, o_tmem, s_tmem + kk * 8, smem_desc(v_lo + kk * (2048 >> 4)), idesc_pv, !first || kk > 0 ? 1u : 0u);
                    }
                    if (!ok) break;
                    ++ops;
                    if (more) {
                        if (single && !(ok = stage_full(2 * (t + step)))) break;
                        scores(t + step);
                    } else {
                        umma_commit_by(leader, &hd->o_full[l]);
                    }
                    release(2 * t + 1);
                    if (more) {
                        release(2 * (t + step));
                        if (t + 2 * step >= end) umma_commit_by(leader, q_empty);
                    }
                }
                if (!ok) break;
                segs += any;
                if (single) ++singles; else ++pairs;
                tile0 = end;
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsMany));
        // =============================================================== softmax and results
        const int l = (warp - 4) >> 2;                       // lane of the segments
        const int row = 32 * (warp & 3) + lane;              // TMEM lane == query row
        const uint32_t s_addr = tmem + kColS + l * 128 + ((uint32_t)(32 * (warp & 3)) << 16);   // O: kColO - kColS further
        const uint32_t base = smem_u32(hd), my_bars = base + 8 * l, abort_at = base + (uint32_t)offsetof(Header, abort_flag);
        constexpr uint32_t kAtFull = offsetof(Header, s_full), kAtDone = offsetof(Header, o_full);
        constexpr uint32_t kAtFree = offsetof(Header, o_free);
        const uint32_t at_ready = base + (uint32_t)offsetof(Header, p_ready) + 16 * l;
        uint32_t ops = 0, segs = 0, tile0 = 0;               // products and segments of this lane; tiles of the CTA in front of this segment
        uint32_t joins = 0;                                  // segments of the CTA whose lanes have been joined
        Ring ring{0, 0};
        bool ok = true;
        uint32_t v[128];

        for (;;) {
            ok = wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status);
            if (!ok) break;
            const Segment& sg = hd->seg[ring.at];
            if (sg.n == 0) break;
            const int step = sg.single ? 2 : 1, t_end = sg.t_first + sg.n;
            const int turn = sg.single ? (tile0 ^ l) & 1 : l;   // a single M tile's key tiles are dealt on where the segment in front ended
            const int m_tile = sg.single ? 0 : l;
            const int rows = sg.rows[m_tile];
            const bool row_valid = row < rows, warp_has_rows = (row & ~31) < rows;
            // keys that the M tile's first token sees; from t_masked on a tile has keys behind a token
            auto seen = [&]() { return sg.ctx + sg.token + m_tile * a.wk.t + 1; };
            const int t_masked = seen() / kChunkTile;
            float m_run = -INFINITY, l_run = 0.f;
            bool first = true;
            for (int t = sg.t_first + (sg.single ? turn : 0); t < t_end; t += step) {
                ok = wait_at(my_bars + kAtFull, ops & 1, abort_at, a.status);
                if (!ok) break;
                tc_fence_after();
                // ragged end: V rows past the last key may hold anything -> zeros (by either lane of a tile that both use)
                if ((t + 1) * kChunkTile > sg.n_keys) {
                    const uint32_t load = 2 * (tile0 + (t - sg.t_first)) + 1, st = load % kStages;
                    ok = wait_for(hd, &hd->v_there[l], ops & 1, a.status);
                    if (!ok) break;
                    const int first_off = max(sg.n_keys - t * kChunkTile, 0) * 128;
                    for (int off = first_off + row * 16; off < kHalfBytes; off += 128 * 16) {
                        *reinterpret_cast<uint4*>(kv_smem + st * kStageBytes + off) = make_uint4(0, 0, 0, 0);
                        *reinterpret_cast<uint4*>(kv_smem + st * kStageBytes + kHalfBytes + off) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async();
                }
                if (warp_has_rows) {
                    TMEM_LD32(s_addr, v, 0); TMEM_LD32(s_addr + 32, v, 32);
                    TMEM_LD32(s_addr + 64, v, 64); TMEM_LD32(s_addr + 96, v, 96);
                    tmem_wait_ld();
                    if (t >= t_masked) {
                        const int upto = seen() + row / a.g - t * kChunkTile;   // columns that the row sees
                        uint32_t vw[4];
#pragma unroll
                        for (int w = 0; w < 4; ++w) vw[w] = upto >= 32 * w + 32 ? 0xFFFFFFFFu : upto <= 32 * w ? 0u : (1u << (upto - 32 * w)) - 1;
#pragma unroll
                        for (int c = 0; c < 128; ++c) v[c] = ((vw[c >> 5] >> (c & 31)) & 1u) ? v[c] : 0xFF800000u;   // -inf
                    }
                    float mx[8] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 128; c += 16)
#pragma unroll
                        for (int e = 0; e < 8; ++e) mx[e] = max3(mx[e], __uint_as_float(v[c + 2 * e]), __uint_as_float(v[c + 2 * e + 1]));
#pragma unroll
                    for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], mx[e + 4]);
                    const float m_new = fmaxf(m_run, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2);   // scale > 0
                    if (__any_sync(0xFFFFFFFFu, first || (row_valid && m_new > m_run + kRescaleThreshold))) {
                        const float alpha = (m_run == -INFINITY) ? 0.f : ex2(m_run - m_new);
                        if (!first) {                        // (these scores are there: so is the product in front of them)
                            uint32_t o[16];
#pragma unroll
                            for (int cc = 0; cc < 8; ++cc) {
                                TMEM_LD16(s_addr + (kColO - kColS) + cc * 16, o, 0);
                                tmem_wait_ld();
#pragma unroll
                                for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
                                TMEM_ST16(s_addr + (kColO - kColS) + cc * 16, o, 0);
                            }
                            tmem_wait_st();
                        }
                        l_run *= alpha;
                        m_run = m_new;
                    }
                    const float neg_m = (m_run == -INFINITY) ? 0.f : -m_run;
                    const unsigned long long scale2 = pack_f32x2(a.scale_log2, a.scale_log2), neg2 = pack_f32x2(neg_m, neg_m);
                    unsigned long long ls2[2] = {0, 0};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int e = 32 * h; e < 32 * h + 32; ++e) {
                            const float2 x2 = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), scale2, neg2));
                            const float p0 = ex2(x2.x), p1 = ex2(x2.y);
                            ls2[e & 1] = add_f32x2(ls2[e & 1], pack_f32x2(p0, p1));
                            v[e] = pack_bf16x2(p0, p1);   // P as V's type, as the product takes it: 2^-9 of a term, either way; the sum above is of p itself
                        }
                        TMEM_ST32(s_addr + 32 * h, v, 32 * h);
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive_at(at_ready + 8 * h);
                    }
                    const float2 l2 = unpack_f32x2(add_f32x2(ls2[0], ls2[1]));
                    l_run += l2.x + l2.y;
                } else {
                    tc_fence_before();
                    __syncwarp();                            // (all lanes' zeros are in front of the arrivals)
                    if (lane == 0) { arrive_at(at_ready); arrive_at(at_ready + 8); }
                }
                first = false;
                ++ops;
            }
            if (!ok) break;
            ok = wait_for(hd, &hd->seg_checked[ring.at], ring.phase, a.status);
            if (!ok) break;
            const bool two = sg.single && sg.n > 1;          // both lanes have key tiles of the one M tile
            if (!first) {
                ok = wait_at(my_bars + kAtDone, segs & 1, abort_at, a.status);
                if (!ok) break;
                ++segs;
                tc_fence_after();
            }
            if (!first && two && turn != ((sg.n - 1) & 1)) { // the lane that has the last tile takes what this one has
                hd->other[row] = make_float2(m_run, l_run);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at(base + (uint32_t)offsetof(Header, other_full));
            } else if (!first) {
                if (two) {
                    ok = wait_at(base + (uint32_t)offsetof(Header, other_full), joins & 1, abort_at, a.status);
                    if (!ok) break;
                    tc_fence_after();
                }
                auto release = [&]() {                       // the accumulators have been read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        arrive_at(my_bars + kAtFree);
                        if (two) arrive_at(base + kAtFree + 8 * (l ^ 1));
                    }
                };
                if (!warp_has_rows) {
                    release();
                } else {
                    const uint32_t o_addr = s_addr + (kColO - kColS);
                    if (two) {                               // (into tensor memory again: a row and a part of another one are more than the registers hold)
                        const float2 other = hd->other[row];
                        const float m = fmaxf(m_run, other.x);
                        const float mine = m_run == -INFINITY ? 0.f : ex2(m_run - m), theirs = other.x == -INFINITY ? 0.f : ex2(other.x - m);
                        // (a lane whose scores are all NaN has a sum of NaN and no maximum)
                        l_run = l_run * (m_run == -INFINITY ? 1.f : mine) + other.y * (other.x == -INFINITY ? 1.f : theirs);
                        m_run = m;
                        const uint32_t other_addr = tmem + kColO + (l ^ 1) * 128 + ((uint32_t)(32 * (warp & 3)) << 16);
#pragma unroll
                        for (int cc = 0; cc < 4; ++cc) {
                            TMEM_LD32(o_addr + 32 * cc, v, 0); TMEM_LD32(other_addr + 32 * cc, v, 32);
                            tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(__uint_as_float(v[c]) * mine + __uint_as_float(v[32 + c]) * theirs);
                            TMEM_ST32(o_addr + 32 * cc, v, 0);
                        }
                        tmem_wait_st();
                    }
                    TMEM_LD32(o_addr, v, 0); TMEM_LD32(o_addr + 32, v, 32);
                    TMEM_LD32(o_addr + 64, v, 64); TMEM_LD32(o_addr + 96, v, 96);
                    tmem_wait_ld();
                    release();
                    const int first_token = sg.s * a.wk.B + sg.token + m_tile * a.wk.t;
                    if (sg.whole) {
                        if (row_valid) {
                            const int node = row / a.g;
                            const size_t at = ((size_t)first_token + node) * a.H + sg.hk * a.g + (row - node * a.g);
                            const float inv = 1.f / l_run;
                            __nv_bfloat16* dst = a.out + at * kHeadDim;
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                uint32_t w[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    w[e] = sg.bad ? 0u : pack_bf16x2(__uint_as_float(v[16 * c + 2 * e]) * inv, __uint_as_float(v[16 * c + 2 * e + 1]) * inv);
                                if (a.wide) {                // (rows are far apart: half the requests; 5 prompts, 52 heads: 144 us, by 16 bytes 146)
                                    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst + 16 * c), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                                                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
                                } else {
                                    reinterpret_cast<uint4*>(dst)[2 * c] = make_uint4(w[0], w[1], w[2], w[3]);
                                    reinterpret_cast<uint4*>(dst)[2 * c + 1] = make_uint4(w[4], w[5], w[6], w[7]);
                                }
                            }
                            if (a.lse) a.lse[at] = sg.bad ? kNoLse : (m_run + log2f(l_run)) * kLn2;
                        }
                    } else {
                        if (row_valid) {
                            uint4* part = a.parts + (size_t)(4 * blockIdx.x + (sg.t_first == 0 ? 2 : 0) + m_tile) * kPartBlock + row;
#pragma unroll
                            for (int c = 0; c < kPartSums; ++c) part[c * kChunkTile] = make_uint4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                            *reinterpret_cast<float2*>(part + kPartSums * kChunkTile) = make_float2(m_run, sg.bad ? -1.f : l_run);
                        }
                        __threadfence();
                        __syncwarp();
                        int32_t* counter = a.counters + (2 * sg.c0 + m_tile) * 4 + (warp & 3);
                        int last = 0;
                        if (lane == 0) last = atomicAdd(counter, 1) == sg.parts - 1;
                        last = __shfl_sync(0xFFFFFFFFu, last, 0);
                        if (last) {
                            __threadfence();
                            if (lane == 0) *counter = 0;
                            const int row0 = row & ~31, here = min(rows - row0, 32);
                            const int width = here > 1 ? 1 << (32 - __clz(here - 1)) : 1;
                            const int r = row0 + (lane & (width - 1)), node = r / a.g;
                            const size_t at = ((size_t)first_token + node) * a.H + sg.hk * a.g + (r - node * a.g);
                            // few rows are a chain of parts, many are requests (a token behind 2400 rows, groups of 4: 18 us, the other way 20; 60 tokens behind 500: 25, and 29)
                            if (width <= 4) join_parts<16, 4>(a, sg.c0, sg.parts, m_tile, row0, rows, lane, at, width, a.lse != nullptr);
                            else join_parts<32, 2>(a, sg.c0, sg.parts, m_tile, row0, rows, lane, at, width, a.lse != nullptr);
                        }
                    }
                }
            }
            joins += two;
            tile0 += sg.n;
            __syncwarp();
            if (lane == 0) mbar_arrive(&hd->seg_empty[ring.at]);
            ring.next(kSegments);
        }
    }

    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

}  // namespace

template <typename Int>
static cudaError_t launch_as(goose_ctx* c, const ChunkAttn& x, cudaStream_t st) {
    ChunkArgs<Int> a{};
    a.g = x.H / x.Hkv; a.H = x.H;
    a.wk.ctx_len = x.ctx_len; a.wk.n_new = x.n_new; a.wk.S = x.S; a.wk.B = x.B; a.wk.Hkv = x.Hkv; a.wk.G = c->num_sms;
    a.wk.t = kChunkTile / a.g; a.wk.room = (int)x.pages.room(0);
    a.pages = x.pages; a.box_log2 = x.pages.size_log2 < 7 ? x.pages.size_log2 : 7;
    a.nb = a.wk.t < x.B ? a.wk.t : x.B;
    a.wide = (reinterpret_cast<uintptr_t>(x.out) & 31) == 0;
    a.scale_log2 = x.scale * kLog2e;
    a.parts = static_cast<uint4*>(c->chunk_parts);
    a.counters = c->chunk_counters; a.status = c->status; a.out = x.out; a.lse = x.lse;
    CUtensorMap mq, mk, mv;
    const int64_t rows = (int64_t)x.pages.n << x.pages.size_log2;
    if (!make_q_map(c->encode_tiled, &mq, x.q, (int64_t)x.S * x.B, x.Hkv, a.g, a.nb) || !make_map(c->encode_tiled, &mk, x.k_cache, rows, x.Hkv, 1 << a.box_log2) ||
        !make_map(c->encode_tiled, &mv, x.v_cache, rows, x.Hkv, 1 << a.box_log2))
        return cudaErrorInvalidValue;
    cudaError_t e = launch_pdl(chunk_attn_kernel<Int>, dim3(c->num_sms), dim3(kChunkThreads), kChunkSmem, st, mq, mk, mv, a);
    c->launches++;
    return e;
}

cudaError_t launch_chunk_attn(goose_ctx* c, const ChunkAttn& x, cudaStream_t st) {
    if (!c->encode_tiled) return cudaErrorNotSupported;
    if (x.S == 0) return cudaSuccess;
    if (cudaError_t e = grow(c, &c->chunk_parts, &c->chunk_bytes, sizeof(uint4) * kPartBlock * 4 * (size_t)c->num_sms)) return e;
    const bool small = ChunkWork<int>::most(x.S, x.B, x.Hkv, kChunkTile / (x.H / x.Hkv), (int)x.pages.room(0)) < kShortPlaces;
    return small ? launch_as<int>(c, x, st) : launch_as<long long>(c, x, st);
}

cudaError_t init_chunk_kernels() {
    cudaError_t e = cudaFuncSetAttribute(chunk_attn_kernel<int>, cudaFuncAttributeMaxDynamicSharedMemorySize, kChunkSmem);
    return e == cudaSuccess ? cudaFuncSetAttribute(chunk_attn_kernel<long long>, cudaFuncAttributeMaxDynamicSharedMemorySize, kChunkSmem) : e;
}

}  // namespace goose
