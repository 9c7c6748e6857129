// The attention that every cached row got from a chunk's tokens: W[s][hk][j] += sum_{i, h in group hk} exp(x_ihj - lse_ih), x_ihj = scale q_ih . k_j,
// over the tokens i >= j - ctx.
//
// Persistent, one CTA an SM, tcgen05: S^T = K Q^T with the keys as rows, so that a thread has a key, and its sum needs no exchange; up to
// four key tiles of a run stay in shared memory while the Q tiles pass by.  The log-sum-exps come with the product: one more step of 16 of its inner
// dimension adds -lse / scale to every score of a column, in three bf16 that together have its 24 bits, times ones.  It is the last step, so that the
// steps in front of it are rounded by the size of the scores alone.  (A thread that reads every column's from shared memory instead, 16 bytes at a
// time, takes as much of its bandwidth as the product does: 2048 tokens behind 4096, 32 heads over 8: 127 us, so 112.)  Work list: weights_work.cuh.  Roles (768 threads):
//   warp 0            Q tiles into a ring of two, by TMA
//   warp 1            MMA issuer: the scores of key tile u of the run into columns 128 u of tensor memory
//   warp 2            planner: walks the work list and puts the segments' descriptions into a ring
//   warp 3            the product's last step for a Q tile's rows, and which of the rows count
//   warps 4..19       exponentials, four warps a key tile of the run, a key and a sum a thread.  At the segment's end the sums are added to the
//                     rows' weights, or, where several CTAs have Q tiles of the item, left in the workspace; the warp that completes a count adds up what
//                     all have left, in the order of the tokens.
//   warps 20..23      K tiles into a ring of four, 32 keys of a tile a warp, by 16-byte copies: a TMA box a page took 110 to 156 cycles a box, and pages of
//                     16 rows have sixteen a tile (64 sequences of 8192 rows, a token each: 255 us then, 177 now, 6.25 TB/s; pages of 128 rows 218, 173)
// What bounds it.  Many tokens: the exponentials, 770 cycles a tile of 128 x 128 of the special function units', and scores that wait for their buffers, of which
// tensor memory has no more (4096 tokens behind 8192, 32 heads over 8: 371 us, 1230 cycles a tile; 2048 behind 4096: 109.5).  A token a sequence: HBM (16 sequences of 1000 to
// 8192 rows, 32 over 8: 36 us).
// Every wait is bounded: one that runs out raises the CTA's abort flag and GOOSE_ST_TIMEOUT, and every role unwinds.
#include <stddef.h>

#include "goose_internal.cuh"
#include "tcgen05.cuh"
#include "tree_attn_combine.cuh"
#include "weights_work.cuh"

namespace goose {

namespace {

constexpr int kStages = 4, kQStages = 2;
constexpr int kTileBytes = kWeightTile * kHeadDim * 2;       // 32 KB: one K or one Q tile
constexpr int kHalfBytes = kWeightTile * 128;                // 16 KB: 128 rows x 64 bf16 (one swizzle-atom column)
constexpr int kStepBytes = kWeightTile * 32;                 // 4 KB: 128 rows x 16 bf16, without swizzle
constexpr int kHeaderBytes = 1024;
constexpr int kWeightSmem = 1008 /*alignment slack*/ + (kStages + kQStages) * kTileBytes + (1 + kQStages) * kStepBytes + kHeaderBytes;
// warps: four of the roles below, four a key tile of a run for the exponentials, four for the copies of the key tiles
constexpr int kSumWarp = 4, kCopyWarp = kSumWarp + 4 * kRun, kCopyWarps = 4;
constexpr int kWeightThreads = 32 * (kCopyWarp + kCopyWarps);
constexpr uint32_t kTmemCols = 512;
constexpr float kLog2e = 1.4426950408889634f;
constexpr long long kWaitCycles = 2000000000ll;              // bound of every wait: about one second of SM clock
constexpr int kSegments = 6;

// a segment, as the planner describes it
struct Segment {
    int n, q_first;                                          // Q tiles; 0: the end.  The first of them
    int s, hk, ctx, nn;
    int key0, run;                                           // first key, key tiles
    int whole, slot, c0, parts;                              // the CTA has all of the item; else the place of its sums, and who has the others
};

struct Header {
    Segment seg[kSegments];
    alignas(16) uint32_t counts[kQStages][4];                // which rows of the Q tile count
    unsigned long long k_full[kStages], k_empty[kStages], q_full[kQStages], q_empty[kQStages], lse_full[kQStages], lse_empty[kQStages];
    unsigned long long seg_full[kSegments], seg_empty[kSegments];
    unsigned long long s_full[kRun], s_free[kRun];
    uint32_t tmem_base;
    volatile int abort_flag;
};
static_assert(sizeof(Header) <= kHeaderBytes, "header");
static_assert(kWeightSmem <= 232448, "shared memory of a block");

template <typename Int>
struct WeightArgs {
    WeightWork<Int> wk;
    Pages pages;
    const __nv_bfloat16* k_cache;
    int g, H, nb;                                            // heads of a group, heads, tokens of a box of queries
    float scale_log2, inv_scale;
    const float* lse;
    float* row_weight;
    int64_t ldw;
    float* sums;                                             // [CTA][2][kRun][128]
    int32_t* counters;                                       // [CTA][kRun][4], zero between launches
    int32_t* status;
};

__device__ __forceinline__ bool wait_for(Header* hd, unsigned long long* bar, uint32_t parity, int32_t* status) {
    const int r = mbar_wait_bounded(bar, parity, kWaitCycles, &hd->abort_flag);
    if (r == 2) {
        hd->abort_flag = 1;
        atomicOr(status, GOOSE_ST_TIMEOUT);
    }
    return r == 0;
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
__device__ __forceinline__ bool locate(WeightWork<Int>& wk, WeightCursor<Int>& cu, WeightSeq<Int>& q, Int& from, Int& to, int cta, int lane) {
    Int sum = 0;
    bool several = false;
    for (int s0 = 0; s0 < wk.S; s0 += 32)
        if (s0 + lane < wk.S) {
            const WeightSeq<Int> x = wk.seq(s0 + lane);
            several |= x.n > wk.t;
            sum += x.before(x.items);
        }
    wk.set(warp_sum(sum), __any_sync(0xFFFFFFFFu, several));
    from = wk.start(cta);
    to = wk.start(cta + 1);
    if (from >= to) return false;
    Int begin = 0;
    for (int s0 = 0; s0 < wk.S; s0 += 32) {
        Int own = 0;
        if (s0 + lane < wk.S) {
            const WeightSeq<Int> x = wk.seq(s0 + lane);
            own = wk.Hkv * x.before(x.items);
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

// 2^x of two numbers x <= 0 on the FMA pipe: x = n + f with |f| <= 1/2 (adding 1.5 2^23 + 127 rounds x to n and leaves n + 127 in the low bits),
// a polynomial of degree 5 for 2^f, times 2^n.  Its constant term is 1, the others make the largest relative error as small as it gets (a linear program over 4001 places): 0.9e-7, with
// fp32 coefficients and steps 1.7e-7, as much as the special function unit's.  NaN stays NaN; probabilities are not above 1, so that an
// x beyond 127 is of no consequence as long as its result is as absurd: 2^127.
__device__ __forceinline__ unsigned long long ex2_fma(float2 x) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-126.f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-126.f));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(127.f));
    asm("min.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(127.f));
    auto both = [](float c) { return pack_f32x2(c, c); };
    constexpr float kRound = 12582912.f + 127.f;
    const unsigned long long v = pack_f32x2(x.x, x.y), r = add_f32x2(v, both(kRound)), f = fma_f32x2(add_f32x2(r, both(-kRound)), both(-1.f), v);
    unsigned long long p = both(0.0013264653f);
    for (float c : {0.009671511f, 0.05550734f, 0.24022242f, 0.693147f, 1.f}) p = fma_f32x2(p, f, both(c));
    const float2 n = unpack_f32x2(r);
    return mul_f32x2(p, pack_f32x2(__uint_as_float(__float_as_uint(n.x) << 23), __uint_as_float(__float_as_uint(n.y) << 23)));
}

// Sums over 32 columns of exp2(score * scale); kMasked: over those that count.  Of whole tiles every fourth pair's exponentials come from the FMA pipe: the
// special function unit has 16 a cycle (none of them, one in eight, one in four, one in three, 4096 tokens behind 8192, 32 heads over 8: 412, 380, 381, 387 us on one and the same device;
// with a polynomial of degree 4, whose error was 2.6e-6, 1 % less)
template <bool kMasked>
__device__ __forceinline__ void add_columns(const uint32_t (&v)[32], unsigned long long scale2, uint32_t counts, unsigned long long (&part)[2]) {
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
        const float2 x = unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), scale2));
        auto one = [&](int b, float z) { return !kMasked || (counts >> b & 1) ? ex2(z) : 0.f; };
        part[c >> 1 & 1] = add_f32x2(part[c >> 1 & 1], !kMasked && (c & 7) == 6 ? ex2_fma(x) : pack_f32x2(one(c, x.x), one(c + 1, x.y)));
    }
}

// matrix descriptor of 16 K-major columns without swizzle: 8 rows x 16 bytes together, the other 16 bytes of the rows 128 further, the next 8 rows 256
__device__ __forceinline__ uint64_t step_desc(uint32_t addr) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(((addr >> 4) & 0x3FFF) | ((128u >> 4) << 16)), "r"((256u >> 4) | (1u << 14)));
    return d;
}
// M = 128 keys, N = n query rows (a multiple of 16), both K-major
__device__ __forceinline__ uint32_t scores_desc(int n) { return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24); }

template <typename Int>
__global__ void __launch_bounds__(kWeightThreads, 1)
kv_weights_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ WeightArgs<Int> a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* k_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* q_smem = k_smem + kStages * kTileBytes;
    unsigned char* step_smem = q_smem + kQStages * kTileBytes;   // ones, then a Q tile's log-sum-exps each
    Header* hd = reinterpret_cast<Header*>(step_smem + (1 + kQStages) * kStepBytes);
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(&hd->k_full[i], 32 * kCopyWarps); mbar_init(&hd->k_empty[i], 1); }
        for (int i = 0; i < kQStages; ++i) { mbar_init(&hd->q_full[i], 1); mbar_init(&hd->q_empty[i], 1); mbar_init(&hd->lse_full[i], 1); mbar_init(&hd->lse_empty[i], 4 * kRun); }
        for (int i = 0; i < kSegments; ++i) { mbar_init(&hd->seg_full[i], 1); mbar_init(&hd->seg_empty[i], 3 + 4 * kRun + kCopyWarps); }
        for (int u = 0; u < kRun; ++u) { mbar_init(&hd->s_full[u], 1); mbar_init(&hd->s_free[u], 4); }
        hd->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&tmap_q);
    }
    for (int i = threadIdx.x; i < (1 + kQStages) * kStepBytes / 16; i += kWeightThreads) {   // of 16 bytes: 8 rows' first halves, their second ones, ...
        const bool one = i < kStepBytes / 16 && !(i >> 3 & 1);
        reinterpret_cast<uint4*>(step_smem)[i] = one ? make_uint4(0x3F803F80u, 0x00003F80u, 0u, 0u) : make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async();
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
    auto all = [](bool x) { return __all_sync(0xFFFFFFFFu, x) != 0; };

    if (warp < 4) {
        if (warp == 2) {
            // =============================================================== planner
            WeightWork<Int> wk = a.wk;
            if (blockIdx.x == 0)
                for (int s = lane; s < wk.S; s += 32) {
                    const int flaw = (nodes_bad(wk.n_new, s, wk.B) ? GOOSE_ST_BAD_NODES : 0) | (wk.seq(s).bad ? GOOSE_ST_BAD_ROWS : 0);
                    if (flaw) atomicOr(&a.status[s], flaw);
                }
            WeightCursor<Int> cu{};
            WeightSeq<Int> q{};
            Int from, to;
            bool live = locate(wk, cu, q, from, to, blockIdx.x, lane);
            auto advance = [&]() {
                if (cu.next(wk, q)) return;
                do {
                    if (++cu.s < wk.S) q = wk.seq(cu.s);
                } while (cu.s < wk.S && q.items == 0);
                cu.hk = cu.k = 0;
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
                        sg->q_first = q.first(cu.k) + cu.t0;
                        sg->s = cu.s; sg->hk = cu.hk; sg->ctx = q.ctx; sg->nn = q.n;
                        sg->key0 = cu.k * q.span();
                        sg->run = min(kRun, (q.ctx + q.n - sg->key0 + kWeightTile - 1) / kWeightTile);
                        sg->whole = cu.c0 == cu.c1; sg->slot = 2 * blockIdx.x + (cu.t0 == 0); sg->c0 = cu.c0; sg->parts = cu.c1 - cu.c0 + 1;
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&hd->seg_full[ring.at]);
                if (!any) break;
                ring.next(kSegments);
                advance();
            }
        } else if (warp == 0) {
            // =============================================================== Q tiles (the warp runs converged)
            const bool leader = elect_leader();
            uint32_t loads = 0;
            Ring qs{0, 0}, ring{0, 0};
            bool ok = true;
            while (ok) {
                ok = all(wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status));
                if (!ok) break;
                const Segment sg = hd->seg[ring.at];
                __syncwarp();
                if (leader) mbar_arrive(&hd->seg_empty[ring.at]);
                ring.next(kSegments);
                if (sg.n == 0) break;
                for (int i = 0; i < sg.n; ++i) {
                    ok = all(wait_for(hd, &hd->q_empty[qs.at], qs.phase ^ 1, a.status));
                    if (!ok) break;
                    if (leader) {
                        const int token = sg.s * a.wk.B + (sg.q_first + i) * a.wk.t;
                        mbar_expect_tx(&hd->q_full[qs.at], (uint32_t)(a.nb * a.g) * 256u);
                        tma_load_4d(q_smem + qs.at * kTileBytes, &tmap_q, &hd->q_full[qs.at], 0, 0, sg.hk, token);
                        tma_load_4d(q_smem + qs.at * kTileBytes + kHalfBytes, &tmap_q, &hd->q_full[qs.at], 64, 0, sg.hk, token);
                    }
                    __syncwarp();
                    ++loads;
                    qs.next(kQStages);
                }
            }
            // the products' arrivals have landed, too, before the CTA ends
            for (int i = 0; i < kQStages && ok; ++i, qs.next(kQStages)) ok = all(wait_for(hd, &hd->q_empty[qs.at], qs.phase ^ 1, a.status));
            if (!ok)                                             // copies still in flight land before the CTA ends
                for (uint32_t i = 0; i < kQStages; ++i)
                    if (loads > i) drain(&hd->q_full[i], ((loads - 1 - i) / kQStages) & 1);
        } else if (warp == 1) {
            // =============================================================== MMA issuer
            const bool leader = elect_leader();                  // the warp runs converged, this lane acts
            const uint32_t q_addr = smem_u32(q_smem), k_addr = smem_u32(k_smem), step_addr = smem_u32(step_smem);
            uint32_t k_tile = 0, used = 0;                       // K tiles in front of this segment; a bit a score buffer: its parity
            Ring qs{0, 0}, ring{0, 0};
            bool ok = true;
            while (ok) {
                ok = wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status);
                if (!ok) break;
                const Segment* sg = &hd->seg[ring.at];
                const int n = __shfl_sync(0xFFFFFFFFu, sg->n, 0), run = __shfl_sync(0xFFFFFFFFu, sg->run, 0);
                const int q_first = __shfl_sync(0xFFFFFFFFu, sg->q_first, 0), nn = __shfl_sync(0xFFFFFFFFu, sg->nn, 0);
                __syncwarp();
                if (leader) mbar_arrive(&hd->seg_empty[ring.at]);
                ring.next(kSegments);
                if (n == 0) break;
                for (int i = 0; i < n && ok; ++i) {
                    ok = wait_for(hd, &hd->q_full[qs.at], qs.phase, a.status) && wait_for(hd, &hd->lse_full[qs.at], qs.phase, a.status);
                    if (!ok) break;
                    const int rows = min(nn - (q_first + i) * a.wk.t, a.wk.t) * a.g;
                    const uint32_t idesc = scores_desc((rows + 15) & ~15);
                    const uint32_t q_lo = smem_desc_lo(q_addr + qs.at * kTileBytes, 16);
                    for (int u = 0; u < run; ++u) {
                        const uint32_t load = k_tile + u, at = load % kStages;
                        if (i == 0 && !(ok = wait_for(hd, &hd->k_full[at], load / kStages & 1, a.status))) break;
                        if (!(ok = wait_for(hd, &hd->s_free[u], (used >> u & 1) ^ 1, a.status))) break;
                        used ^= 1u << u;
                        fence_proxy_async();                     // (the copies of the keys)
                        tc_fence_after();
                        const uint32_t k_lo = smem_desc_lo(k_addr + at * kTileBytes, 16);
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk) {         // 16 of the 128 head dims per instruction
                            const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
                            umma_f16_by(leader, tmem + u * 128, smem_desc(k_lo + off), smem_desc(q_lo + off), idesc, kk > 0 ? 1u : 0u);
                        }
                        umma_f16_by(leader, tmem + u * 128, step_desc(step_addr), step_desc(step_addr + (1 + qs.at) * kStepBytes), idesc, 1u);
                        umma_commit_by(leader, &hd->s_full[u]);
                        if (i == n - 1) umma_commit_by(leader, &hd->k_empty[at]);
                    }
                    if (!ok) break;
                    umma_commit_by(leader, &hd->q_empty[qs.at]);
                    qs.next(kQStages);
                }
                k_tile += run;
            }
        } else if (warp == 3) {
            // =============================================================== log-sum-exps
            Ring qs{0, 0}, ring{0, 0};
            bool ok = true;
            while (ok) {
                ok = all(wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status));
                if (!ok) break;
                const Segment sg = hd->seg[ring.at];
                __syncwarp();
                if (lane == 0) mbar_arrive(&hd->seg_empty[ring.at]);
                ring.next(kSegments);
                if (sg.n == 0) break;
                for (int i = 0; i < sg.n; ++i) {
                    const int t0 = (sg.q_first + i) * a.wk.t, rows = min(sg.nn - t0, a.wk.t) * a.g;
                    const float* lse = a.lse + ((size_t)sg.s * a.wk.B + t0) * a.H + sg.hk * a.g;
                    float x[4];
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const int r = 32 * w + lane, token = r / a.g;
                        x[w] = r < rows ? lse[(size_t)token * a.H + (r - token * a.g)] : -INFINITY;
                        if (__float_as_uint(x[w]) == __float_as_uint(kNoLse)) x[w] = -INFINITY;
                    }
                    ok = all(wait_for(hd, &hd->lse_empty[qs.at], qs.phase ^ 1, a.status));
                    if (!ok) break;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t word = __ballot_sync(0xFFFFFFFFu, x[w] != -INFINITY);   // (NaN counts)
                        const float v = x[w] == -INFINITY ? 0.f : -a.inv_scale * x[w];
                        const __nv_bfloat16 high = __float2bfloat16_rn(v);
                        const float left = __hisinf(high) ? 0.f : v - __bfloat162float(high);   // (the largest fp32 round to infinity)
                        const __nv_bfloat16 mid = __float2bfloat16_rn(left), low = __float2bfloat16_rn(left - __bfloat162float(mid));
                        const int r = 32 * w + lane;
                        *reinterpret_cast<uint4*>(step_smem + (1 + qs.at) * kStepBytes + (r >> 3) * 256 + (r & 7) * 16) =
                            make_uint4((uint32_t)__bfloat16_as_ushort(high) | (uint32_t)__bfloat16_as_ushort(mid) << 16, __bfloat16_as_ushort(low), 0u, 0u);
                        if (lane == 0) hd->counts[qs.at][w] = word;
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&hd->lse_full[qs.at]);
                    qs.next(kQStages);
                }
            }
        }
    } else if (warp >= kCopyWarp) {
        // =============================================================== K tiles: 32 keys of a tile a warp
        const int part = warp - kCopyWarp;
        const uint32_t k_addr = smem_u32(k_smem) + 4096 * part;
        const unsigned long long pol_once = l2_policy_evict_first(), pol_again = l2_policy_evict_last();
        // 16 bytes of a row a lane, two rows at a time; where they go in a tile of swizzled rows, for each of four such pairs of rows
        const size_t row_bytes = (size_t)a.wk.Hkv * kHeadDim * 2;
        uint32_t place[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 2 * i + (lane >> 4);
            place[i] = (lane >> 3 & 1) * kHalfBytes + r * 128 + (((lane & 7) ^ r) << 4);
        }
        Ring ks{0, 0}, ring{0, 0};
        bool ok = true;
        Segment next{};
        int next_row = -1;
        // The next segment, and the cache rows where 16 of its keys lie (a page has as many at least), lane 2 u + q: the q-th of this warp's in tile u; -1 where
        // there are none.  No page behind the sequence's last row is looked up.
        auto take = [&]() {
            ok = all(wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status));
            if (!ok) return;
            next = hd->seg[ring.at];
            __syncwarp();
            if (lane == 0) mbar_arrive(&hd->seg_empty[ring.at]);
            ring.next(kSegments);
            const int u = lane >> 1, j = next.key0 + u * kWeightTile + 32 * part + 16 * (lane & 1);
            next_row = -1;
            if (next.n > 0 && u < next.run && j < next.ctx + next.nn) next_row = (int)a.pages.row(next.s, j);
        };
        take();
        while (ok && next.n > 0) {
            const Segment sg = next;
            const int rows = next_row;
            // the one behind it now, if the planner has it, so that its look-ups run beside these copies
            const bool early = all(mbar_try_wait(&hd->seg_full[ring.at], ring.phase));
            if (early) take();
            const unsigned long long pol = sg.nn > a.wk.t ? pol_again : pol_once;
            const char* from0 = reinterpret_cast<const char*>(a.k_cache) + (size_t)sg.hk * kHeadDim * 2 + (lane >> 4) * row_bytes + (lane & 15) * 16;
            for (int u = 0; u < sg.run && ok; ++u) {
                ok = all(wait_for(hd, &hd->k_empty[ks.at], ks.phase ^ 1, a.status));
                if (!ok) break;
                const uint32_t dst = k_addr + ks.at * kTileBytes;
                const int keys = sg.ctx + sg.nn - sg.key0 - u * kWeightTile - 32 * part - (lane >> 4);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int row = __shfl_sync(0xFFFFFFFFu, rows, 2 * u + q);
                    const char* from = from0 + (size_t)max(row, 0) * row_bytes;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        cp_async_16(dst + 2048 * q + 1024 * (i >> 2) + place[i & 3], from + 2 * i * row_bytes, row >= 0 && 16 * q + 2 * i < keys, pol);
                }
                cp_async_arrive(&hd->k_full[ks.at]);
                ks.next(kStages);
            }
            if (ok && !early) take();
        }
        for (int i = 0; i < kStages && ok; ++i, ks.next(kStages)) ok = all(wait_for(hd, &hd->k_empty[ks.at], ks.phase ^ 1, a.status));
        if (!ok) cp_async_wait_all();
    } else {
        // =============================================================== exponentials and sums
        const int u = (warp - kSumWarp) >> 2, wq = warp & 3; // key tile of a run
        const int row = 32 * wq + lane;                      // TMEM lane == key of the tile
        const uint32_t from = tmem + u * 128 + ((uint32_t)(32 * wq) << 16);
        const unsigned long long scale2 = pack_f32x2(a.scale_log2, a.scale_log2);
        uint32_t used = 0;                                   // the score buffer's parity
        Ring qs{0, 0}, ring{0, 0};
        bool ok = true;
        while (ok) {
            ok = all(wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status));
            if (!ok) break;
            const Segment& sg = hd->seg[ring.at];
            const int n = sg.n;
            if (n == 0) break;
            const bool live = u < sg.run;
            const int ahead = sg.key0 + u * kWeightTile - sg.ctx, g = a.g;   // tokens of the chunk in front of the first that sees the tile's first key
            const bool mine = live && ahead + row < sg.nn;
            const int page = mine ? a.pages.table[sg.s * a.pages.ldt + ((ahead + sg.ctx + row) >> a.pages.size_log2)] : -1;   // (looked at when the sum is there)
            float sum = 0.f;
            int t0 = sg.q_first * a.wk.t, left = sg.nn - t0;
            for (int i = 0; i < n; ++i, t0 += a.wk.t, left -= a.wk.t) {
                ok = all(wait_for(hd, &hd->lse_full[qs.at], qs.phase, a.status));
                if (!ok) break;
                if (live) {
                    ok = all(wait_for(hd, &hd->s_full[u], used, a.status));
                    if (!ok) break;
                    used ^= 1;
                    tc_fence_after();
                    const int rows = min(left, a.wk.t) * g;
                    const uint32_t* counts = hd->counts[qs.at];
                    const bool masked = (counts[0] & counts[1] & counts[2] & counts[3]) != 0xFFFFFFFFu || ahead + kWeightTile - 1 > t0;
                    const int first = max(ahead + row - t0, 0) * g;  // columns in front of it are tokens in front of the key
                    unsigned long long part[2] = {0, 0};
#pragma unroll 1
                    for (int w = 0; 32 * w < rows; ++w) {
                        uint32_t v[32];
                        TMEM_LD32(from + 32 * w, v, 0);
                        tmem_wait_ld();
                        if (32 * w + 32 >= rows) {                   // all scores are in registers, or have been
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&hd->s_free[u]);
                        }
                        if (!masked) {
                            add_columns<false>(v, scale2, 0, part);
                        } else {
                            const int out = first - 32 * w;
                            add_columns<true>(v, scale2, counts[w] & (out <= 0 ? 0xFFFFFFFFu : out >= 32 ? 0u : 0xFFFFFFFFu << out), part);
                        }
                    }
                    const float2 s2 = unpack_f32x2(add_f32x2(part[0], part[1]));
                    sum += s2.x + s2.y;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&hd->lse_empty[qs.at]);
                qs.next(kQStages);
            }
            if (!ok) break;
            if (live) {
                const bool there = page >= 0 && page < a.pages.n;
                if (mine && !there) atomicOr(&a.status[sg.s], GOOSE_ST_BAD_ROWS);
                float* weight = a.row_weight + ((size_t)sg.s * a.wk.Hkv + sg.hk) * a.ldw + sg.key0 + u * kWeightTile + row;
                bool last = true;
                if (!sg.whole) {
                    a.sums[((size_t)sg.slot * kRun + u) * kWeightTile + row] = sum;
                    __threadfence();
                    __syncwarp();
                    int32_t* counter = a.counters + (sg.c0 * kRun + u) * 4 + wq;
                    int came = 0;
                    if (lane == 0) came = atomicAdd(counter, 1);
                    last = __shfl_sync(0xFFFFFFFFu, came, 0) == sg.parts - 1;
                    if (last) {
                        __threadfence();
                        if (lane == 0) *counter = 0;
                        sum = 0.f;
                        for (int k = 0; k < sg.parts; ++k) sum += __ldcg(&a.sums[((size_t)(2 * (sg.c0 + k) + (k == 0)) * kRun + u) * kWeightTile + row]);
                    }
                }
                // (a reduction: nobody waits for what the row had.  One a row and call: the order of the calls is the order of the sums)
                if (last && there) atomicAdd(weight, sum);
            }
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
static cudaError_t launch_as(goose_ctx* c, const KvWeights& x, cudaStream_t st) {
    WeightArgs<Int> a{};
    a.g = x.H / x.Hkv; a.H = x.H;
    a.wk.ctx_len = x.ctx_len; a.wk.n_new = x.n_new; a.wk.S = x.S; a.wk.B = x.B; a.wk.Hkv = x.Hkv; a.wk.G = c->num_sms;
    a.wk.t = kWeightTile / a.g; a.wk.room = (int)x.pages.room(x.ldw);
    a.pages = x.pages;
    a.nb = a.wk.t < x.B ? a.wk.t : x.B;
    a.k_cache = x.k_cache;
    a.scale_log2 = x.scale * kLog2e; a.inv_scale = 1.f / x.scale;
    a.lse = x.lse; a.row_weight = x.row_weight; a.ldw = x.ldw;
    a.sums = c->weight_sums; a.counters = c->weight_counters; a.status = c->status;
    CUtensorMap mq;
    if (!make_q_map(c->encode_tiled, &mq, x.q, (int64_t)x.S * x.B, x.Hkv, a.g, a.nb)) return cudaErrorInvalidValue;
    cudaError_t e = launch_pdl(kv_weights_kernel<Int>, dim3(c->num_sms), dim3(kWeightThreads), kWeightSmem, st, mq, a);
    c->launches++;
    return e;
}

cudaError_t launch_kv_weights(goose_ctx* c, const KvWeights& x, cudaStream_t st) {
    if (!c->encode_tiled) return cudaErrorNotSupported;
    if (x.S == 0) return cudaSuccess;
    const bool small = WeightWork<int>::most(x.S, x.B, x.Hkv, kWeightTile / (x.H / x.Hkv), (int)x.pages.room(x.ldw)) < kShortWeightPlaces;
    return small ? launch_as<int>(c, x, st) : launch_as<long long>(c, x, st);
}

cudaError_t init_weights_kernels() {
    cudaError_t e = cudaFuncSetAttribute(kv_weights_kernel<int>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWeightSmem);
    return e == cudaSuccess ? cudaFuncSetAttribute(kv_weights_kernel<long long>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWeightSmem) : e;
}

}  // namespace goose
