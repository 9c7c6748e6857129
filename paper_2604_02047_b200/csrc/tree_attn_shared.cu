// Tree attention of a batch whose sequences share a long prefix: the shared rows are streamed once for 256 query rows of all
// sequences, every sequence's own rows (its prefix and its tree) once for its own queries, and the two are merged by their
// maxima and sums:  out = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p,  where O_p = sum_j 2^(x_j - m_p) v_j and l_p = sum_j 2^(x_j - m_p) over
// the keys of part p, x_j the scaled scores (base 2), M the largest m_p.
//
// Main kernel: persistent, one CTA an SM, tcgen05 with TMEM accumulators, TMA loads, mbarrier pipeline; work list and lanes:
// shared_work.cuh.  A sequence's own rows are never met by another sequence's queries, not even masked: what they hold (infinities, NaN)
// stays in that sequence.  Roles (384 threads):
//   warp 0, lane 0    TMA producer: the queries of a segment, then K and V tiles into a ring of 32 KB stages
//   warps 1, 3        MMA issuers of lane 0 and of lane 1: S = Q K^T, O += P V; while one lane's softmax runs, the tensor cores have the
//                     other's products
//   warp 2            planner: walks the work list ahead of the others and puts the segments' descriptions into a ring, parents included
//   warps 4..7, 8..11 softmax of lane 0 and of lane 1: one query row a thread: maximum, exponentials, P (bf16) over S in tensor
//                     memory, lazy rescaling of O, at the segment's end the partial result into the workspace.
// Tensor memory: S of both lanes in columns 0..255, O of both in 256..511.
// Why so: the shared rows are read once for 256 query rows, which makes them work for the tensor cores instead of HBM; two lanes, since a row's
// exponentials (16 a cycle and SM: 1060 cycles a tile) and a tile's products (1024 cycles) follow one another within a lane; tiles of 128 keys
// and a row a thread, so that maximum and sum need no exchange.
// What bounds it.  Many query rows: a pair of tiles takes 3150 to 3400 cycles, of which the exponentials are 2120, the products 2048 (16
// sequences of 64 nodes, 32 heads over 8, under 8192 rows: 151 us, 1.05 PFLOP/s; under the power cap 175).  Few: HBM (64 sequences, a token each, 32 over 8,
// under 16k rows: 106 us, 4.7 TB/s, 5.7 without merge; 121 under the power cap).  Small calls: planner 1.8 us, first tile 1.6, epilogue 1.3, merge 3 (4 sequences, a
// token each, under 512 rows: 11.8 to 12.2 us).  A change of item takes 3 us where the item has a tile or two (26 x 52 heads, 32 nodes, 5423 rows: 207 us).
// Every wait is bounded: one that runs out raises the CTA's abort flag and GOOSE_ST_TIMEOUT, and every role unwinds.
#include <stddef.h>

#include "goose_internal.cuh"
#include "shared_work.cuh"
#include "tcgen05.cuh"
#include "tree_attn_combine.cuh"

namespace goose {

namespace {

constexpr int kStages = 5;
constexpr int kStageBytes = kSharedTile * kHeadDim * 2;      // 32 KB: one K or one V tile
constexpr int kHalfBytes = kSharedTile * 128;                // 16 KB: 128 rows x 64 bf16 (one swizzle-atom column)
constexpr int kQBytes = 2 * kHalfBytes;
constexpr int kHeaderBytes = 2048;
constexpr int kSharedSmem = 1008 /*alignment slack*/ + 2 * kQBytes + kStages * kStageBytes + kHeaderBytes;
constexpr int kSharedThreads = 384;
// registers: 168 a thread at launch; the warps of the loads and products give 112 each to the others (56 + 2 x 224 = 3 x 168)
constexpr int kRegsFew = 56, kRegsMany = 224;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleThreshold = 8.0f;                    // rescale O only when the running max grew by > 2^8
constexpr long long kWaitCycles = 2000000000ll;              // bound of every wait: about one second of SM clock

// Partial result of an M tile: O in three bytes an element, fp32 without its last byte: sign, exponent and 16 bits of significand (the output has 8)
// of every element by itself, whatever its row's or its column's others are, infinities and NaN among them.  A row is 25 words of 16 bytes: the
// two upper bytes of 8 columns in each of 16, the third ones of 16 columns in each of 8, and (m, l) in fp32, the maximum that the
// exponentials are relative to (base 2) and their sum.  l < 0: a sequence that cannot be computed (no tree, rows outside the cache).
// (Half precision times a power of two of the row's largest element, two bytes, lost the elements below 2^-25 of it.  What the third byte
// costs: 16 x 64 nodes, 32 heads over 8, under 8192 rows 148.6 -> 151.3 us, 64 sequences of a token 107.6 -> 108.2, one sequence of 4 nodes, 16 heads over 2,
// under 30k rows 33 -> 37; 26 x 52 heads, 32 nodes, 128 rows 56.9 -> 53.4, 42 x 52 heads, a token each, 174 -> 168.)
// Words of neighbouring rows lie next to one another, a row's words 128 apart (see SharedWork::place(): with 128 rows for every M tile, however few
// it can have, 64 sequences of a token, 40 heads, had 300 MB instead of 25; a distance of the rows that there can be instead of 128 made the
// addresses arithmetic: 15 x 52 heads, 80 nodes 103.3 -> 106.8 us).
constexpr int kPartThird = 16, kPartSums = 24;               // words of a row in front of the third bytes, of (m, l)
// four elements' words: the upper halves of two, the third bytes of four, and back (the last byte comes back as a copy of the third: within 2^-15)
__device__ __forceinline__ uint32_t upper_halves(uint32_t x0, uint32_t x1) { return __byte_perm(x0, x1, 0x7632); }
__device__ __forceinline__ uint32_t third_bytes(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
    return __byte_perm(__byte_perm(x0, x1, 0x0051), __byte_perm(x2, x3, 0x0051), 0x5410);
}
template <int kAt>                                           // element 0..3 of the four
__device__ __forceinline__ float part_element(uint32_t halves, uint32_t thirds) {
    constexpr uint32_t third = 4 + kAt, upper = kAt & 1 ? 0x3200 : 0x1000;
    return __uint_as_float(__byte_perm(halves, thirds, upper | third << 4 | third));
}

// a segment, as the planner describes it
struct Segment {
    int n;                                                   // key tiles; 0: the end
    int t_first;
    int ctx, n_keys;                                         // keys in front of the tree, and all
    int single, own;                                         // one M tile; a sequence's own rows
    int hk, token;                                           // key/value head, first token of the first M tile
    int row;                                                 // cache row of the first key tile
    uint32_t part[2];                                        // places in the workspace: of the pair's M tiles; of a single one's even and odd key tiles
    int rows[2];                                             // query rows of the M tiles
    int node;                                                // tree node of the first M tile's first row
    int bad;
    int pad;
};
constexpr int kSegments = 6;

struct Header {
    Segment seg[kSegments];
    signed char par[kSegments][kMaxB];                       // parent[] of the segment's sequence
    // Full: of the key tiles of single M tiles lane by lane (0, 1), of pairs (2).  A parity tells two phases apart, not three: nobody may wait
    // for a phase of a barrier whose phases it has not all followed, and a lane does not follow the tiles of the other one.
    unsigned long long kv_full[3][kStages];
    unsigned long long kv_empty[kStages];
    unsigned long long seg_full[kSegments], seg_empty[kSegments];
    // The two places of query tiles.  A pair has both, each lane its own; single M tiles have them in turn, so that the next one's queries come
    // while the segment in front still uses the other.  With barriers of their own nobody waits on a phase that it has not followed.
    unsigned long long pair_full[2], pair_empty[2], single_full[2], single_empty[2];
    unsigned long long s_full[2], v_there[2], o_full[2], o_free[2];
    unsigned long long p_ready[2][2];                        // of a lane, P of either half of a tile's keys
    uint32_t tmem_base;
    volatile int abort_flag;
};
static_assert(sizeof(Header) <= kHeaderBytes, "header");
static_assert(kSharedSmem <= 232448, "shared memory of a block");

struct SharedArgs {
    const int64_t* row_off;
    const int32_t* parent;
    SharedWork wk;
    int g;                                                   // query heads per key/value head
    int shared_nb, own_nb;                                   // tokens of an M tile: of the batch, of one sequence
    int shared_row, shared_len;
    float scale_log2;
    uint4* parts;
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

// the list's length and a place in it, by a whole warp (lane = sequence)
__device__ __forceinline__ void locate(SharedWork& wk, SharedCursor& cu, long long& w_end, int cta, int lane) {
    const int mine = lane < wk.S ? wk.tiles(lane) : 0;
    long long sum = __reduce_add_sync(0xFFFFFFFFu, (uint32_t)mine);
    int live = __popc(__ballot_sync(0xFFFFFFFFu, mine > 0));
    for (int s0 = 32; s0 < wk.S; s0 += 32) {
        const int more = s0 + lane < wk.S ? wk.tiles(s0 + lane) : 0;
        sum += __reduce_add_sync(0xFFFFFFFFu, (uint32_t)more);
        live += __popc(__ballot_sync(0xFFFFFFFFu, more > 0));
    }
    wk.set(sum, live);
    const long long w0 = wk.start(cta);
    w_end = wk.start(cta + 1);
    cu.w = w0; cu.s = -1; cu.i = 0; cu.t = 0; cu.T = wk.shared_tiles;
    if (w0 >= w_end) return;
    if (w0 < wk.shared_total) { cu.enter(wk, w0); return; }
    long long rem = w0 - wk.shared_total;
    const long long per = (long long)wk.Hkv * wk.own_pairs();
    for (int s0 = 0; s0 < wk.S; s0 += 32) {
        const int T = s0 == 0 ? mine : s0 + lane < wk.S ? wk.tiles(s0 + lane) : 0;
        const uint32_t own = (uint32_t)wk.width(s0, T);
        uint32_t upto = own;                                 // (32 widths of 5 * 2^24 + 16 at most: below 2^32)
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += u;
        }
        const uint32_t here = __ballot_sync(0xFFFFFFFFu, per * upto > rem);
        if (here) {
            const int l = __ffs(here) - 1;
            cu.s = s0 + l;
            cu.T = __shfl_sync(0xFFFFFFFFu, T, l);
            cu.enter(wk, rem - per * __shfl_sync(0xFFFFFFFFu, upto - own, l));
            return;
        }
        rem -= per * __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
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

__global__ void __launch_bounds__(kSharedThreads, 1)
tree_attn_shared_kernel(const __grid_constant__ CUtensorMap tmap_q_shared, const __grid_constant__ CUtensorMap tmap_q_own,
                        const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                        const __grid_constant__ SharedArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* q_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* kv_smem = q_smem + 2 * kQBytes;
    Header* hd = reinterpret_cast<Header*>(kv_smem + kStages * kStageBytes);
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { for (int u = 0; u < 3; ++u) mbar_init(&hd->kv_full[u][i], 1); mbar_init(&hd->kv_empty[i], 2); }
        for (int i = 0; i < kSegments; ++i) { mbar_init(&hd->seg_full[i], 1); mbar_init(&hd->seg_empty[i], 3 + 8); }
        for (int l = 0; l < 2; ++l) {
            mbar_init(&hd->pair_full[l], 1); mbar_init(&hd->pair_empty[l], 1); mbar_init(&hd->single_full[l], 1); mbar_init(&hd->single_empty[l], 2);
            mbar_init(&hd->s_full[l], 1); mbar_init(&hd->v_there[l], 1); mbar_init(&hd->p_ready[l][0], 4); mbar_init(&hd->p_ready[l][1], 4); mbar_init(&hd->o_full[l], 1); mbar_init(&hd->o_free[l], 4);
        }
        hd->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_tmap(&tmap_q_shared); prefetch_tmap(&tmap_q_own); prefetch_tmap(&tmap_k); prefetch_tmap(&tmap_v);
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
            SharedWork wk = a.wk;
            if (wk.n_nodes && blockIdx.x == 0)
                for (int s = lane; s < wk.S; s += 32)
                    if (nodes_bad(wk.n_nodes, s, wk.B)) atomicOr(&a.status[s], GOOSE_ST_BAD_NODES);
            SharedCursor cu;
            long long w_end;
            locate(wk, cu, w_end, blockIdx.x, lane);
            // of the sequence that the items are of (a head after the other): asked for together, kept until the next one's
            int of = -1, nn = 0, ctx = 0, par[kMaxB / 32];
            int64_t row0 = 0;
            bool bad = false;
            Ring ring{0, 0};
            for (;;) {
                if (!wait_for(hd, &hd->seg_empty[ring.at], ring.phase ^ 1, a.status)) break;
                const bool any = cu.w < w_end, shared = cu.s < 0;
                Segment* sg = &hd->seg[ring.at];
                if (any) {
                    const int s = cu.s, n = cu.run(wk, w_end);
                    const int pairs = shared ? wk.shared_pairs() : wk.own_pairs(), n_m = shared ? wk.shared_m : wk.own_m;
                    const int nb = shared ? a.shared_nb : a.own_nb;
                    const int hk = cu.i / pairs, m = 2 * (cu.i - hk * pairs);
                    if (shared) {
                        ctx = a.shared_len; row0 = a.shared_row;
                    } else {
                        if (s != of) {
#pragma unroll
                            for (int j = 0; j < kMaxB / 32; ++j) par[j] = lane + 32 * j < wk.B ? a.parent[(size_t)s * wk.B + lane + 32 * j] : 0;
                            row0 = a.row_off[s];
                            const int given = wk.ctx_len[s];
                            nn = nodes_of(wk.n_nodes, s, wk.B);
                            ctx = wk.prefix(given);
                            of = s;
                            // a sequence of a parent[] that is no tree, or whose rows leave the cache: every part of it says so
                            bool no_tree = false;
#pragma unroll
                            for (int j = 0; j < kMaxB / 32; ++j) {
                                const int i = lane + 32 * j;
                                no_tree |= i < nn && (i == 0 ? par[j] != -1 : (par[j] < 0 || par[j] >= i));
                            }
                            no_tree = __any_sync(0xFFFFFFFFu, no_tree);
                            const bool bad_rows = rows_outside(row0, given, nn, wk.kv_rows);
                            bad = no_tree || bad_rows;
                            if (bad && lane == 0) atomicOr(&a.status[s], (no_tree ? GOOSE_ST_BAD_PARENT : 0) | (bad_rows ? GOOSE_ST_BAD_ROWS : 0));
                        }
#pragma unroll
                        for (int j = 0; j < kMaxB / 32; ++j)
                            if (lane + 32 * j < nn) hd->par[ring.at][lane + 32 * j] = (signed char)par[j];
                    }
                    if (lane < 2) sg->part[lane] = wk.place(wk.slot(wk.item(s, cu.i), blockIdx.x, cu.t == 0, cu.t + n == cu.T, lane));
                    if (lane == 0) {
                        sg->n = n; sg->t_first = cu.t; sg->ctx = ctx; sg->n_keys = ctx + nn;
                        sg->single = m + 1 >= n_m; sg->own = !shared; sg->hk = hk;
                        sg->token = (shared ? 0 : s * wk.B) + m * nb;
                        sg->row = (int)((uint64_t)row0 + (uint64_t)cu.t * kSharedTile);
                        const int left = shared ? wk.S * wk.B : nn;
                        sg->rows[0] = max(min(nb, left - m * nb), 0) * a.g;
                        sg->rows[1] = max(min(nb, left - (m + 1) * nb), 0) * a.g;
                        sg->node = m * nb; sg->bad = bad;
                    }
                    cu.skip(wk, n);
                } else if (lane == 0) {
                    sg->n = 0;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&hd->seg_full[ring.at]);
                if (!any) break;
                ring.next(kSegments);
            }
        } else if (warp == 0) {
            // =========================================================== TMA producer
            if (lane == 0) {
                // a sequence's own rows are read by one or two CTAs, the shared ones by many
                const unsigned long long pol_own = l2_policy_evict_first(), pol_shared = l2_policy_evict_last();
                uint32_t pairs = 0, singles = 0, tile0 = 0;  // segments of either kind, tiles in front of this segment
                uint32_t phases = 0, users = 0;              // a bit a kv_full barrier; two bits a stage: who has it, 3: nobody yet
                for (int i = 0; i < kStages; ++i) users |= 3u << 2 * i;
                Ring st{0, 0}, ring{0, 0};
                bool ok = true;
                Segment sg{};
                uint32_t asked = 0;                          // query tiles of the segment that still wait for their place
                auto load_q = [&](int b) {
                    const int nb = sg.own ? a.own_nb : a.shared_nb, m = sg.single ? 0 : b;
                    const CUtensorMap* mq = sg.own ? &tmap_q_own : &tmap_q_shared;
                    unsigned long long* full = sg.single ? &hd->single_full[b] : &hd->pair_full[b];
                    mbar_expect_tx(full, (uint32_t)(nb * a.g) * 256u);
                    tma_load_4d(q_smem + b * kQBytes, mq, full, 0, 0, sg.hk, sg.token + m * nb);
                    tma_load_4d(q_smem + b * kQBytes + kHalfBytes, mq, full, 64, 0, sg.hk, sg.token + m * nb);
                    asked &= ~(1u << b);
                };
                // place b is free when the last pair and the last single M tile that had it are done
                auto pair_parity = [&]() { return (pairs & 1) ^ 1; };
                auto single_parity = [&](int b) { return ((singles + 1 - b) >> 1 & 1) ^ 1; };
                auto load_free_q = [&]() {
                    for (int b = 0; b < 2; ++b)
                        if ((asked >> b & 1) && mbar_done(&hd->pair_empty[b], pair_parity()) && mbar_done(&hd->single_empty[b], single_parity(b)))
                            load_q(b);
                };
                // The key tiles do not wait for the queries' place: a pair's is free only when the products of the segment in front
                // are done, and the ring would run dry meanwhile.
                auto stage_free = [&]() {
                    const long long t0 = clock64();
                    while (asked) {
                        load_free_q();
                        if (mbar_done(&hd->kv_empty[st.at], st.phase ^ 1)) return true;
                        if (hd->abort_flag || clock64() - t0 > kWaitCycles) break;   // (the wait below says so)
                    }
                    return wait_for(hd, &hd->kv_empty[st.at], st.phase ^ 1, a.status);
                };
                while (ok) {
                    for (int b = 0; b < 2 && ok; ++b)        // of the segment in front
                        if (asked >> b & 1) {
                            ok = wait_for(hd, &hd->pair_empty[b], pair_parity(), a.status) && wait_for(hd, &hd->single_empty[b], single_parity(b), a.status);
                            if (ok) load_q(b);
                        }
                    if (ok && sg.n > 0) { if (sg.single) ++singles; else ++pairs; sg.n = 0; }
                    ok = ok && wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status);
                    if (!ok) break;
                    sg = hd->seg[ring.at];
                    mbar_arrive(&hd->seg_empty[ring.at]);
                    ring.next(kSegments);
                    if (sg.n == 0) break;
                    asked = sg.single ? 1u << (singles & 1) : 3u;
                    uint32_t krow = (uint32_t)sg.row;
                    const unsigned long long pol = sg.own ? pol_own : pol_shared;
                    for (int i = 0; i < sg.n && ok; ++i, krow += kSharedTile) {
                        const uint32_t user = sg.single ? (tile0 + i) & 1 : 2;
                        for (int kv = 0; kv < 2 && ok; ++kv) {
                            ok = stage_free();
                            if (!ok) break;
                            unsigned char* dst = kv_smem + st.at * kStageBytes;
                            unsigned long long* full = &hd->kv_full[user][st.at];
                            mbar_expect_tx(full, kStageBytes);
                            const CUtensorMap* mp = kv ? &tmap_v : &tmap_k;
                            tma_load_3d_hint(dst, mp, full, 0, sg.hk, (int)krow, pol);
                            tma_load_3d_hint(dst + kHalfBytes, mp, full, 64, sg.hk, (int)krow, pol);
                            phases ^= 1u << (user * kStages + st.at);
                            users = (users & ~(3u << 2 * st.at)) | user << 2 * st.at;
                            st.next(kStages);
                        }
                    }
                    tile0 += sg.n;
                }
                // The products' arrivals have landed, too, before the CTA ends: those that free stages and queries' places are behind the one
                // that the epilogue waits for.
                for (int i = 0; i < kStages && ok; ++i, st.next(kStages)) ok = wait_for(hd, &hd->kv_empty[st.at], st.phase ^ 1, a.status);
                for (int b = 0; b < 2 && ok; ++b)
                    ok = wait_for(hd, &hd->pair_empty[b], pair_parity(), a.status) && wait_for(hd, &hd->single_empty[b], single_parity(b), a.status);
                if (!ok) {                                   // copies still in flight land before the CTA ends
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
            }
        } else {
            // =========================================================== MMA issuers: warp 1 for lane 0, warp 3 for lane 1
            {
                const bool leader = elect_leader();          // the warp runs converged, this lane acts
                const uint32_t l = warp >> 1;
                const uint32_t q_addr = smem_u32(q_smem), kv_addr = smem_u32(kv_smem);
                const uint32_t s_tmem = tmem + kColS + l * 128, o_tmem = tmem + kColO + l * 128;
                constexpr uint32_t idesc_qk = instr_desc(false), idesc_pv = instr_desc(true);
                uint32_t ops = 0, segs = 0, tile0 = 0;       // products, segments of this lane; tiles of the CTA
                uint32_t pairs = 0, singles = 0;             // segments of the CTA
                Ring ring{0, 0};
                bool ok = true;
                uint32_t phases = 0;                         // a bit a kv_full barrier of this lane and, kStages further, of pairs
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
                    auto release = [&](uint32_t load) {      // every stage has two arrivals
                        umma_commit_by(leader, &hd->kv_empty[load % kStages]);
                        if (single && leader) mbar_arrive(&hd->kv_empty[load % kStages]);
                    };
                    auto scores = [&](uint32_t t) {
                        tc_fence_after();
                        const uint32_t k_lo = smem_desc_lo(kv_addr + (2 * t % kStages) * kStageBytes, 16);
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk) {     // 16 of the 128 head dims per instruction
                            const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
                            umma_f16_by(leader, s_tmem, smem_desc(q_lo + off), smem_desc(k_lo + off), idesc_qk, kk > 0 ? 1u : 0u);
                        }
                        umma_commit_by(leader, &hd->s_full[l]);         // (and with it the product in front of it)
                    };
                    uint32_t t = tile0 + (single ? (tile0 ^ l) & 1 : 0);
                    const bool any = t < end;
                    if (any) {
                        ok = stage_full(2 * t);
                        if (!ok) break;
                        scores(t);
                        release(2 * t);
                    }
                    if (t + step >= end) {                   // the lane's last Q K^T of the segment
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
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsMany));
        // =============================================================== softmax and partial results
        const int l = (warp - 4) >> 2;                       // lane of the segments
        const int row = 32 * (warp & 3) + lane;              // TMEM lane == query row
        const uint32_t s_addr = tmem + kColS + l * 128 + ((uint32_t)(32 * (warp & 3)) << 16);   // O: kColO - kColS further
        const uint32_t base = smem_u32(hd), my_bars = base + 8 * l, abort_at = base + (uint32_t)offsetof(Header, abort_flag);
        constexpr uint32_t kAtFull = offsetof(Header, s_full), kAtDone = offsetof(Header, o_full);
        constexpr uint32_t kAtFree = offsetof(Header, o_free);
        const uint32_t at_ready = base + (uint32_t)offsetof(Header, p_ready) + 16 * l;
        uint32_t ops = 0, segs = 0, tile0 = 0;               // products and segments of this lane; tiles of the CTA in front of this segment
        Ring ring{0, 0};
        bool ok = true;
        uint32_t v[128], anc[4] = {0, 0, 0, 0};
        int anc_of = -1;                                     // first token of the M tile that anc[] is of

        for (;;) {
            ok = wait_for(hd, &hd->seg_full[ring.at], ring.phase, a.status);
            if (!ok) break;
            const Segment& sg = hd->seg[ring.at];
            if (sg.n == 0) break;
            const int step = sg.single ? 2 : 1, t_end = sg.t_first + sg.n;
            const int turn = sg.single ? (tile0 ^ l) & 1 : l;   // a single M tile's key tiles are dealt on where the segment in front ended
            const int rows = sg.rows[sg.single ? 0 : l];
            const bool row_valid = row < rows, warp_has_rows = (row & ~31) < rows;
            const int t_masked = sg.ctx / kSharedTile;       // from here on a tile reaches the tree rows, or the ragged end
            // the row's ancestors, where the segment reaches the tree (while its first scores are on their way); the heads of a sequence have
            // the same
            if (sg.own && t_end > t_masked && anc_of != sg.token + (sg.single ? 0 : l) * a.own_nb) {
                anc_of = sg.token + (sg.single ? 0 : l) * a.own_nb;
                anc[0] = anc[1] = anc[2] = anc[3] = 0;
                int vtx = sg.node + (sg.single ? 0 : l) * a.own_nb + row / a.g;
                for (int up = row_valid && !sg.bad ? 0 : kMaxB; up < kMaxB && vtx >= 0; ++up) {
                    const uint32_t bit = 1u << (vtx & 31);
                    const int wsel = vtx >> 5;
                    anc[0] |= (wsel == 0) ? bit : 0; anc[1] |= (wsel == 1) ? bit : 0;
                    anc[2] |= (wsel == 2) ? bit : 0; anc[3] |= (wsel == 3) ? bit : 0;
                    vtx = hd->par[ring.at][vtx];
                }
            }
            float m_run = -INFINITY, l_run = 0.f;
            bool first = true;
            for (int t = sg.t_first + (sg.single ? turn : 0); t < t_end; t += step) {
                ok = wait_at(my_bars + kAtFull, ops & 1, abort_at, a.status);
                if (!ok) break;
                tc_fence_after();
                // ragged end: V rows past the last key may hold anything -> zeros (by either lane of a tile that both use)
                if (t >= t_masked && (t + 1) * kSharedTile > sg.n_keys) {
                    const uint32_t load = 2 * (tile0 + (t - sg.t_first)) + 1, st = load % kStages;
                    ok = wait_for(hd, &hd->v_there[l], ops & 1, a.status);
                    if (!ok) break;
                    const int first_off = max(sg.n_keys - t * kSharedTile, 0) * 128;
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
                        const int pc = sg.ctx - t * kSharedTile;   // tile column of the first key behind the prefix
                        // visibility of the tile's 128 keys as one mask: the prefix keys, and the row's ancestors from where the tree rows start
                        const unsigned __int128 a128 =
                            ((unsigned __int128)(((unsigned long long)anc[3] << 32) | anc[2]) << 64) |
                            (unsigned __int128)(((unsigned long long)anc[1] << 32) | anc[0]);
                        unsigned __int128 vm;
                        if (pc > 0) vm = (((unsigned __int128)1 << pc) - 1) | (a128 << pc);
                        else if (pc > -128) vm = a128 >> (-pc);
                        else vm = 0;
                        const uint32_t vw[4] = {(uint32_t)vm, (uint32_t)(vm >> 32), (uint32_t)(vm >> 64), (uint32_t)(vm >> 96)};
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
            if (!first) {
                // ---------------- partial result of this lane
                ok = wait_at(my_bars + kAtDone, segs & 1, abort_at, a.status);
                if (!ok) break;
                ++segs;
                tc_fence_after();
                if (warp_has_rows) {
                    const uint32_t o_addr = s_addr + (kColO - kColS);
                    TMEM_LD32(o_addr, v, 0); TMEM_LD32(o_addr + 32, v, 32);
                    TMEM_LD32(o_addr + 64, v, 64); TMEM_LD32(o_addr + 96, v, 96);
                    tmem_wait_ld();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at(my_bars + kAtFree);
                if (row_valid) {
                    uint4* part = a.parts + sg.part[turn] + row;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const uint32_t* x = v + 16 * c;
                        part[2 * c * 128] = make_uint4(upper_halves(x[0], x[1]), upper_halves(x[2], x[3]), upper_halves(x[4], x[5]), upper_halves(x[6], x[7]));
                        part[(2 * c + 1) * 128] = make_uint4(upper_halves(x[8], x[9]), upper_halves(x[10], x[11]), upper_halves(x[12], x[13]), upper_halves(x[14], x[15]));
                        part[(kPartThird + c) * 128] = make_uint4(third_bytes(x[0], x[1], x[2], x[3]), third_bytes(x[4], x[5], x[6], x[7]),
                                                                  third_bytes(x[8], x[9], x[10], x[11]), third_bytes(x[12], x[13], x[14], x[15]));
                    }
                    *reinterpret_cast<float2*>(part + kPartSums * 128) = make_float2(m_run, sg.bad ? -1.f : l_run);
                }
            }
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

// Merge: 32 rows of one key/value head of one sequence (lane <-> row, warp & 7 <-> 16 columns).  The rows lie in two M tiles at most of the shared
// rows' work, and in two of the sequence's own; a warp makes the list of each tile's parts.  Where a sequence has no more than 16 rows, several
// lanes share a row's parts and join what they have.  What bounds it is latency: lists, a barrier, a round of loads or two.  Three forms:
//   few blocks     four parts a round in flight
//   many           (more than two an SM) two parts a round in 64 registers, four blocks an SM.  16 x 64 nodes, 32 heads over 8: 156.0 -> 151.1 us
//                  with the main kernel; 42 sequences, 52 heads, a token each, under 203 rows 178 -> 168; 15 x 52 heads, 80 nodes 115.6 -> 105.2; with parts of
//                  two bytes an element 256 blocks 46.1 -> 46.5, 32 blocks 11.9 -> 12.8
//   long lists     (blocks fewer than the SMs, parts may be many) three times eight warps, which share the parts too, three parts a round (with
//                  four they spill: 22 -> 24.5, 37 -> 46): with few heads a row has a hundred and more.  16 heads over 2: two sequences, a
//                  token each, under 21k rows 44 -> 22 us; one sequence, 4 nodes, under 30k 51 -> 37; joined without need, 4 sequences of 32
//                  heads over 8, a token each, under 512 rows 11.4 -> 12.2
enum MergeForm { kFewBlocks, kManyBlocks, kLongLists };
constexpr int kMaxParts = 2 * 256;                           // lanes x CTAs that an item may lie in

constexpr int kJoiners = 3;                                  // warps that share the parts of 16 columns

template <MergeForm kForm>
__global__ void __launch_bounds__(kForm == kLongLists ? kJoiners * kCombineThreads : kCombineThreads, kForm == kManyBlocks ? 4 : 1)
tree_attn_shared_merge_kernel(const __grid_constant__ SharedArgs a, int H, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
    constexpr bool kJoin = kForm == kLongLists;
    constexpr int kRound = kForm == kManyBlocks ? 2 : kForm == kLongLists ? 3 : 4;   // parts whose loads are in flight together
    __shared__ uint32_t s_part[4][kMaxParts];                // places in the workspace
    __shared__ int s_parts[4];
    __shared__ float s_join[kJoin ? 18 : 1][8][32];
    const int s = blockIdx.z, hk = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, columns = kJoin ? warp & 7 : warp;
    const int joiner = kJoin ? warp >> 3 : 0, joiners = kJoin ? kJoiners : 1;
    const int nn = nodes_of(a.wk.n_nodes, s, a.wk.B), g = a.g;
    const int r0 = blockIdx.x * 32, in_block = min(32, a.wk.B * g - r0);
    const int width = in_block > 1 ? 1 << (32 - __clz(in_block - 1)) : 1;   // lanes beside one another, a row each; the next as many share their parts
    const int r = r0 + (lane & (width - 1)), node = r / g, member = r - node * g;
    const bool row_valid = (lane & (width - 1)) < in_block && node < nn;
    const int shared_first = (s * a.wk.B + r0 / g) / a.shared_nb, own_first = r0 / g / a.own_nb;   // M tiles of the block's first row
    if (warp < 4) {
        // (the lengths are final: the main kernel has let this one in behind its own wait)
        SharedWork wk = a.wk;
        long long sum = 0, before = 0;                       // tiles of all sequences, of those in front of this one
        int live_all = 0, live = 0;                          // and how many have any
        for (int s0 = 0; s0 < wk.S; s0 += 32) {
            const int T = s0 + lane < wk.S ? wk.tiles(s0 + lane) : 0;
            sum += __reduce_add_sync(0xFFFFFFFFu, (uint32_t)T);
            live_all += __popc(__ballot_sync(0xFFFFFFFFu, T > 0));
            const bool ahead = s0 + lane < s;
            before += __reduce_add_sync(0xFFFFFFFFu, (uint32_t)(ahead ? T : 0));
            live += __popc(__ballot_sync(0xFFFFFFFFu, ahead && T > 0));
        }
        wk.set(sum, live_all);
        const bool own = warp >= 2;
        const int m = (own ? own_first : shared_first) + (warp & 1), n_m = own ? wk.own_m : wk.shared_m;
        int n = 0;
        if (m < n_m) {
            const int T = own ? wk.tiles(s) : wk.shared_tiles, i = hk * (own ? wk.own_pairs() : wk.shared_pairs()) + (m >> 1);
            const long long first = own ? wk.shared_total + (long long)wk.Hkv * wk.own_pairs() * (before * wk.places(0) + (long long)wk.change(0) * live) : 0;
            SharedParts ps;
            ps.set(wk, own ? s : -1, i, first + (long long)i * wk.width(own ? s : -1, T), T, (m | 1) >= n_m, m & 1);
            for (int k0 = 0; k0 < ps.n; k0 += 32) {
                const int slot = k0 + lane < ps.n ? ps.slot(wk, k0 + lane) : -1;
                const uint32_t there = __ballot_sync(0xFFFFFFFFu, slot >= 0);
                if (slot >= 0) s_part[warp][n + __popc(there & ((1u << lane) - 1))] = wk.place(slot);
                n += __popc(there);
            }
        }
        if (lane == 0) s_parts[warp] = n;
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    // this row's lists and its rows in the M tiles
    const int tok = s * a.wk.B + node, m_shared = tok / a.shared_nb, m_own = node / a.own_nb;
    const int list0 = m_shared - shared_first, list1 = 2 + m_own - own_first;
    const int row0 = (tok - m_shared * a.shared_nb) * g + member, row1 = (node - m_own * a.own_nb) * g + member;
    const int n0 = row_valid ? s_parts[list0] : 0, n = row_valid ? n0 + s_parts[list1] : 0;
    const int sharers = 32 / width * joiners, sharer = lane / width + 32 / width * joiner;
    float M = -INFINITY, L = 0.f, acc[16];
    bool bad = false;
#pragma unroll
    for (int c = 0; c < 16; ++c) acc[c] = 0.f;
    for (int k0 = sharer; k0 < n; k0 += sharers * kRound) {
        float2 ml[kRound];
        uint4 x[kRound][3];
#pragma unroll
        for (int q = 0; q < kRound; ++q) {
            const int k = k0 + q * sharers;
            ml[q] = make_float2(-INFINITY, 0.f);
            x[q][0] = x[q][1] = x[q][2] = make_uint4(0, 0, 0, 0);
            if (k < n) {
                const uint4* part = a.parts + (k < n0 ? s_part[list0][k] + row0 : s_part[list1][k - n0] + row1);
                ml[q] = __ldcg(reinterpret_cast<const float2*>(part + kPartSums * 128));
                x[q][0] = __ldcg(part + (2 * columns) * 128);
                x[q][1] = __ldcg(part + (2 * columns + 1) * 128);
                x[q][2] = __ldcg(part + (kPartThird + columns) * 128);
            }
        }
        float M_new = M;
#pragma unroll
        for (int q = 0; q < kRound; ++q) { M_new = fmaxf(M_new, ml[q].x); bad |= ml[q].y < 0.f; }
        const float old = M == -INFINITY ? 0.f : ex2(M - M_new);
        L *= old;
#pragma unroll
        for (int c = 0; c < 16; ++c) acc[c] *= old;
#pragma unroll
        for (int q = 0; q < kRound; ++q) {
            if (ml[q].x == -INFINITY && ml[q].y == 0.f) continue;   // no key of the part is visible to the row
            const float w = ex2(ml[q].x - M_new);
            L += w * ml[q].y;
            const uint32_t thirds[4] = {x[q][2].x, x[q][2].y, x[q][2].z, x[q][2].w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t h0 = u & 1 ? x[q][u >> 1].z : x[q][u >> 1].x, h1 = u & 1 ? x[q][u >> 1].w : x[q][u >> 1].y;
                acc[4 * u] += w * part_element<0>(h0, thirds[u]);
                acc[4 * u + 1] += w * part_element<1>(h0, thirds[u]);
                acc[4 * u + 2] += w * part_element<2>(h1, thirds[u]);
                acc[4 * u + 3] += w * part_element<3>(h1, thirds[u]);
            }
        }
        M = M_new;
    }
    auto join = [&](float m, float l, auto part) {           // another's share
        const float M_new = fmaxf(M, m), mine = M == -INFINITY ? 0.f : ex2(M - M_new), theirs = m == -INFINITY ? 0.f : ex2(m - M_new);
        L = L * mine + l * theirs;
#pragma unroll
        for (int c = 0; c < 16; ++c) acc[c] = acc[c] * mine + part(c) * theirs;
        M = M_new;
    };
    for (int o = width; o < 32; o <<= 1) {
        const float m = __shfl_xor_sync(0xFFFFFFFFu, M, o), l = __shfl_xor_sync(0xFFFFFFFFu, L, o);
        bad |= __shfl_xor_sync(0xFFFFFFFFu, (int)bad, o) != 0;
        join(m, l, [&](int c) { return __shfl_xor_sync(0xFFFFFFFFu, acc[c], o); });
    }
    for (int j = joiners - 1; j > 0; --j) {
        if (joiner == j) {
            s_join[16][columns][lane] = M;
            s_join[17][columns][lane] = bad ? -1.f : L;
#pragma unroll
            for (int c = 0; c < 16; ++c) s_join[c][columns][lane] = acc[c];
        }
        __syncthreads();
        if (joiner == 0) {
            const float l = s_join[17][columns][lane];
            bad |= l < 0.f;
            join(s_join[16][columns][lane], l, [&](int c) { return s_join[c][columns][lane]; });
        }
        __syncthreads();
    }
    if (!row_valid || sharer > 0) return;
    const size_t at = ((size_t)s * a.wk.B + node) * H + hk * g + member;
    if (bad) {
        uint4* dst = reinterpret_cast<uint4*>(out + at * kHeadDim + 16 * columns);
        dst[0] = dst[1] = make_uint4(0, 0, 0, 0);
    } else {
        store_merged(out + at * kHeadDim + 16 * columns, acc, L);
    }
    if (lse && warp == 0) lse[at] = bad ? 0.f : (M + log2f(L)) * kLn2;
}

}  // namespace

// what the launch and its workspace are made of; false where the tensor maps cannot be made
static SharedArgs shared_args(const goose_ctx* c, int64_t kv_rows, int64_t shared_row, int shared_len, const int64_t* row_off,
                              const int32_t* ctx_len, const int32_t* parent, const int32_t* n_nodes, int S, int B, int H, int Hkv,
                              float scale) {
    SharedArgs a{};
    const int g = H / Hkv;
    a.row_off = row_off; a.parent = parent; a.g = g;
    a.shared_nb = min(kSharedTile / g, S * B);
    a.own_nb = min(B, kSharedTile / g);
    a.shared_row = (int)shared_row; a.shared_len = shared_len;
    a.scale_log2 = scale * kLog2e;
    a.wk.ctx_len = ctx_len; a.wk.n_nodes = n_nodes; a.wk.S = S; a.wk.B = B; a.wk.Hkv = Hkv; a.wk.kv_rows = (int)kv_rows;
    a.wk.shared_tiles = (int)(((int64_t)shared_len + kSharedTile - 1) / kSharedTile);
    a.wk.shared_m = (S * B + a.shared_nb - 1) / a.shared_nb;
    a.wk.own_m = (B + a.own_nb - 1) / a.own_nb;
    a.wk.G = c->num_sms < kMaxParts / 2 ? c->num_sms : kMaxParts / 2;
    a.status = c->status;
    return a;
}

cudaError_t launch_tree_attn_shared(goose_ctx* c, const __nv_bfloat16* q, const __nv_bfloat16* kc, const __nv_bfloat16* vc,
                                    int64_t kv_rows, int64_t shared_row, int shared_len, const int64_t* row_off,
                                    const int32_t* ctx_len, const int32_t* parent, const int32_t* n_nodes, int S, int B, int H,
                                    int Hkv, float scale, __nv_bfloat16* out, float* lse, cudaStream_t st) {
    if (!c->encode_tiled) return cudaErrorNotSupported;
    if (S == 0) return cudaSuccess;
    SharedArgs a = shared_args(c, kv_rows, shared_row, shared_len, row_off, ctx_len, parent, n_nodes, S, B, H, Hkv, scale);
    const size_t words = (size_t)a.wk.lay(a.shared_nb * a.g, a.own_nb * a.g) * kPartBlock;
    if (words > 0xFFFFFFFFull) return cudaErrorMemoryAllocation;   // (64 GB)
    if (cudaError_t e = grow(c, &c->shared_parts, &c->shared_bytes, sizeof(uint4) * words)) return e;
    a.parts = static_cast<uint4*>(c->shared_parts);
    CUtensorMap mqs, mqo, mk, mv;
    if (!make_q_map(c->encode_tiled, &mqs, q, (int64_t)S * B, Hkv, a.g, a.shared_nb) ||
        !make_q_map(c->encode_tiled, &mqo, q, (int64_t)S * B, Hkv, a.g, a.own_nb) ||
        !make_map(c->encode_tiled, &mk, kc, kv_rows, Hkv, kSharedTile) || !make_map(c->encode_tiled, &mv, vc, kv_rows, Hkv, kSharedTile))
        return cudaErrorInvalidValue;
    cudaError_t e = launch_pdl(tree_attn_shared_kernel, dim3(a.wk.G), dim3(kSharedThreads), kSharedSmem, st, mqs, mqo, mk, mv, a);
    c->launches++;
    if (e != cudaSuccess) return e;
    const dim3 blocks((B * a.g + 31) / 32, Hkv, S);
    // CTAs that an item may lie in, as far as the host knows: more warps a row where that makes many parts
    auto ctas = [&](long long tiles, long long items) { return tiles < a.wk.G / items ? tiles : a.wk.G / items; };
    const long long most = ctas(a.wk.shared_tiles, Hkv * a.wk.shared_pairs()) + ctas((kv_rows + kSharedTile - 1) / kSharedTile, (long long)S * Hkv * a.wk.own_pairs());
    const long long n_blocks = (long long)blocks.x * Hkv * S;
    const bool join = n_blocks < c->num_sms && most >= 12;
    auto merge = join ? tree_attn_shared_merge_kernel<kLongLists> : n_blocks > 2 * c->num_sms ? tree_attn_shared_merge_kernel<kManyBlocks>
                                                                                               : tree_attn_shared_merge_kernel<kFewBlocks>;
    e = launch_pdl(merge, blocks, dim3(join ? kJoiners * kCombineThreads : kCombineThreads), 0, st, a, H, out, lse);
    c->launches++;
    return e;
}

cudaError_t init_shared_kernel() {
    cudaError_t e = cudaFuncSetAttribute(tree_attn_shared_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedSmem);
    return e == cudaSuccess ? load_kernels({(const void*)tree_attn_shared_merge_kernel<kFewBlocks>, (const void*)tree_attn_shared_merge_kernel<kManyBlocks>,
                                            (const void*)tree_attn_shared_merge_kernel<kLongLists>}) : e;
}

}  // namespace goose
