// Tree attention of a batch whose sequences share a long prefix: the shared rows are streamed once for 256 query rows of all
// sequences, every sequence's own rows (its prefix and its tree) once for its own queries, and the two are merged by their
// log-sum-exp:  out = sum_p 2^(e_p - M) x_p / sum_p 2^(e_p - M),  x_p the normalised result over the keys of part p, e_p the logarithm
// (base 2) of its sum of exponentials, M the largest e_p.
//
// Main kernel: persistent, one CTA an SM, tcgen05 with TMEM accumulators, TMA loads, mbarrier pipeline; work list and lanes:
// shared_work.cuh.  A sequence's own rows are never met by another sequence's queries, not even masked: what they hold (infinities, NaN)
// stays in that sequence.  Roles (384 threads):
//   warp 0, lane 0    TMA producer: the queries of a segment, then K and V tiles into a ring of 32 KB stages
//   warp 1, lane 0    MMA issuer: S = Q K^T, O += P V, the two lanes in turn: while one lane's softmax runs, the tensor cores have the other's
//                     products
//   warps 4..7, 8..11 softmax of lane 0 and of lane 1: one query row a thread: maximum, exponentials, P (bf16) over S in tensor
//                     memory, lazy rescaling of O, at the segment's end the partial result into the workspace.
// Tensor memory: S of both lanes in columns 0..255, O of both in 256..511.
// Every wait is bounded: one that runs out raises the CTA's abort flag and GOOSE_ST_TIMEOUT, and every role unwinds.
#include <cuda_fp16.h>

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
constexpr int kHeaderBytes = 1024;
constexpr int kSharedSmem = kHeaderBytes + 1024 /*alignment slack*/ + 2 * kQBytes + kStages * kStageBytes;
constexpr int kSharedThreads = 384;
// registers: 168 a thread at launch; the warps of the loads and products give 112 each to the others (56 + 2 x 224 = 3 x 168)
constexpr int kRegsFew = 56, kRegsMany = 224;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0, kColO = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleThreshold = 8.0f;                    // rescale O only when the running max grew by > 2^8
constexpr long long kWaitCycles = 2000000000ll;              // bound of every wait: about one second of SM clock

// Partial result: x / scale as fp16, uint4 [16 groups of 8 columns][128 rows], then (e, scale) fp32 [128].  scale is the power of two of
// the row's largest element, so that a row of any size has 11 bits of its largest elements (the output has 8);  0: a sequence that
// cannot be computed (no tree, rows outside the cache).
constexpr int kPartWords = 16 * 128 * 4;
constexpr int kPartFloats = kPartWords + 2 * 128;

struct Header {
    unsigned long long kv_full[kStages];
    unsigned long long kv_empty[kStages];
    unsigned long long q_full, q_empty;
    unsigned long long s_full[2], p_ready[2], pv_done[2], o_free[2], group_bar[2];
    uint32_t tmem_base;
    volatile int abort_flag;
    int bad[2];
    signed char par[2][kMaxB];                               // parent[] of the current sequence, a copy a lane
};
static_assert(sizeof(Header) <= kHeaderBytes, "header");

struct SharedArgs {
    const int64_t* row_off;
    const int32_t* parent;
    SharedWork wk;
    int g;                                                   // query heads per key/value head
    int shared_nb, own_nb;                                   // tokens of an M tile: of the batch, of one sequence
    int shared_row, shared_len;
    float scale_log2;
    float* parts;
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
        const uint32_t own = (uint32_t)wk.width(T);
        uint32_t upto = own;                                 // (32 widths of 2^24 + 2 at most)
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

// the item at the cursor: its key/value head, its M tiles and their first tokens
struct Item {
    int hk, m, tokens[2];
    bool single;
    __device__ __forceinline__ Item(const SharedArgs& a, const SharedCursor& cu) {
        const bool shared = cu.s < 0;
        const int pairs = shared ? a.wk.shared_pairs() : a.wk.own_pairs(), n_m = shared ? a.wk.shared_m : a.wk.own_m;
        const int nb = shared ? a.shared_nb : a.own_nb;
        hk = cu.i / pairs;
        m = 2 * (cu.i - hk * pairs);
        single = m + 1 >= n_m;
        tokens[0] = (shared ? 0 : cu.s * a.wk.B) + m * nb;
        tokens[1] = tokens[0] + nb;
    }
};

__global__ void __launch_bounds__(kSharedThreads, 1)
tree_attn_shared_kernel(const __grid_constant__ CUtensorMap tmap_q_shared, const __grid_constant__ CUtensorMap tmap_q_own,
                        const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const SharedArgs a) {
    extern __shared__ unsigned char smem_raw[];
    Header* hd = reinterpret_cast<Header*>(smem_raw);
    unsigned char* q_smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + kHeaderBytes + 1023) & ~(uintptr_t)1023);
    unsigned char* kv_smem = q_smem + 2 * kQBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { mbar_init(&hd->kv_full[i], 1); mbar_init(&hd->kv_empty[i], 1); }
        mbar_init(&hd->q_full, 1); mbar_init(&hd->q_empty, 1);
        for (int l = 0; l < 2; ++l) {
            mbar_init(&hd->s_full[l], 1); mbar_init(&hd->p_ready[l], 128); mbar_init(&hd->pv_done[l], 1);
            mbar_init(&hd->o_free[l], 128); mbar_init(&hd->group_bar[l], 128);
            hd->bad[l] = 0;
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
    const uint32_t tmem = hd->tmem_base;
    pdl_wait();
    pdl_trigger();

    SharedWork wk = a.wk;
    if (wk.n_nodes && blockIdx.x == 0 && threadIdx.x == 33)
        for (int s = 0; s < wk.S; ++s)
            if (nodes_bad(wk.n_nodes, s, wk.B)) atomicOr(&a.status[s], GOOSE_ST_BAD_NODES);
    SharedCursor cu;
    long long w_end;
    locate(wk, cu, w_end, blockIdx.x, lane);

    if (cu.w < w_end) {
      if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
        if (warp == 0) {
            // =========================================================== TMA producer
            if (lane == 0) {
                // the shared rows are read by many CTAs, a sequence's own by one or two
                const unsigned long long pol_own = l2_policy_evict_first(), pol_shared = l2_policy_evict_last();
                uint32_t ring = 0, st = 0, phase = 0, seg = 0;
                bool ok = true;
                while (ok && cu.w < w_end) {
                    const Item it(a, cu);
                    const bool shared = cu.s < 0;
                    ok = wait_for(hd, &hd->q_empty, (seg & 1) ^ 1, a.status);
                    if (!ok) break;
                    const int tiles_q = it.single ? 1 : 2;
                    mbar_expect_tx(&hd->q_full, (uint32_t)(tiles_q * (shared ? a.shared_nb : a.own_nb) * a.g) * 256u);
                    const CUtensorMap* mq = shared ? &tmap_q_shared : &tmap_q_own;
                    for (int m = 0; m < tiles_q; ++m) {
                        tma_load_4d(q_smem + m * kQBytes, mq, &hd->q_full, 0, 0, it.hk, it.tokens[m]);
                        tma_load_4d(q_smem + m * kQBytes + kHalfBytes, mq, &hd->q_full, 64, 0, it.hk, it.tokens[m]);
                    }
                    ++seg;
                    const int n = cu.run(w_end);
                    int krow = (int)((shared ? a.shared_row : a.row_off[cu.s]) + (int64_t)cu.t * kSharedTile);
                    const unsigned long long pol = shared ? pol_shared : pol_own;
                    for (int i = 0; i < n && ok; ++i, krow += kSharedTile) {
                        for (int kv = 0; kv < 2 && ok; ++kv) {
                            ok = wait_for(hd, &hd->kv_empty[st], phase ^ 1, a.status);
                            if (!ok) break;
                            unsigned char* dst = kv_smem + st * kStageBytes;
                            mbar_expect_tx(&hd->kv_full[st], kStageBytes);
                            const CUtensorMap* mp = kv ? &tmap_v : &tmap_k;
                            tma_load_3d_hint(dst, mp, &hd->kv_full[st], 0, it.hk, krow, pol);
                            tma_load_3d_hint(dst + kHalfBytes, mp, &hd->kv_full[st], 64, it.hk, krow, pol);
                            ++ring;
                            if (++st == kStages) { st = 0; phase ^= 1; }
                        }
                    }
                    cu.skip(wk, n);
                }
                if (!ok) {                                   // copies still in flight land before the CTA ends
                    for (uint32_t r = ring > kStages ? ring - kStages : 0; r < ring; ++r) drain(&hd->kv_full[r % kStages], (r / kStages) & 1);
                    if (seg > 0) drain(&hd->q_full, (seg - 1) & 1);
                }
            }
        } else if (warp == 1) {
            // =========================================================== MMA issuer
            if (lane == 0) {
                const uint32_t q_addr = smem_u32(q_smem), kv_addr = smem_u32(kv_smem);
                constexpr uint32_t idesc_qk = instr_desc(false), idesc_pv = instr_desc(true);
                uint32_t k_st = 0, k_phase = 0, v_st = 1, v_phase = 0;   // every second stage of the ring
                auto next_stage = [](uint32_t& st, uint32_t& phase) {
                    st += 2;
                    if (st >= kStages) { st -= kStages; phase ^= 1; }
                };
                uint32_t ops[2] = {0, 0}, segs[2] = {0, 0}, seg = 0;     // products and segments of a lane; segments
                bool ok = true;
                while (ok && cu.w < w_end) {
                    const Item it(a, cu);
                    ok = wait_for(hd, &hd->q_full, seg & 1, a.status);
                    if (!ok) break;
                    const int n = cu.run(w_end), n_ops = it.single ? n : 2 * n;
                    // step o: P V of step o - 2 (the same lane), then Q K^T of step o over what that P was
                    for (int o = 0; o < n_ops + 2 && ok; ++o) {
                        const int l = o & 1;
                        if (o >= 2) {
                            if (!(ok = wait_for(hd, &hd->p_ready[l], ops[l] & 1, a.status))) break;
                            if (!(ok = wait_for(hd, &hd->kv_full[v_st], v_phase, a.status))) break;
                            if (o < 4 && segs[l] > 0 && !(ok = wait_for(hd, &hd->o_free[l], (segs[l] - 1) & 1, a.status))) break;
                            tc_fence_after();
                            const uint32_t v_lo = smem_desc_lo(kv_addr + v_st * kStageBytes, kHalfBytes);   // MN-major: LBO = next 64 d
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)   // 16 keys per instruction
                                umma_f16_ts(tmem + kColO + l * 128, tmem + kColS + l * 128 + kk * 8, smem_desc(v_lo + kk * (2048 >> 4)), idesc_pv,
                                            (o >= 4 || kk > 0) ? 1u : 0u);
                            const bool last_use = it.single || l == 1;
                            if (last_use) umma_commit(&hd->kv_empty[v_st]);
                            umma_commit(&hd->pv_done[l]);
                            if (last_use) next_stage(v_st, v_phase);
                            ++ops[l];
                        }
                        if (o < n_ops) {
                            if (!(ok = wait_for(hd, &hd->kv_full[k_st], k_phase, a.status))) break;
                            tc_fence_after();
                            const uint32_t q_lo = smem_desc_lo(q_addr + (it.single ? 0 : l) * kQBytes, 16);
                            const uint32_t k_lo = smem_desc_lo(kv_addr + k_st * kStageBytes, 16);
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk) { // 16 of the 128 head dims per instruction
                                const uint32_t off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
                                umma_f16(tmem + kColS + l * 128, smem_desc(q_lo + off), smem_desc(k_lo + off), idesc_qk, kk > 0 ? 1u : 0u);
                            }
                            umma_commit(&hd->s_full[l]);
                            if (it.single || l == 1) {
                                umma_commit(&hd->kv_empty[k_st]);
                                next_stage(k_st, k_phase);
                            }
                            if (o == n_ops - 1) umma_commit(&hd->q_empty);
                        }
                    }
                    if (!ok) break;
                    ++segs[0];
                    if (n_ops > 1) ++segs[1];
                    ++seg;
                    cu.skip(wk, n);
                }
            }
        }
      } else {
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsMany));
            // =========================================================== softmax and partial results (two groups of 128 threads)
            const int l = warp >= 8;                         // lane of the segment
            const int row = 32 * (warp & 3) + lane;          // TMEM lane == query row
            const uint32_t lane_sel = (uint32_t)(32 * (warp & 3)) << 16;
            const uint32_t s_addr = tmem + kColS + l * 128 + lane_sel, o_addr = tmem + kColO + l * 128 + lane_sel;
            const int tid = threadIdx.x - 128 - 128 * l;
            const int g = a.g, i_local = row / g;
            uint32_t ops = 0, tile0 = 0, syncs = 0;          // products of this lane; tiles of the CTA in front of this segment
            bool ok = true;
            uint32_t v[128];
            int cur_s = -1;
            bool bad = false;
            auto group_sync = [&]() {
                mbar_arrive(&hd->group_bar[l]);
                const bool done = wait_for(hd, &hd->group_bar[l], syncs & 1, a.status);
                ++syncs;
                return done;
            };

            while (ok && cu.w < w_end) {
                const Item it(a, cu);
                const bool shared = cu.s < 0;
                const int s = cu.s, n = cu.run(w_end), t_first = cu.t, t_end = t_first + n;
                const int step = it.single ? 2 : 1;
                const int t_mine = it.single ? t_first + l : t_first;        // this lane's first tile
                if (t_mine >= t_end) {                       // one key tile: lane 0 has it
                    tile0 += n;
                    cu.skip(wk, n);
                    continue;
                }
                const int m = it.m + (it.single ? 0 : l);
                const int nn = shared ? 0 : nodes_of(wk.n_nodes, s, wk.B);
                const int ctx = shared ? a.shared_len : wk.prefix(wk.ctx_len[s]);
                const int n_keys = ctx + nn;
                const int rows = shared ? min(a.shared_nb, wk.S * wk.B - m * a.shared_nb) * g : min(a.own_nb, nn - m * a.own_nb) * g;
                const bool row_valid = row < rows, warp_has_rows = 32 * (warp & 3) < rows;
                const int node = m * a.own_nb + i_local;     // (of a sequence's own rows)
                if (!shared && s != cur_s) {
                    // parent[] and rows of the sequence: both groups come to the same verdict
                    cur_s = s;
                    if (tid < nn) {
                        const int p = a.parent[(size_t)s * wk.B + tid];
                        hd->par[l][tid] = (signed char)p;
                        if (tid == 0 ? p != -1 : (p < 0 || p >= tid)) hd->bad[l] = 1;
                    }
                    const bool bad_rows = rows_outside(a.row_off[s], wk.ctx_len[s], nn, wk.kv_rows);
                    if (bad_rows && tid == 0) { hd->bad[l] = 1; atomicOr(&a.status[s], GOOSE_ST_BAD_ROWS); }
                    ok = group_sync();
                    bad = hd->bad[l] != 0;
                    ok = ok && group_sync();
                    if (!ok) break;
                    if (tid == 0 && bad) { hd->bad[l] = 0; if (!bad_rows) atomicOr(&a.status[s], GOOSE_ST_BAD_PARENT); }
                }
                uint32_t anc[4] = {0, 0, 0, 0};
                if (!shared && t_end * kSharedTile > ctx && row_valid && !bad) {
                    int vtx = node;
                    for (int up = 0; up < kMaxB && vtx >= 0; ++up) {
                        const uint32_t bit = 1u << (vtx & 31);
                        const int wsel = vtx >> 5;
                        anc[0] |= (wsel == 0) ? bit : 0; anc[1] |= (wsel == 1) ? bit : 0;
                        anc[2] |= (wsel == 2) ? bit : 0; anc[3] |= (wsel == 3) ? bit : 0;
                        vtx = hd->par[l][vtx];
                    }
                }
                float m_run = -INFINITY, l_run = 0.f;
                for (int t = t_mine; t < t_end; t += step) {
                    const bool first = t == t_mine;
                    ok = wait_for(hd, &hd->s_full[l], ops & 1, a.status);
                    if (!ok) break;
                    tc_fence_after();
                    if (warp_has_rows) {
                        TMEM_LD32(s_addr, v, 0); TMEM_LD32(s_addr + 32, v, 32);
                        TMEM_LD32(s_addr + 64, v, 64); TMEM_LD32(s_addr + 96, v, 96);
                        tmem_wait_ld();
                        const int key0 = t * kSharedTile;
                        if (key0 + kSharedTile > ctx) {      // the tree rows, or the ragged end
                            // visibility of the tile's 128 keys as one mask: the prefix keys, and the ancestors shifted to where
                            // the tree rows start
                            const int pc = ctx - key0;       // tile column of tree node 0 (may be < 0 or >= 128)
                            const unsigned __int128 a128 =
                                ((unsigned __int128)(((unsigned long long)anc[3] << 32) | anc[2]) << 64) |
                                (unsigned __int128)(((unsigned long long)anc[1] << 32) | anc[0]);
                            unsigned __int128 vm;
                            if (pc >= 128) vm = ~(unsigned __int128)0;
                            else if (pc > 0) vm = (((unsigned __int128)1 << pc) - 1) | (a128 << pc);
                            else if (pc > -128) vm = a128 >> (-pc);
                            else vm = 0;
                            const uint32_t vw[4] = {(uint32_t)vm, (uint32_t)(vm >> 32), (uint32_t)(vm >> 64), (uint32_t)(vm >> 96)};
#pragma unroll
                            for (int c = 0; c < 128; ++c) v[c] = ((vw[c >> 5] >> (c & 31)) & 1u) ? v[c] : 0xFF800000u;   // -inf
                        }
                        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int c = 0; c < 128; c += 8)
#pragma unroll
                            for (int e = 0; e < 4; ++e) mx4[e] = max3(mx4[e], __uint_as_float(v[c + 2 * e]), __uint_as_float(v[c + 2 * e + 1]));
                        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * a.scale_log2;   // scale > 0
                        const float m_new = fmaxf(m_run, mx);
                        if (__any_sync(0xFFFFFFFFu, first || (row_valid && m_new > m_run + kRescaleThreshold))) {
                            const float alpha = (m_run == -INFINITY) ? 0.f : ex2(m_run - m_new);
                            if (!first) {
                                ok = wait_for(hd, &hd->pv_done[l], (ops - 1) & 1, a.status);
                                if (ok) {
                                    tc_fence_after();
                                    uint32_t o[16];
#pragma unroll
                                    for (int cc = 0; cc < 8; ++cc) {
                                        TMEM_LD16(o_addr + cc * 16, o, 0);
                                        tmem_wait_ld();
#pragma unroll
                                        for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
                                        TMEM_ST16(o_addr + cc * 16, o, 0);
                                    }
                                    tmem_wait_st();
                                }
                            }
                            l_run *= alpha;
                            m_run = m_new;
                        }
                        const float neg_m = (m_run == -INFINITY) ? 0.f : -m_run;
                        const unsigned long long scale2 = pack_f32x2(a.scale_log2, a.scale_log2), neg2 = pack_f32x2(neg_m, neg_m);
                        unsigned long long ls2[2] = {0, 0};
#pragma unroll
                        for (int e = 0; e < 64; ++e) {
                            const float2 x2 = unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1])), scale2, neg2));
                            const float p0 = ex2(x2.x), p1 = ex2(x2.y);
                            ls2[e & 1] = add_f32x2(ls2[e & 1], pack_f32x2(p0, p1));
                            v[e] = pack_bf16x2(p0, p1);
                        }
                        const float2 l2 = unpack_f32x2(add_f32x2(ls2[0], ls2[1]));
                        l_run += l2.x + l2.y;
                        TMEM_ST32(s_addr, v, 0);
                        TMEM_ST32(s_addr + 32, v, 32);
                        tmem_wait_st();
                    }
                    // observe every phase of pv_done in order
                    if (ok && ops > 0) ok = wait_for(hd, &hd->pv_done[l], (ops - 1) & 1, a.status);
                    if (!ok) break;
                    // ragged end: V rows past the last key may hold anything -> zeros, in a tile that both lanes use by lane 0, whose
                    // product comes first
                    if ((t + 1) * kSharedTile > n_keys && (it.single || l == 0)) {
                        const uint32_t ring = 2 * (tile0 + (t - t_first)) + 1, st = ring % kStages;
                        ok = wait_for(hd, &hd->kv_full[st], (ring / kStages) & 1, a.status);
                        if (!ok) break;
                        const int first_off = max(n_keys - t * kSharedTile, 0) * 128;
                        for (int off = first_off + tid * 16; off < kHalfBytes; off += 128 * 16) {
                            *reinterpret_cast<uint4*>(kv_smem + st * kStageBytes + off) = make_uint4(0, 0, 0, 0);
                            *reinterpret_cast<uint4*>(kv_smem + st * kStageBytes + kHalfBytes + off) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async();
                    }
                    tc_fence_before();
                    mbar_arrive(&hd->p_ready[l]);
                    ++ops;
                }
                if (!ok) break;
                // ---------------- partial result of this lane
                ok = wait_for(hd, &hd->pv_done[l], (ops - 1) & 1, a.status);
                if (!ok) break;
                tc_fence_after();
                if (warp_has_rows) {
                    TMEM_LD32(o_addr, v, 0); TMEM_LD32(o_addr + 32, v, 32);
                    TMEM_LD32(o_addr + 64, v, 64); TMEM_LD32(o_addr + 96, v, 96);
                    tmem_wait_ld();
                }
                tc_fence_before();
                mbar_arrive(&hd->o_free[l]);
                if (row_valid) {
                    float* part = a.parts + (size_t)wk.slot(wk.item(s, cu.i), blockIdx.x, t_first == 0, t_end == cu.T, l) * kPartFloats;
                    float top = 0.f;
#pragma unroll
                    for (int c = 0; c < 128; ++c) top = fmaxf(top, fabsf(__uint_as_float(v[c])));
                    float inv = l_run == 0.f ? 0.f : 1.f / l_run;
                    top *= inv;
                    // power of two of the largest element; 1 where there is none (zeros, infinities)
                    const uint32_t ex = __float_as_uint(top) & 0x7F800000u;
                    const float scale = ex == 0 || ex >= 0x7F000000u ? 1.f : __uint_as_float(ex);
                    inv *= 1.f / scale;
                    uint4* dst = reinterpret_cast<uint4*>(part) + row;
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        uint32_t hw[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const __half2 h2 = __floats2half2_rn(__uint_as_float(v[8 * c + 2 * e]) * inv, __uint_as_float(v[8 * c + 2 * e + 1]) * inv);
                            hw[e] = *reinterpret_cast<const uint32_t*>(&h2);
                        }
                        dst[c * 128] = make_uint4(hw[0], hw[1], hw[2], hw[3]);
                    }
                    reinterpret_cast<float2*>(part + kPartWords)[row] =
                        make_float2(l_run == 0.f ? -INFINITY : m_run + log2f(l_run), !shared && bad ? 0.f : scale);
                }
                tile0 += n;
                cu.skip(wk, n);
            }
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

// Merge: 32 rows of one key/value head of one sequence (lane <-> row, warp <-> 16 columns), parts in rounds of kCombineRound.
__global__ void __launch_bounds__(kCombineThreads)
tree_attn_shared_merge_kernel(const SharedArgs a, int H, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
    const int s = blockIdx.z, hk = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    SharedWork wk = a.wk;
    // (the lengths are final: the main kernel has let this one in behind its own wait)
    long long sum = 0, before = 0;                           // tiles of all sequences, of those in front of this one
    int live_all = 0, live = 0;                              // and how many have any
    for (int s0 = 0; s0 < wk.S; s0 += 32) {
        const int T = s0 + lane < wk.S ? wk.tiles(s0 + lane) : 0;
        sum += __reduce_add_sync(0xFFFFFFFFu, (uint32_t)T);
        live_all += __popc(__ballot_sync(0xFFFFFFFFu, T > 0));
        const bool ahead = s0 + lane < s;
        before += __reduce_add_sync(0xFFFFFFFFu, (uint32_t)(ahead ? T : 0));
        live += __popc(__ballot_sync(0xFFFFFFFFu, ahead && T > 0));
    }
    wk.set(sum, live_all);
    const int T = wk.tiles(s), nn = nodes_of(wk.n_nodes, s, wk.B);
    const int g = a.g, r = blockIdx.x * 32 + lane, node = r / g, member = r - node * g;
    SharedParts ps[2];
    int at_row[2];
    {
        const int tok = s * wk.B + node, m = tok / a.shared_nb, pair = m >> 1;
        const int i = hk * wk.shared_pairs() + pair;
        ps[0].set(wk, -1, i, (long long)i * wk.width(wk.shared_tiles), wk.shared_tiles, (m | 1) >= wk.shared_m, m & 1);
        at_row[0] = (tok - m * a.shared_nb) * g + member;
    }
    {
        const int m = node / a.own_nb, pair = m >> 1;
        const int i = hk * wk.own_pairs() + pair;
        const long long per = (long long)wk.Hkv * wk.own_pairs();
        ps[1].set(wk, s, i, wk.shared_total + per * (before + wk.pad * live) + (long long)i * wk.width(T), T, (m | 1) >= wk.own_m, m & 1);
        at_row[1] = (node - m * a.own_nb) * g + member;
    }
    pdl_wait();
    pdl_trigger();
    if (node >= nn) return;

    float M = -INFINITY, L = 0.f, acc[16];
    bool bad = false;
#pragma unroll
    for (int c = 0; c < 16; ++c) acc[c] = 0.f;
    const int n = ps[0].n + ps[1].n;
    for (int k0 = 0; k0 < n; k0 += kCombineRound) {
        float2 meta[kCombineRound];
        uint4 x[kCombineRound][2];
#pragma unroll
        for (int q = 0; q < kCombineRound; ++q) {
            const int k = k0 + q;
            const bool own = k >= ps[0].n;
            const int slot = k < n ? (own ? ps[1].slot(wk, k - ps[0].n) : ps[0].slot(wk, k)) : -1;
            meta[q] = make_float2(-INFINITY, 1.f);
            x[q][0] = x[q][1] = make_uint4(0, 0, 0, 0);
            if (slot >= 0) {
                const float* part = a.parts + (size_t)slot * kPartFloats;
                const int rr = own ? at_row[1] : at_row[0];
                meta[q] = __ldcg(reinterpret_cast<const float2*>(part + kPartWords) + rr);
                x[q][0] = __ldcg(reinterpret_cast<const uint4*>(part) + (2 * warp) * 128 + rr);
                x[q][1] = __ldcg(reinterpret_cast<const uint4*>(part) + (2 * warp + 1) * 128 + rr);
            }
        }
        float M_new = M;
#pragma unroll
        for (int q = 0; q < kCombineRound; ++q) { M_new = fmaxf(M_new, meta[q].x); bad |= meta[q].y == 0.f; }
        const float old = M == -INFINITY ? 0.f : ex2(M - M_new);
        L *= old;
#pragma unroll
        for (int c = 0; c < 16; ++c) acc[c] *= old;
#pragma unroll
        for (int q = 0; q < kCombineRound; ++q) {
            if (meta[q].x == -INFINITY) continue;
            const float w = ex2(meta[q].x - M_new), wx = w * meta[q].y;
            L += w;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t hw[4] = {x[q][u].x, x[q][u].y, x[q][u].z, x[q][u].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&hw[e]));
                    acc[8 * u + 2 * e] += wx * f.x;
                    acc[8 * u + 2 * e + 1] += wx * f.y;
                }
            }
        }
        M = M_new;
    }
    const size_t at = ((size_t)s * wk.B + node) * H + hk * g + member;
    if (bad) {
        uint4* dst = reinterpret_cast<uint4*>(out + at * kHeadDim + 16 * warp);
        dst[0] = dst[1] = make_uint4(0, 0, 0, 0);
    } else {
        store_merged(out + at * kHeadDim + 16 * warp, acc, L);
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
    a.wk.G = c->num_sms;
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
    const size_t need = sizeof(float) * (size_t)a.wk.slots() * kPartFloats;
    if (cudaError_t e = grow(&c->shared_parts, &c->shared_bytes, need)) return e;
    a.parts = static_cast<float*>(c->shared_parts);
    CUtensorMap mqs, mqo, mk, mv;
    if (!make_q_map(c->encode_tiled, &mqs, q, (int64_t)S * B, Hkv, a.g, a.shared_nb) ||
        !make_q_map(c->encode_tiled, &mqo, q, (int64_t)S * B, Hkv, a.g, a.own_nb) ||
        !make_map(c->encode_tiled, &mk, kc, kv_rows, Hkv, kSharedTile) || !make_map(c->encode_tiled, &mv, vc, kv_rows, Hkv, kSharedTile))
        return cudaErrorInvalidValue;
    cudaError_t e = launch_pdl(tree_attn_shared_kernel, dim3(a.wk.G), dim3(kSharedThreads), kSharedSmem, st, mqs, mqo, mk, mv, a);
    c->launches++;
    if (e != cudaSuccess) return e;
    e = launch_pdl(tree_attn_shared_merge_kernel, dim3((B * a.g + 31) / 32, Hkv, S), dim3(kCombineThreads), 0, st, a, H, out, lse);
    c->launches++;
    return e;
}

cudaError_t init_shared_kernel() {
    cudaError_t e = cudaFuncSetAttribute(tree_attn_shared_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedSmem);
    return e == cudaSuccess ? load_kernels({(const void*)tree_attn_shared_merge_kernel}) : e;
}

}  // namespace goose
