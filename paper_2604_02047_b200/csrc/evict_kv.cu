// Eviction: the rows of a key/value head that stay, and the rows behind the budget among them to the places of those in front of it that do not.
//
// A row's key is an unsigned number in the order of what stays: the first and the latest positions above everything, then the weights, NaN below all.
// The budget-th largest key is found digit by digit (11, 11 and 10 bits, as far as it takes: the first has the exponent and two bits more, so that weights spread over some
// fifty of its counters); of the rows that have that very key the lowest stay.
// The first kernel, a block of 256 to 1024 threads a (sequence, head), reads weights and positions once, has the keys in shared memory, and leaves a list of (place, row) pairs;
// the second copies the rows.  Places lie in front of the budget, rows behind it, so that no copy reads what another one writes.
// (Closing the rows up instead would move nearly every row that stays.)  What bounds it: trips to L2 and barriers of the first kernel, 8 us for 4096 rows, 13 for 9000,
// then HBM (16 sequences of 9000 rows, 8 heads, to 4096: 71 us, of which the copies of 308 MB are 55).
#include <algorithm>

#include "goose_internal.cuh"

namespace goose {

constexpr int kMoveThreads = 256;
constexpr int kMovesOnce = 2;
constexpr int kBatch = 4;
constexpr int kBins = 2048;                           // counters of a digit
constexpr int kMostKeys = 24576;                      // keys in shared memory: two blocks an SM; rows behind them are looked up again
constexpr int kSelectSmem = 212992;                   // of a block, at most: a bit a row, a number for 32 rows, keys
constexpr int kSelectStatic = 4 * kBins + 1536;       // and what it has besides (the system's 1024 bytes included)
constexpr int kSmemOfAnSm = 233472;

constexpr int kMovesAhead = 4;                        // words that stand in front of a head's list (its length)

// of the row's position and weight
__device__ __forceinline__ uint32_t evict_key(float w, int pos, int sink, int64_t recent_from) {
    if (pos < sink || pos >= recent_from) return 0xFFFFFFFFu;
    if (!(w == w)) return 0;
    const uint32_t b = __float_as_uint(w + 0.f);      // (-0 + 0 = +0)
    return b >> 31 ? ~b : b | 0x80000000u;
}

// exclusive prefix sum over the block's threads; total in every thread.  s_warp: kThreads / 32 words of its own
template <int kThreads>
__device__ __forceinline__ int block_prefix(int v, int* s_warp, int& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int upto = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += u;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    int w = lane < kThreads / 32 ? s_warp[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(0xFFFFFFFFu, w, o);
        if (lane >= o) w += u;
    }
    total = __shfl_sync(0xFFFFFFFFu, w, 31);
    const int before = __shfl_sync(0xFFFFFFFFu, w, warp == 0 ? 0 : warp - 1);
    return upto - v + (warp == 0 ? 0 : before);
}

// kBatch loads of a thread in flight: what bounds a block is the trips to L2 (one at a time, and one row a lane group in the copies: 4096 rows to 2048 12.7 us, 16 sequences
// 45.9; these 12.4, 45.2; 8 and 4 of them 16.8, 53: registers)
template <int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
evict_select_kernel(const EvictKv a, int32_t* __restrict__ moves, int64_t moves_ld, int keep_words, int keys_there, int32_t* __restrict__ status) {
    extern __shared__ uint32_t s_keep[];              // a bit a row: it stays
    int* const s_rank = reinterpret_cast<int*>(s_keep + keep_words);   // of a word's first pair
    uint32_t* const s_key = s_keep + 2 * keep_words;  // of the first keys_there rows
    __shared__ int s_hist[kBins], s_warp[kThreads / 32], s_digit, s_above, s_equal;
    constexpr int kDigits = kBins / kThreads;
    const int s = blockIdx.y, hk = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
    const size_t head = (size_t)s * a.Hkv + hk;
    for (int b = tid; b < kBins; b += kThreads) s_hist[b] = 0;
    pdl_wait();
    pdl_trigger();
    const int ctx = a.ctx_len[s], off = a.pos_off ? a.pos_off[s] : 0, left = min(ctx, a.budget);
    int32_t* list = moves + head * moves_ld;
    const int64_t room = a.pages.room(a.ldw);
    bool bad = ctx < 0 || ctx > room || left > a.ldw_new;
    const int pages = bad ? 0 : (ctx + (1 << a.pages.size_log2) - 1) >> a.pages.size_log2;
#pragma unroll 4
    for (int p = tid; p < pages; p += kThreads) {
        const int page = a.pages.table[s * a.pages.ldt + p];
        bad |= page < 0 || page >= a.pages.n;
    }
    bad = __syncthreads_or(bad);
    if (tid == 0) {
        list[0] = 0;
        if (hk == 0) {
            a.new_ctx_len[s] = bad ? ctx : left;
            a.new_pos_off[s] = bad ? off : (int)((int64_t)off + (ctx - left));
            if (bad) atomicOr(&status[s], GOOSE_ST_BAD_ROWS);
        }
    }
    if (bad) return;
    const float* __restrict__ weight = a.row_weight + head * a.ldw;
    const int32_t* __restrict__ pos = a.row_pos + head * a.ldw;
    float* __restrict__ new_weight = a.new_weight + head * a.ldw_new;
    int32_t* __restrict__ new_pos = a.new_pos + head * a.ldw_new;
    // f(row, weight, position) for the rows first + tid, first + tid + kThreads, ... in front of n
    auto each_row = [&](int n, auto f) {
        for (int j0 = tid; j0 < n; j0 += kBatch * kThreads) {
            float w[kBatch];
            int p[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int j = min(j0 + u * kThreads, n - 1);
                w[u] = weight[j];
                p[u] = pos[j];
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (j0 + u * kThreads < n) f(j0 + u * kThreads, w[u], p[u]);
        }
    };
    if (ctx <= a.budget) {
        each_row(ctx, [&](int j, float w, int p) { new_weight[j] = w; new_pos[j] = p; });
        return;
    }
    const int64_t recent_from = (int64_t)off + ctx - a.recent;
    auto key = [&](int j) { return j < keys_there ? s_key[j] : evict_key(weight[j], pos[j], a.sink, recent_from); };
    // the budget-th largest key: its upper digits so far, and how many of the rows that have them are still to be taken
    uint32_t prefix = 0;
    int need = a.budget, total, low = 0;
    for (const int shift : {21, 10, 0}) {
        const int digit_bits = shift == 0 ? 10 : 11;
        if (shift == 21) {
            each_row(ctx, [&](int j, float w, int p) {
                const uint32_t k = evict_key(w, p, a.sink, recent_from);
                if (j < keys_there) s_key[j] = k;
                atomicAdd(&s_hist[k >> 21], 1);
            });
        } else {
#pragma unroll 4
            for (int j = tid; j < ctx; j += kThreads) {
                const uint32_t k = key(j);
                if (k >> (shift + digit_bits) == prefix) atomicAdd(&s_hist[k >> shift & ((1 << digit_bits) - 1)], 1);
            }
        }
        __syncthreads();
        // thread t has the digits from kBins - 1 - kDigits t down: how many rows have a larger one
        const int high = kBins - 1 - kDigits * tid;
        int mine[kDigits], sum = 0;
#pragma unroll
        for (int u = 0; u < kDigits; ++u) {
            mine[u] = s_hist[high - u];
            s_hist[high - u] = 0;
            sum += mine[u];
        }
        int above = block_prefix<kThreads>(sum, s_warp, total);
#pragma unroll
        for (int u = 0; u < kDigits; ++u) {
            if (above < need && above + mine[u] >= need) {
                s_digit = high - u;
                s_above = above;
                s_equal = mine[u];
            }
            above += mine[u];
        }
        __syncthreads();
        prefix = prefix << digit_bits | (uint32_t)s_digit;
        need -= s_above;
        low = shift;
        if (s_equal == need) break;                   // all that have these digits stay: the others do not matter
    }
    // what stays, in words of 32 rows; a warp's rows are consecutive
    const int words = (ctx + 31) >> 5, per = (words + kThreads / 32 - 1) / (kThreads / 32);
    const int w0 = min((tid >> 5) * per, words), w1 = min(w0 + per, words);
    int before = 0;                                   // rows of that very key in front of the warp's
    const bool ties = s_equal != need;                // (else all of them stay)
    if (ties) {
        int equal = 0;
        for (int w = w0; w < w1; ++w) {
            const int j = 32 * w + lane;
            equal += __popc(__ballot_sync(0xFFFFFFFFu, j < ctx && key(j) == prefix));
        }
        before = block_prefix<kThreads>(lane == 0 ? equal : 0, s_warp, total);
        before = __shfl_sync(0xFFFFFFFFu, before, 0);
    }
#pragma unroll 4
    for (int w = w0; w < w1; ++w) {
        const int j = 32 * w + lane;
        const uint32_t k = j < ctx ? key(j) >> low : 0u;
        bool stays = j < ctx && k >= prefix;
        if (ties) {
            const uint32_t same = __ballot_sync(0xFFFFFFFFu, j < ctx && k == prefix);
            stays = stays && (k > prefix || before + __popc(same & ((1u << lane) - 1)) < need);
            before += __popc(same);
        }
        const uint32_t word = __ballot_sync(0xFFFFFFFFu, stays);
        if (lane == 0) s_keep[w] = word;
    }
    __syncthreads();
    // Pairs of a dropped row in front of the budget and a kept one from it on.  Both counted in one row of words: those of the dropped up to the word that
    // the budget is in, then, from that word on, those of the kept.
    const int b0 = a.budget >> 5;
    const uint32_t inside = (1u << (a.budget & 31)) - 1;   // of word b0: rows in front of the budget
    const int entries = words + 1, each = (entries + kThreads - 1) / kThreads, e0 = min(tid * each, entries), e1 = min(e0 + each, entries);
    auto pairs = [&](int e) { return e < b0 ? ~s_keep[e] : e == b0 ? ~s_keep[e] & inside : s_keep[e - 1] & (e == b0 + 1 ? ~inside : 0xFFFFFFFFu); };
    int count = 0;
    for (int e = e0; e < e1; ++e) count += __popc(pairs(e));
    int at = block_prefix<kThreads>(count, s_warp, total);
    for (int e = e0; e < e1; ++e) {
        s_rank[e] = at;
        at += __popc(pairs(e));
    }
    const int n = total / 2;                          // (as many dropped as kept)
    int32_t* const list_to = list + kMovesAhead;
    int32_t* const list_of = list_to + (moves_ld - kMovesAhead) / 2;
    // (the keys are not needed any more, and the pairs are no more than half as many)
    const bool fit = ctx <= keys_there;
    int32_t* const to = fit ? reinterpret_cast<int32_t*>(s_key) : list_to;
    int32_t* const of = fit ? to + ctx / 2 : list_of;
    if (tid == 0) list[0] = n;
    __syncthreads();
    for (int j = a.budget + tid; j < ctx; j += kThreads) {
        const uint32_t word = s_keep[j >> 5] & (j >> 5 == b0 ? ~inside : 0xFFFFFFFFu);
        if (word >> (j & 31) & 1) of[s_rank[(j >> 5) + 1] - n + __popc(word & ((1u << (j & 31)) - 1))] = j;
    }
    // weights and positions of what stays where it is, then of what changes its place; the lists go on with rows of the caches in place of the sequence's
    each_row(a.budget, [&](int j, float w, int p) {
        const uint32_t word = s_keep[j >> 5];
        if (word >> (j & 31) & 1) { new_weight[j] = w; new_pos[j] = p; }
        else to[s_rank[j >> 5] + __popc(~word & ((1u << (j & 31)) - 1))] = j;
    });
    __syncthreads();
    for (int m0 = tid; m0 < n; m0 += kBatch * kThreads) {
        int t[kBatch], f[kBatch], p[kBatch], row_t[kBatch], row_f[kBatch];
        float w[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int m = m0 + u * kThreads < n ? m0 + u * kThreads : m0;   // (its own: the lists may lie where the results go)
            t[u] = to[m];
            f[u] = of[m];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            w[u] = weight[f[u]];
            p[u] = pos[f[u]];
            row_t[u] = (int32_t)a.pages.row(s, t[u]);
            row_f[u] = (int32_t)a.pages.row(s, f[u]);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int m = m0 + u * kThreads;
            if (m >= n) break;
            new_weight[t[u]] = w[u];
            new_pos[t[u]] = p[u];
            list_to[m] = row_t[u];
            list_of[m] = row_f[u];
        }
    }
}

// 16 lanes have a row (16 bytes a lane), kMovesOnce rows in flight
__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(const EvictKv a, const int32_t* __restrict__ moves, int64_t moves_ld) {
    const int s = blockIdx.z, hk = blockIdx.y, lane = threadIdx.x & 15;
    pdl_wait();
    pdl_trigger();
    const int32_t* list = moves + ((size_t)s * a.Hkv + hk) * moves_ld;
    const int n = list[0], step = gridDim.x * (kMoveThreads / 16);
    const int32_t* to = list + kMovesAhead;
    const int32_t* of = to + (moves_ld - kMovesAhead) / 2;
    uint4* k = reinterpret_cast<uint4*>(a.k_cache);
    uint4* v = reinterpret_cast<uint4*>(a.v_cache);
    for (int m = blockIdx.x * (kMoveThreads / 16) + (threadIdx.x >> 4); m < n; m += kMovesOnce * step) {
        size_t at[kMovesOnce];
        uint4 x[kMovesOnce], y[kMovesOnce];
#pragma unroll
        for (int u = 0; u < kMovesOnce; ++u)
            if (m + u * step < n) {
                const size_t from = ((size_t)of[m + u * step] * a.Hkv + hk) * (kHeadDim / 8) + lane;
                at[u] = ((size_t)to[m + u * step] * a.Hkv + hk) * (kHeadDim / 8) + lane;
                x[u] = k[from];
                y[u] = v[from];
            }
#pragma unroll
        for (int u = 0; u < kMovesOnce; ++u)
            if (m + u * step < n) {
                k[at[u]] = x[u];
                v[at[u]] = y[u];
            }
    }
}

cudaError_t launch_evict_kv(goose_ctx* c, const EvictKv& a, cudaStream_t st) {
    if (a.S == 0) return cudaSuccess;
    const int64_t room = a.pages.room(a.ldw);
    int64_t most = room - a.budget < a.budget ? room - a.budget : a.budget;   // rows of a head that can change places
    if (most < 0) most = 0;
    const int64_t ld = kMovesAhead + 2 * most;
    if (cudaError_t e = grow(c, &c->evict_moves, &c->evict_bytes, sizeof(int32_t) * (size_t)ld * a.S * a.Hkv)) return e;
    int32_t* moves = static_cast<int32_t*>(c->evict_moves);
    const int keep_words = (int)((room + 31) / 32) + 1, keys_there = std::min({(int)room, kMostKeys, kSelectSmem / 4 - 2 * keep_words});
    const size_t smem = sizeof(uint32_t) * (size_t)(2 * keep_words + keys_there);
    // Of more heads than SMs smaller blocks, two or four an SM where their shared memory allows it, so that one's trips to L2 go beside another's work (512 heads of 2500
    // rows to 2048: 72 us, two 63, four 59; of 517 to 500 33, 22, 19; 320 of 4200 to 4096 46, 40, 40).  Fewer heads want all threads (128 heads of 3500 to 9000 rows 45, 51, 65).
    auto fits = [&](int blocks) { return (size_t)blocks * (smem + kSelectStatic) <= (size_t)kSmemOfAnSm; };
    const int64_t heads = (int64_t)a.S * a.Hkv;
    auto select = heads > 2 * c->num_sms && fits(4) ? evict_select_kernel<256> : heads > c->num_sms && fits(2) ? evict_select_kernel<512> : evict_select_kernel<1024>;
    const int threads = select == evict_select_kernel<256> ? 256 : select == evict_select_kernel<512> ? 512 : 1024;
    cudaError_t e = launch_pdl(select, dim3(a.Hkv, a.S), dim3(threads), smem, st, a, moves, ld, keep_words, keys_there, c->status);
    c->launches++;
    if (e != cudaSuccess || most == 0) return e;
    // blocks of a head: one for every batch of rows that can move, but few of them beyond two rounds of what the SMs hold, since most heads move fewer (always 64: 512 heads of
    // 2500 rows to 2048 60 us, these 57; 128 heads 45 and 43; one round 58, 46)
    const int64_t rows = kMovesOnce * kMoveThreads / 16;
    const int64_t blocks = std::min({(most + rows - 1) / rows, (int64_t)64, (2 * 8 * c->num_sms + heads - 1) / heads});
    e = launch_pdl(evict_move_kernel, dim3((unsigned)blocks, a.Hkv, a.S), dim3(kMoveThreads), 0, st, a, moves, ld);
    c->launches++;
    return e;
}

cudaError_t init_evict_kernels() {
    cudaError_t e = cudaSuccess;
    for (auto select : {evict_select_kernel<1024>, evict_select_kernel<512>, evict_select_kernel<256>})
        if (e == cudaSuccess) e = cudaFuncSetAttribute(select, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelectSmem);
    return e == cudaSuccess ? load_kernels({(const void*)evict_move_kernel}) : e;
}

}  // namespace goose
