// Work partition of goose_kv_weights.  It compiles for the host too, where a test walks it.
//
// The work list is a row of items, sequence by sequence, key/value head by head: each a run of up to four 128-key tiles with all Q tiles (t tokens with
// the heads of a group, 128 query rows) that see any of its keys.  The list is laid out in places, as many as an item costs, and dealt to the CTAs in
// ranges of equal length: a Q tile is of the range that its first place is in.  Int holds places: 32 bits where the host can tell that all of them
// fit.  What a CTA does of an item is a segment.
#pragma once

#include "goose_internal.cuh"

namespace goose {

constexpr int kWeightTile = 128;                 // keys of a tile, rows of a Q tile
// so many places fit 32 bits, sums of a few included (64 bits wherever that is so too: one token behind 511 rows 8.7 us instead of 8.1, 17 tokens behind 3000 10.7 instead of 10.0)
constexpr double kShortWeightPlaces = 1 << 30;
// key tiles of an item, at most; short lists have runs too (16 sequences of a token: 37.8 us, runs of two 42.6, none 65; a token behind 6000 rows 10, 11, 11.5)
constexpr int kRun = 4;

template <typename Int>
struct WeightWork;

template <typename Int>
struct WeightSeq {            // a sequence's part of the list
    int n, ctx, t;            // new tokens, rows in front of them, tokens of a Q tile
    int items;                // of a key/value head
    int change;               // places of the change to an item
    bool bad;                 // its rows do not fit: nothing of it is done
    static __host__ __device__ __forceinline__ int span() { return kRun * kWeightTile; }
    // first token that sees item k
    __host__ __device__ __forceinline__ int token(int k) const { const int i = k * span() - ctx; return i > 0 ? i : 0; }
    __host__ __device__ __forceinline__ int first(int k) const { return token(k) / t; }               // Q tile of it
    __host__ __device__ __forceinline__ int tiles(int k) const { return (n + t - 1) / t - first(k); }   // Q tiles of the item
    __host__ __device__ __forceinline__ Int width(int k) const { return change + (Int)kRun * ((Int)n + t - token(k)); }
    __host__ __device__ __forceinline__ Int before(int k) const {
        Int w = (Int)k * (change + (Int)kRun * ((Int)n + t));
        const int whole = (ctx + span() - 1) / span();       // items from here on begin behind the prefix
        if (k > whole) {
            const Int a = k, b = whole;
            w -= kRun * (span() * ((a * (a - 1) - b * (b - 1)) / 2) - (Int)ctx * (a - b));
        }
        return w;
    }
    // of T Q tiles of an item that begins at place w0, those whose first place is in front of place w
    __host__ __device__ __forceinline__ int cut(Int w0, int T, Int w) const {
        const Int x = w - w0 - change;
        if (x <= 0) return 0;
        const Int pitch = kRun * t;
        return x >= T * pitch ? T : (int)WeightWork<Int>::divide(x + pitch - 1, pitch);
    }
};

template <typename Int>
struct WeightWork {
    const int32_t *ctx_len, *n_new;
    int S, B, Hkv, G;         // G: CTAs
    int t;                    // tokens of a Q tile
    int room;                 // rows that a sequence may have
    // worked out
    Int total, quantum;

    __host__ __device__ __forceinline__ WeightSeq<Int> seq(int s) const {
        WeightSeq<Int> q;
        q.n = nodes_of(n_new, s, B);
        q.ctx = ctx_len[s];
        q.bad = q.n > 0 && rows_outside(0, q.ctx, q.n, room);
        if (q.bad) q.n = 0;
        if (q.n == 0) q.ctx = 0;
        q.t = t;
        q.items = q.n > 0 ? (q.ctx + q.n + q.span() - 1) / q.span() : 0;
        q.change = q.n > t ? kRun * t : 0;
        return q;
    }
    // sum: places of one key/value head of all sequences;  several: there is one of several Q tiles
    __host__ __device__ __forceinline__ void set(Int sum, bool several) {
        total = Hkv * sum;
        quantum = total > 0 ? (total + G - 1) / G : 1;
        // every CTA between an item's first and its last one has a Q tile of it
        if (several && quantum < kRun * t) quantum = kRun * t;
    }
    static __host__ __device__ __forceinline__ Int divide(Int a, Int b) {
        return sizeof(Int) == 4 || ((a | b) >> 31 >> 1) == 0 ? (Int)((uint32_t)a / (uint32_t)b) : a / b;
    }
    // a bound of all places, whatever the lengths are
    static __host__ double most(int S, int B, int Hkv, int t, int room) {
        const double n = B < room ? B : room, items = room / (double)kWeightTile + 2;
        return (double)S * Hkv * items * (kRun * t + kRun * (n + t));
    }
    __host__ __device__ __forceinline__ Int start(int c) const { const Int w = c * quantum; return w < total ? w : total; }
};

// where a CTA is in the list: item k of head hk of sequence s, which begins at place w0
template <typename Int>
struct WeightCursor {
    int s, hk, k;
    Int w0;
    // the segment there of CTA `cta`, whose range is [from, to): Q tiles t0 .. t1 - 1 of T; c0, c1: the first and the last CTA that have Q tiles of the item
    int t0, t1, T, c0, c1;
    __host__ __device__ __forceinline__ void look(const WeightWork<Int>& wk, const WeightSeq<Int>& q, int cta, Int from, Int to) {
        T = q.tiles(k);
        t0 = q.cut(w0, T, from);
        t1 = q.cut(w0, T, to);
        c0 = c1 = cta;                           // (what begins or ends here needs no division)
        const Int first = w0 + q.change;
        if (t0 > 0) c0 = (int)WeightWork<Int>::divide(first, wk.quantum);
        if (t1 < T) c1 = (int)WeightWork<Int>::divide(first + (Int)(T - 1) * kRun * q.t, wk.quantum);
    }
    // the next item; false: the sequence has no more
    __host__ __device__ __forceinline__ bool next(const WeightWork<Int>& wk, const WeightSeq<Int>& q) {
        w0 += q.width(k);
        if (++k < q.items) return true;
        k = 0;
        return ++hk < wk.Hkv;
    }
    // to the item of the sequence that begins at place `begin` which has place w
    __host__ __device__ __forceinline__ void enter(const WeightSeq<Int>& q, Int begin, Int w) {
        const Int of_head = q.before(q.items);
        hk = (int)WeightWork<Int>::divide(w - begin, of_head);
        const Int rem = w - begin - hk * of_head;
        int lo = 0, hi = q.items;                // the last item that begins at rem or in front of it
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (q.before(mid) <= rem) lo = mid; else hi = mid;
        }
        k = lo;
        w0 = begin + hk * of_head + q.before(k);
    }
};

}  // namespace goose
