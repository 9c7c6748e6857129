// Work partition of the attention of chunks over pages.  It compiles for the host too, where a test walks it.
//
// The work list is a row of items, sequence by sequence, key/value head by head: each a pair of M tiles (t tokens with the heads of a group, 128 query
// rows; a chunk's last item may be a single one) over the 128-key tiles that its last token sees.  The list is laid out in places, as many as an item costs
// (a tile's, and those of the change to it), and dealt to the CTAs in ranges of equal length: a tile is of the range that its first place is in.
// Int holds places: 32 bits where the host can tell that all of them fit (64-bit divisions and products are slow on the GPU, and every CTA does a few dozen
// ahead of its first load).  What a CTA does of an item is a segment.  An item that one CTA has alone is written out by it; the segments of any other leave a partial result each.
#pragma once

#include "goose_internal.cuh"

namespace goose {

constexpr int kChunkTile = 128;                  // keys of a tile, rows of an M tile
// so many places fit 32 bits, sums of a few included (64 bits wherever that is so too: one token behind 511 rows 13.2 us instead of 12.5, drafts of 8 tokens, 40 heads, 145 instead of 143)
constexpr double kShortPlaces = 1 << 30;
// places of a key, and of the change to another item, for items of which some are pairs and for single M tiles.  Short lists have the changes too, although they leave
// CTAs idle: fewer parts of an item to join (60 tokens behind 500, 32 heads over 8: 24 us, without them 41; one token behind 511 rows 10.8 and 12.5).  A change of single tiles as 4, 6
// and 8 x 128 places: 16 drafts of up to 17 tokens, 40 heads 144, 140, 140 us; 32 sequences of a token, 40 heads 155, 151, 148; 64, 32 over 8 235, 235.5, 237.
constexpr int kPairKey = 5, kSingleKey = 4, kPairChange = 16 * kChunkTile, kSingleChange = 6 * kChunkTile;

template <typename Int>
struct ChunkSeq {             // a sequence's part of the list
    int n, ctx, step, pairs;  // new tokens, rows in front of them, tokens of an item, items a key/value head
    int key, change;
    bool bad;                 // its rows do not fit its part of the table: it counts as one without a prefix
    // places of item p, of the items in front of it
    __host__ __device__ __forceinline__ Int width(int p) const { return (Int)key * (ctx + (Int)(p + 1) * step) + change; }
    __host__ __device__ __forceinline__ Int before(int p) const {
        return (Int)p * ((Int)key * ctx + change) + (Int)key * step * ((Int)p * (p + 1) / 2);
    }
    __host__ __device__ __forceinline__ int keys(int p) const { const int left = n - p * step; return ctx + p * step + (left < step ? left : step); }
    __host__ __device__ __forceinline__ int tiles(int p) const { return (int)(((uint32_t)keys(p) + kChunkTile - 1) / kChunkTile); }
    // of T tiles of an item that begins at place w0, those whose first place is in front of place w
    __host__ __device__ __forceinline__ int cut(Int w0, int T, Int w) const {
        const Int x = w - w0 - change;
        if (x <= 0) return 0;
        const Int pitch = key * kChunkTile;
        if (x >= T * pitch) return T;
        return (int)(key == kPairKey ? (x + (kPairKey * kChunkTile - 1)) / (kPairKey * kChunkTile) : (x + (kSingleKey * kChunkTile - 1)) / (kSingleKey * kChunkTile));
    }
};

template <typename Int>
struct ChunkWork {
    const int32_t *ctx_len, *n_new;
    int S, B, Hkv, G;         // G: CTAs
    int t;                    // tokens of an M tile
    int room;                 // rows that a sequence may have
    // worked out
    Int total, quantum;

    __host__ __device__ __forceinline__ ChunkSeq<Int> seq(int s) const {
        ChunkSeq<Int> q;
        q.n = nodes_of(n_new, s, B);
        const int ctx = ctx_len[s];
        q.bad = rows_outside(0, ctx, q.n, room);
        q.ctx = q.bad ? 0 : ctx;
        q.step = q.n > 2 * t ? 2 * t : q.n;
        q.pairs = q.n > q.step ? (q.n + q.step - 1) / q.step : q.n > 0;
        q.key = q.n > t ? kPairKey : kSingleKey;
        q.change = q.n > t ? kPairChange : kSingleChange;
        return q;
    }
    // a bound of all places, whatever the lengths are
    static __host__ double most(int S, int B, int Hkv, int t, int room) {
        const double pairs = B > t ? (B + 2.0 * t - 1) / (2.0 * t) + 1 : 1;
        return (double)S * Hkv * pairs * (kPairKey * (room + t * pairs + 2.0 * t) + kPairChange);
    }
    // sum: places of one key/value head of all sequences;  several: there are pairs
    __host__ __device__ __forceinline__ void set(Int sum, bool several) {
        const Int tile = (several ? kPairKey : kSingleKey) * kChunkTile;
        total = Hkv * sum;
        quantum = total > 0 ? (total + G - 1) / G : 1;
        if (quantum < tile) quantum = tile;      // every CTA between an item's first and its last one then has a tile of it
    }
    static __host__ __device__ __forceinline__ Int divide(Int a, Int b) {
        return sizeof(Int) == 4 || ((a | b) >> 31 >> 1) == 0 ? (Int)((uint32_t)a / (uint32_t)b) : a / b;
    }
    __host__ __device__ __forceinline__ Int start(int c) const { const Int w = c * quantum; return w < total ? w : total; }
};

// where a CTA is in the list: item p of head hk of sequence s, which begins at place w0
template <typename Int>
struct ChunkCursor {
    int s, hk, p;
    Int w0;
    // the segment there of CTA `cta`, whose range is [from, to): tiles t0 .. t1 - 1 of T; c0, c1: the first and the last CTA that have tiles of the item
    int t0, t1, T, c0, c1;
    __host__ __device__ __forceinline__ void look(const ChunkWork<Int>& wk, const ChunkSeq<Int>& q, int cta, Int from, Int to) {
        T = q.tiles(p);
        t0 = q.cut(w0, T, from);
        t1 = q.cut(w0, T, to);
        c0 = c1 = cta;                           // (what begins or ends here needs no division)
        const Int first = w0 + q.change;
        if (t0 > 0) c0 = (int)ChunkWork<Int>::divide(first, wk.quantum);
        if (t1 < T) c1 = (int)ChunkWork<Int>::divide(first + (Int)(T - 1) * q.key * kChunkTile, wk.quantum);
    }
    // the next item; false: the sequence has no more
    __host__ __device__ __forceinline__ bool next(const ChunkWork<Int>& wk, const ChunkSeq<Int>& q) {
        w0 += q.width(p);
        if (++p < q.pairs) return true;
        p = 0;
        return ++hk < wk.Hkv;
    }
    // to the item of the sequence that begins at place `begin` which has place w
    __host__ __device__ __forceinline__ void enter(const ChunkSeq<Int>& q, Int begin, Int w) {
        const Int of_head = q.before(q.pairs);
        hk = (int)ChunkWork<Int>::divide(w - begin, of_head);
        const Int rem = w - begin - hk * of_head;
        int lo = 0, hi = q.pairs;                // the last item that begins at rem or in front of it
        while (hi - lo > 1) {
            const int mid = lo + (hi - lo) / 2;
            if (q.before(mid) <= rem) lo = mid; else hi = mid;
        }
        p = lo;
        w0 = begin + hk * of_head + q.before(p);
    }
};

}  // namespace goose
