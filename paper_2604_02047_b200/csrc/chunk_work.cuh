// Work partition of the attention of chunks over pages.  It compiles for the host too, where a test walks it.
//
// The work list is a row of items, sequence by sequence, key/value head by head: each a pair of M tiles (t tokens with the heads of a group, 128 query
// rows; a chunk's last item may be a single one) over the 128-key tiles that its last token sees.  The list is laid out in places, as many as an item costs
// (a tile's, and those of the change to it), and dealt to the CTAs in ranges of equal length: a tile is of the range that its first place is in.
// What a CTA does of an item is a segment.  An item that one CTA has alone is written out by it; the segments of any other leave a partial result each.
#pragma once

#include "goose_internal.cuh"

namespace goose {

constexpr int kChunkTile = 128;                  // keys of a tile, rows of an M tile
// places of a key, and of the change to another item, for items of which some are pairs and for single M tiles
constexpr int kPairKey = 5, kSingleKey = 4, kPairChange = 16 * kChunkTile, kSingleChange = 4 * kChunkTile;

struct ChunkSeq {             // a sequence's part of the list
    int n, ctx, step, pairs;  // new tokens, rows in front of them, tokens of an item, items a key/value head
    int key, change;
    bool bad;                 // its rows do not fit its part of the table: it counts as one without a prefix
    // places of item p, of the items in front of it
    __host__ __device__ __forceinline__ long long width(int p) const { return (long long)key * (ctx + (long long)(p + 1) * step) + change; }
    __host__ __device__ __forceinline__ long long before(int p) const {
        return (long long)p * ((long long)key * ctx + change) + (long long)key * step * ((long long)p * (p + 1) / 2);
    }
    __host__ __device__ __forceinline__ int keys(int p) const { const long long last = (long long)(p + 1) * step; return ctx + (last < n ? (int)last : n); }
    __host__ __device__ __forceinline__ int tiles(int p) const { return (int)(((long long)keys(p) + kChunkTile - 1) / kChunkTile); }
    // of T tiles of an item that begins at place w0, those whose first place is in front of place w
    __host__ __device__ __forceinline__ int cut(long long w0, int T, long long w) const {
        const long long x = w - w0 - change;
        if (x <= 0) return 0;
        const long long pitch = key * kChunkTile, all = (long long)T * pitch;
        return x >= all ? T : (int)((x + pitch - 1) / pitch);
    }
};

struct ChunkWork {
    const int32_t *ctx_len, *n_new;
    int S, B, Hkv, G;         // G: CTAs
    int t;                    // tokens of an M tile
    int room;                 // rows that a sequence may have
    // worked out
    bool changes;             // do changes count?  (not in lists of a tile or two a CTA)
    long long total, quantum;

    __host__ __device__ __forceinline__ ChunkSeq seq(int s) const {
        ChunkSeq q;
        q.n = nodes_of(n_new, s, B);
        const int ctx = ctx_len[s];
        q.bad = rows_outside(0, ctx, q.n, room);
        q.ctx = q.bad ? 0 : ctx;
        q.step = q.n > 2 * t ? 2 * t : q.n;
        q.pairs = q.n > 0 ? (q.n + q.step - 1) / q.step : 0;
        q.key = q.n > t ? kPairKey : kSingleKey;
        q.change = !changes ? 0 : q.n > t ? kPairChange : kSingleChange;
        return q;
    }
    // sum: places of one key/value head of all sequences, changes aside;  of_changes: those of its changes
    __host__ __device__ __forceinline__ void set(long long sum, long long of_changes) {
        const long long tile = kPairKey * kChunkTile;
        changes = sum * Hkv >= 2 * tile * G;
        total = Hkv * (sum + (changes ? of_changes : 0));
        quantum = total > 0 ? (total + G - 1) / G : 1;
        if (quantum < tile) quantum = tile;      // every CTA between an item's first and its last one then has a tile of it
    }
    static __host__ __device__ __forceinline__ long long divide(long long a, long long b) {   // 64-bit division is slow on the GPU
        return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
    }
    __host__ __device__ __forceinline__ long long start(int c) const { const long long w = c * quantum; return w < total ? w : total; }
};

// where a CTA is in the list: item p of head hk of sequence s, which begins at place w0
struct ChunkCursor {
    int s, hk, p;
    long long w0;
    // the segment there of a CTA whose range is [from, to): tiles t0 .. t1 - 1 of T; c0, c1: the first and the last CTA that have tiles of the item
    int t0, t1, T, c0, c1;
    __host__ __device__ __forceinline__ void look(const ChunkWork& wk, const ChunkSeq& q, long long from, long long to) {
        T = q.tiles(p);
        t0 = q.cut(w0, T, from);
        t1 = q.cut(w0, T, to);
        const long long first = w0 + q.change;
        c0 = (int)ChunkWork::divide(first, wk.quantum);
        c1 = (int)ChunkWork::divide(first + (long long)(T - 1) * q.key * kChunkTile, wk.quantum);
    }
    // the next item; false: the sequence has no more
    __host__ __device__ __forceinline__ bool next(const ChunkWork& wk, const ChunkSeq& q) {
        w0 += q.width(p);
        if (++p < q.pairs) return true;
        p = 0;
        return ++hk < wk.Hkv;
    }
    // to the item of the sequence that begins at place `begin` which has place w; lanes of a warp search together (on the host: one)
    __host__ __device__ __forceinline__ void enter(const ChunkSeq& q, long long begin, long long w) {
        const long long of_head = q.before(q.pairs);
        hk = (int)ChunkWork::divide(w - begin, of_head);
        const long long rem = w - begin - hk * of_head;
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
