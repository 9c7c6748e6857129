// Work partition of the shared-prefix attention: the same arithmetic for its main kernel and for the merge behind it.  It compiles for
// the host too, where a test walks it.
//
// The work list is a row of items, each a run of 128-key tiles: first, head by head, the pairs of M tiles of the whole batch over the shared
// rows, then, sequence by sequence and head by head, the pairs of M tiles of one sequence over its own rows.  A tile takes as many places as
// it costs, and the list is dealt to the CTAs in ranges of equal length: a tile is of the range that its first place is in.  What a CTA does of
// one item is a segment.  A segment has two lanes, each with a softmax warpgroup and
// accumulators of its own: the two M tiles of the pair, which share the key tiles, or, where an item is a single M tile, every other
// key tile of it.  Every lane of a segment leaves a partial result.
#pragma once

#include "goose_internal.cuh"

namespace goose {

constexpr int kSharedTile = 128;                 // keys of a tile, rows of an M tile
// places of a key tile, and of the change to another item, for a pair of M tiles and for a single one.  (Changes of 10 and 4, 16 and 2 or 16
// and 3 instead: 26 x 52 heads, 32 nodes, 128 shared rows 59.7 -> 59.1, 63.5, 62.9 us; 16 x 32 heads, 16 nodes, 1500 shared rows 61.3 -> 63.7, 59.4, 60.7;
// 8 x 52 heads, 128 nodes, 5423 shared rows 183 -> 185, 192, 189.)
constexpr int kPairPlaces = 5, kSinglePlaces = 4, kPairChange = 16, kSingleChange = 4;

constexpr int kPartWords = 25;                   // words of 16 bytes a row of a partial result
constexpr uint32_t kPartBlock = kPartWords * kSharedTile;

struct SharedWork {
    const int32_t* ctx_len;
    const int32_t* n_nodes;   // or NULL
    int S, B, Hkv, kv_rows;
    int shared_tiles;         // tiles of the shared rows
    int shared_m, own_m;      // M tiles a key/value head: of the whole batch; of one sequence
    int G;                    // CTAs
    // places of the partial results, see lay()
    int shared_log2, own_log2, cta_log2, own_slot, cta_slot;
    uint32_t own_place, cta_place;
    // worked out
    bool changes;             // do changes count?  (not in lists of a tile or two a CTA)
    long long shared_total, total, quantum;

    __host__ __device__ __forceinline__ int shared_pairs() const { return (shared_m + 1) >> 1; }
    __host__ __device__ __forceinline__ int own_pairs() const { return (own_m + 1) >> 1; }
    // a negative length counts as 0, one beyond the cache as the whole cache: such a sequence is flagged, and the list stays one that every
    // division below is right for
    __host__ __device__ __forceinline__ int prefix(int ctx) const {
        const int c = ctx < 0 ? 0 : ctx;
        return c < kv_rows ? c : kv_rows;
    }
    __host__ __device__ __forceinline__ int tiles(int s) const {
        const int ctx = prefix(ctx_len[s]), nn = nodes_of(n_nodes, s, B);
        return nn == 0 ? 0 : (int)(((uint32_t)ctx + (uint32_t)nn + kSharedTile - 1) / kSharedTile);
    }
    // places of a tile of the shared rows (s < 0), of a sequence's own; of an item of T tiles (its region's items count alike)
    __host__ __device__ __forceinline__ int places(int s) const { return (s < 0 ? shared_m : own_m) > 1 ? kPairPlaces : kSinglePlaces; }
    __host__ __device__ __forceinline__ int change(int s) const { return !changes ? 0 : (s < 0 ? shared_m : own_m) > 1 ? kPairChange : kSingleChange; }
    __host__ __device__ __forceinline__ int width(int s, int T) const { return T > 0 ? T * places(s) + change(s) : 0; }
    // sum: tiles of a head of all sequences;  live: sequences that have any
    __host__ __device__ __forceinline__ void set(long long sum, int live) {
        const long long all = (long long)Hkv * shared_pairs() * shared_tiles + (long long)Hkv * own_pairs() * sum;
        changes = all >= 2ll * G;
        shared_total = (long long)Hkv * shared_pairs() * width(-1, shared_tiles);
        total = shared_total + (long long)Hkv * own_pairs() * (sum * places(0) + (long long)change(0) * live);
        quantum = total > 0 ? divide(total + G - 1, G) : 1;
    }
    static __host__ __device__ __forceinline__ long long divide(long long a, long long b) {   // 64-bit division is slow on the GPU
        return (a | b) >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
    }
    __host__ __device__ __forceinline__ long long start(int c) const { return min(c * quantum, total); }
    __host__ __device__ __forceinline__ int cta_of(long long w) const { return (int)divide(w, quantum); }
    __host__ __device__ __forceinline__ int shared_items() const { return shared_tiles > 0 ? Hkv * shared_pairs() : 0; }
    __host__ __device__ __forceinline__ int items() const { return shared_items() + S * Hkv * own_pairs(); }
    __host__ __device__ __forceinline__ int item(int s, int i) const {    // s < 0: the shared rows;  i = head * pairs + pair
        return s < 0 ? i : shared_items() + s * Hkv * own_pairs() + i;
    }
    // Where the partial result of a lane lies.  A segment that is a whole item has the item's place; of any other a CTA has at most one
    // that does not start its item (its first) and one that does (its last).
    __host__ __device__ __forceinline__ int slot(int item, int cta, bool from_start, bool to_end, int lane) const {
        return from_start && to_end ? 2 * item + lane : 2 * items() + 4 * cta + (from_start ? 2 : 0) + lane;
    }
    __host__ __device__ __forceinline__ int slots() const { return 2 * items() + 4 * G; }
    // Where a slot's row 0 lies in the workspace, in words of 16 bytes.  The workspace is made of blocks of 128 rows, kPartWords words a row that lie
    // 128 words apart; slots of M tiles that never have that many rows share a block.
    __host__ __device__ __forceinline__ uint32_t place(int slot) const {
        if (slot < own_slot) return shared_at(slot, shared_log2);
        return slot < cta_slot ? own_place + shared_at(slot - own_slot, own_log2) : cta_place + shared_at(slot - cta_slot, cta_log2);
    }
    static __host__ __device__ __forceinline__ uint32_t shared_at(uint32_t i, int log2) {   // the i-th slot where 2^log2 share a block
        return (i >> log2) * kPartBlock + ((i & ((1u << log2) - 1)) << (7 - log2));
    }
    // lays the slots out for M tiles of at most so many rows (of the batch, of one sequence); returns all blocks
    __host__ long long lay(int of_batch, int of_sequence) {
        auto share = [](int rows) {                          // at least 4 rows: whole sectors
            int l = 0;
            while (l < 5 && 2 * rows << l <= kSharedTile) ++l;
            return l;
        };
        auto blocks = [](long long slots, int l) { return (slots + (1 << l) - 1) >> l; };
        shared_log2 = share(of_batch); own_log2 = share(of_sequence);
        cta_log2 = shared_tiles > 0 ? min(shared_log2, own_log2) : own_log2;   // (a CTA's segment may be of either kind)
        own_slot = 2 * shared_items(); cta_slot = 2 * items();
        const long long own = blocks(own_slot, shared_log2), cta = own + blocks(cta_slot - own_slot, own_log2);
        own_place = (uint32_t)own * kPartBlock; cta_place = (uint32_t)cta * kPartBlock;
        return cta + blocks(4ll * G, cta_log2);
    }
};

struct SharedCursor {         // walks the list
    long long w;              // place in it
    int s, i, t, T;           // sequence or -1, item of it (head * pairs + pair), tile, tiles
    // at place `rem` of the items that begin here, or at the next tile behind it
    __host__ __device__ __forceinline__ void enter(const SharedWork& wk, long long rem) {
        const int wd = wk.width(s, T), u = wk.places(s);
        i = (int)SharedWork::divide(rem, wd);
        const int at = (int)(rem - (long long)i * wd) - wk.change(s);
        t = at > 0 ? (at + u - 1) / u : 0;
        w += t * u - at;
        if (t == T) next(wk);
    }
    // tiles from here on that are of a range which ends at w_end
    __host__ __device__ __forceinline__ int run(const SharedWork& wk, long long w_end) const {
        const int u = wk.places(s);
        const long long n = SharedWork::divide(w_end - w + u - 1, u);
        return n < T - t ? (int)n : T - t;
    }
    // the next item's first tile
    __host__ __device__ __forceinline__ void next(const SharedWork& wk) {
        t = 0; ++i;
        if (i == wk.Hkv * (s < 0 ? wk.shared_pairs() : wk.own_pairs())) {
            i = 0;
            do { ++s; } while (s < wk.S && (T = wk.tiles(s)) == 0);
        }
        w += wk.change(s);
    }
    __host__ __device__ __forceinline__ void skip(const SharedWork& wk, int n) {
        w += n * wk.places(s); t += n;
        if (t == T) next(wk);
    }
};

// the partial results of one M tile of an item, in the order of the keys
struct SharedParts {
    long long w0;             // place of the item's first tile
    int T, u, item, c0, n, lanes, lane;
    // first: the item's first place.  single: the item is one M tile (two lanes of key tiles); else `m` says which of the two
    __host__ __device__ __forceinline__ void set(const SharedWork& wk, int s, int i, long long first, int tiles, bool single, int m) {
        w0 = first + wk.change(s); T = tiles; u = wk.places(s); item = wk.item(s, i);
        lanes = single ? 2 : 1; lane = single ? 0 : m;
        if (T > 0) { c0 = wk.cta_of(w0); n = (wk.cta_of(w0 + (long long)(T - 1) * u) - c0 + 1) * lanes; }
        else { c0 = 0; n = 0; }
    }
    // slot of part k, or -1: that CTA has nothing of the item for the lane
    __host__ __device__ __forceinline__ int slot(const SharedWork& wk, int k) const {
        const int c = c0 + (lanes == 2 ? k >> 1 : k), l = lanes == 2 ? k & 1 : lane;
        const long long a = c * wk.quantum - w0, b = a + wk.quantum, all = (long long)T * u;
        const int ta = a > 0 ? (int)SharedWork::divide(a + u - 1, u) : 0, tb = (int)SharedWork::divide((b < all ? b : all) + u - 1, u);
        return tb - ta > (lanes == 2 ? l : 0) ? wk.slot(item, c, ta == 0, tb == T, l) : -1;
    }
};

}  // namespace goose
