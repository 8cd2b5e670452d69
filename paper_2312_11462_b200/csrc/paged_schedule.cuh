// How the attention over the paged cache divides its work.  An item is a (sequence, row block, kv head); it takes OVER units of time,
// for its queries and for its rows on their way out, and one for each of its key tiles.  The items' units lie one behind the other in the
// order of the indices, and a CTA takes an equal run of them whatever the sequences' lengths are.  (Eight sequences of 77 to 2048
// positions, trees of 12 rows, 32 heads, with tiles alone counted: 56 us, 37 where the lengths are even.)  A run that begins or ends inside an item
// leaves its part of the item in the workspace, and the parts are added up in the order of the runs: by the CTA that arrives last (few rows), or by a
// kernel behind this one (chunks).
// A row of a row block is a (new row, query head of the group) pair: row p of the sequence's rows * group.
#pragma once
#include "paged.cuh"

namespace csd {

typedef unsigned long long u64;

struct AttendArgs {
    const void* q; void* out; const u64* tree;
    long long ldq, ldo;
    int group;                   // query heads a kv head
    float scale;
    RopeView rope;               // (fp32 rows alone)
    unsigned* tickets;           // [CTAs]; behind them a chunk's joins
    float* parts;                // [CTAs][2] parts
};

template <int BR, int KEYS, int OVER> struct Schedule {
    // Positions that the rows of block rb see at most.  (rows * group fits 30 bits: check_attend)
    static __device__ __forceinline__ int seen(const PagedView& w, const PagedSeq& q, int rb, int group, bool tree) {
        const int last = tree ? q.rows : min(q.rows, (int)(((unsigned)(rb + 1) * BR - 1) / (unsigned)group) + 1);
        return min(q.kv + last, w.capacity);
    }
    static __device__ __forceinline__ int blocks(const PagedSeq& q, int group) { return (q.rows * group + BR - 1) / BR; }
    static __device__ __forceinline__ unsigned tiles_of(const PagedView& w, const PagedSeq& q, int rb, int group, bool tree) {
        return (unsigned)(seen(w, q, rb, group, tree) + KEYS - 1) / KEYS;
    }

    // prefix[s]: units before sequence s, prefix[n_seqs]: all of them; with `items` the same of items, and in *longest the longest item's units.
    // THREADS threads; ends with a barrier.
    template <int THREADS>
    static __device__ void count(const PagedView& w, int group, bool tree, u64* prefix, u64* items = nullptr, int* longest = nullptr) {
        __shared__ u64 warp_sums[THREADS / 32];
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        if (items) {
            u64 n = 0;
            int most = 0;
            for (int s = lane; warp == 0 && s < ((w.n_seqs + 31) & ~31); s += 32) {
                PagedSeq q = {0, 0, 0};
                if (s < w.n_seqs) q = paged_seq(w, s);
                const int nb = blocks(q, group);
                if (nb > 0) most = max(most, (int)tiles_of(w, q, nb - 1, group, tree) + OVER);
                u64 x = (u64)nb * w.heads;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 y = __shfl_up_sync(0xffffffffu, x, o);
                    if (lane >= o) x += y;
                }
                if (s < w.n_seqs) items[s + 1] = n + x;
                n += __shfl_sync(0xffffffffu, x, 31);
            }
            most = __reduce_max_sync(0xffffffffu, most);
            if (tid == 0) { items[0] = 0; *longest = most; }
        }
        u64 before = 0;
        for (int s0 = 0; s0 < w.n_seqs; s0 += THREADS) {
            const int s = s0 + tid;
            PagedSeq q = {0, 0, 0};
            if (s < w.n_seqs) q = paged_seq(w, s);
            const int nb = blocks(q, group);
            u64 n = nb > 0 ? tiles_of(w, q, 0, group, tree) + OVER : 0u;
            // sequences of several blocks, a lane a block
            for (unsigned many = __ballot_sync(0xffffffffu, nb > 1); many; many &= many - 1) {
                const int j = __ffs(many) - 1;
                const PagedSeq o = {0, __shfl_sync(0xffffffffu, q.rows, j), __shfl_sync(0xffffffffu, q.kv, j)};
                const int all = __shfl_sync(0xffffffffu, nb, j);
                u64 sum = 0;
                for (int rb = 1 + lane; rb < all; rb += 32) sum += tiles_of(w, o, rb, group, tree) + OVER;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                if (lane == j) n += sum;
            }
            u64 x = n * w.heads;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            if (lane == 31) warp_sums[warp] = x;
            __syncthreads();
            u64 base = before, all = 0;
            for (int i = 0; i < THREADS / 32; ++i) {
                if (i < warp) base += warp_sums[i];
                all += warp_sums[i];
            }
            if (s < w.n_seqs) prefix[s + 1] = base + x;
            before += all;
            __syncthreads();
        }
        if (tid == 0) prefix[0] = 0;
        __syncthreads();
    }

    // A place in the order of units, and what belongs to its item.
    struct Cursor {
        u64 item_first;          // first unit of the item
        PagedSeq q;
        int s, rb, h, tile, tiles, seen;

        __device__ __forceinline__ u64 unit_of(int t) const { return item_first + OVER + t; }      // of a tile
        __device__ __forceinline__ u64 item_end() const { return unit_of(tiles); }
        // the item's tiles in front of a run's end
        __device__ __forceinline__ int tiles_before(u64 end) const { return item_end() <= end ? tiles : (int)(end - unit_of(0)); }

        __device__ __forceinline__ void block(const PagedView& w, int group, bool tree) {
            seen = Schedule::seen(w, q, rb, group, tree);
            tiles = (seen + KEYS - 1) / KEYS;
        }
        // to the item of a unit < prefix[n_seqs], and the tile there (the first, in front of it); whole warps
        __device__ void seek(const PagedView& w, const u64* prefix, u64 unit, int group, bool tree) {
            const int lane = threadIdx.x & 31;
            int lo = 0, hi = w.n_seqs - 1;               // the last s with prefix[s] <= unit
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (prefix[mid] <= unit) lo = mid; else hi = mid - 1;
            }
            s = lo;
            q = paged_seq(w, s);
            const int nb = blocks(q, group);
            u64 at = prefix[s];
            rb = 0;
            if (nb > 1)
                for (int b0 = 0;; b0 += 32) {            // a lane a block
                    const u64 n = b0 + lane < nb ? (u64)(tiles_of(w, q, b0 + lane, group, tree) + OVER) * w.heads : 0;
                    u64 x = n;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const u64 y = __shfl_up_sync(0xffffffffu, x, o);
                        if (lane >= o) x += y;
                    }
                    const unsigned past = __ballot_sync(0xffffffffu, b0 + lane < nb && unit >= at + x);
                    const int k = __popc(past);          // blocks that end at or before the unit
                    at += k ? __shfl_sync(0xffffffffu, x, k - 1) : 0;
                    rb = b0 + k;
                    if (k < 32) break;
                }
            block(w, group, tree);
            h = (int)((unsigned)(unit - at) / (unsigned)(tiles + OVER));         // (a block's units fit 32 bits: check_attend)
            item_first = at + (u64)h * (tiles + OVER);
            tile = max((int)(unit - item_first) - OVER, 0);
        }
        // to the next tile; there has to be one
        __device__ __forceinline__ void next(const PagedView& w, int group, bool tree) {
            if (++tile < tiles) return;
            item_first = item_end();
            tile = 0;
            if (++h < w.heads) return;
            h = 0;
            if (++rb >= blocks(q, group)) {
                rb = 0;
                do q = paged_seq(w, ++s); while (q.rows == 0);
            }
            block(w, group, tree);
        }
    };

    // How far a cut may move: a share of a run, two tiles at most.
    static __device__ __forceinline__ int snap_of(u64 units, unsigned n, unsigned share) { return (int)min((u64)2, units / n / share); }
    // What CTA c of n takes: units [begin, end), with `at` at its first tile.  An equal share, but that a cut in front of an item's first tile or within
    // `snap` tiles of an item's end moves there: a part costs its writing, its adding up and another start.  False: nothing is left for this CTA.
    static __device__ bool run(const PagedView& w, const u64* prefix, int c, unsigned n, int snap, int group, bool tree, u64* begin, u64* end, Cursor* at) {
        const u64 units = prefix[w.n_seqs];
        const bool one = w.max_rows * group <= BR;       // one block a sequence: its items are alike
        auto cut = [&](int i) {
            const u64 raw = (u64)i * units / n;
            if (raw == 0 || raw >= units) return raw;
            u64 first;
            int tiles;
            if (one) {
                int lo = 0, hi = w.n_seqs - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (prefix[mid] <= raw) lo = mid; else hi = mid - 1;
                }
                const unsigned each = (unsigned)(prefix[lo + 1] - prefix[lo]) / (unsigned)w.heads, in = (unsigned)(raw - prefix[lo]) % each;
                tiles = (int)each - OVER;
                first = raw - in;
            } else {
                at->seek(w, prefix, raw, group, tree);
                first = at->item_first; tiles = at->tiles;
            }
            const int tile = max((int)(raw - first) - OVER, 0);
            if (tile <= min(snap, tiles / 2)) return first;
            return tiles - tile <= snap ? first + OVER + tiles : raw;
        };
        *end = cut(c + 1);
        *begin = cut(c);
        if (*begin >= *end) return false;
        at->seek(w, prefix, *begin, group, tree);
        return true;
    }
    // Item i alone, as a run of its own.
    static __device__ void item(const PagedView& w, const u64* items, unsigned i, int group, bool tree, u64* begin, u64* end, Cursor* at) {
        int lo = 0, hi = w.n_seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (items[mid] <= i) lo = mid; else hi = mid - 1;
        }
        const unsigned in = i - (unsigned)items[lo];
        at->s = lo;
        at->q = paged_seq(w, lo);
        at->rb = (int)(in / (unsigned)w.heads);
        at->h = (int)(in % (unsigned)w.heads);
        at->block(w, group, tree);
        at->item_first = *begin = 0;
        at->tile = 0;
        *end = at->item_end();
    }
    // The first and the last CTA that have a part of an item.
    static __device__ __forceinline__ void parts_of(const Cursor& at, u64 units, unsigned n, int snap, int* c0, int* c1) {
        auto last = [&](u64 unit) { return (int)(((unit + 1) * n - 1) / units); };      // the last CTA whose equal share begins at or before a unit
        const u64 front = at.unit_of(min(snap, at.tiles / 2)), back = at.unit_of(max(at.tiles - snap - 1, 0));
        *c0 = last(front);
        *c1 = last(front > back ? front : back);
    }
};

}  // namespace csd
