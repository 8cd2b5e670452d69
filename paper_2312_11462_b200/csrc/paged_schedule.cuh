// How the attention over the paged cache divides its work: units are (sequence, row block, kv head, key tile), in this order, and
// a CTA takes an equal run of them whatever the sequences' lengths are.  A run that begins or ends inside an item (all but
// its key tile) leaves its part of the item in the workspace, and the CTA that arrives last adds the parts up, in their order.
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
    unsigned* tickets;           // [CTAs]
    float* parts;                // [CTAs][2] parts
};

template <int BR, int KEYS> struct Schedule {
    // Positions that the rows of block rb see at most.  (rows * group fits 30 bits: check_attend)
    static __device__ __forceinline__ int seen(const PagedView& w, const PagedSeq& q, int rb, int group, bool tree) {
        const int last = tree ? q.rows : min(q.rows, (int)(((unsigned)(rb + 1) * BR - 1) / (unsigned)group) + 1);
        return min(q.kv + last, w.capacity);
    }
    static __device__ __forceinline__ int blocks(const PagedSeq& q, int group) { return (q.rows * group + BR - 1) / BR; }
    static __device__ __forceinline__ unsigned tiles_of(const PagedView& w, const PagedSeq& q, int rb, int group, bool tree) {
        return (unsigned)(seen(w, q, rb, group, tree) + KEYS - 1) / KEYS;
    }

    // prefix[s]: units before sequence s, prefix[n_seqs]: all of them.  THREADS threads; ends with a barrier.
    template <int THREADS>
    static __device__ void count(const PagedView& w, int group, bool tree, u64* prefix) {
        __shared__ u64 warp_sums[THREADS / 32];
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        u64 before = 0;
        for (int s0 = 0; s0 < w.n_seqs; s0 += THREADS) {
            const int s = s0 + tid;
            PagedSeq q = {0, 0, 0};
            if (s < w.n_seqs) q = paged_seq(w, s);
            const int nb = blocks(q, group);
            u64 n = nb > 0 ? tiles_of(w, q, 0, group, tree) : 0u;
            // sequences of several blocks, a lane a block
            for (unsigned many = __ballot_sync(0xffffffffu, nb > 1); many; many &= many - 1) {
                const int j = __ffs(many) - 1;
                const PagedSeq o = {0, __shfl_sync(0xffffffffu, q.rows, j), __shfl_sync(0xffffffffu, q.kv, j)};
                const int all = __shfl_sync(0xffffffffu, nb, j);
                u64 sum = 0;
                for (int rb = 1 + lane; rb < all; rb += 32) sum += tiles_of(w, o, rb, group, tree);
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

        __device__ __forceinline__ void block(const PagedView& w, int group, bool tree) {
            seen = Schedule::seen(w, q, rb, group, tree);
            tiles = (seen + KEYS - 1) / KEYS;
        }
        // unit < prefix[n_seqs]; whole warps
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
                    const u64 n = b0 + lane < nb ? (u64)tiles_of(w, q, b0 + lane, group, tree) * w.heads : 0;
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
            h = (int)((unsigned)(unit - at) / (unsigned)tiles);
            if ((unit - at) >> 32) h = (int)((unit - at) / (u64)tiles);
            item_first = at + (u64)h * tiles;
            tile = (int)(unit - item_first);
        }
        // to the next unit; there has to be one
        __device__ __forceinline__ void next(const PagedView& w, int group, bool tree) {
            if (++tile < tiles) return;
            item_first += tiles;
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

    // What CTA c of n takes: units [begin, end), with `at` at begin.  An equal share, but that a cut within `snap` tiles of an item's
    // end moves there: a part costs its writing, its adding up and another start.  False: nothing is left for this CTA.
    static __device__ bool run(const PagedView& w, const u64* prefix, int c, unsigned n, int snap, int group, bool tree, u64* begin, u64* end, Cursor* at) {
        const u64 units = prefix[w.n_seqs];
        const bool one = w.max_rows * group <= BR;       // one block a sequence: its items are alike
        auto cut = [&](int i) {
            const u64 raw = (u64)i * units / n;
            if (raw == 0 || raw >= units) return raw;
            int tile, tiles;
            if (one) {
                int lo = 0, hi = w.n_seqs - 1;
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (prefix[mid] <= raw) lo = mid; else hi = mid - 1;
                }
                const unsigned all = (unsigned)(prefix[lo + 1] - prefix[lo]);        // (a sequence has fewer than 2^30 / KEYS tiles a head)
                tiles = (int)(all / (unsigned)w.heads);
                tile = (int)((unsigned)(raw - prefix[lo]) % (unsigned)tiles);
            } else {
                at->seek(w, prefix, raw, group, tree);
                tile = at->tile; tiles = at->tiles;
            }
            if (tile <= min(snap, tiles / 2)) return raw - tile;
            return tiles - tile <= snap ? raw - tile + tiles : raw;
        };
        *end = cut(c + 1);
        *begin = cut(c);
        if (*begin >= *end) return false;
        at->seek(w, prefix, *begin, group, tree);
        return true;
    }
    // The first and the last CTA that have a part of an item.
    static __device__ __forceinline__ void parts_of(const Cursor& at, u64 units, unsigned n, int snap, int* c0, int* c1) {
        auto last = [&](u64 unit) { return (int)(((unit + 1) * n - 1) / units); };      // the last CTA whose equal share begins at or before a unit
        const u64 front = at.item_first + min(snap, at.tiles / 2), back = at.item_first + max(at.tiles - snap - 1, 0);
        *c0 = last(front);
        *c1 = last(front > back ? front : back);
    }
};

}  // namespace csd
