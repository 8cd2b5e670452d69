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
    // Positions that the rows of block rb see at most.
    static __device__ __forceinline__ int seen(const PagedView& w, const PagedSeq& q, int rb, int group, bool tree) {
        const int last = tree ? q.rows : min(q.rows, (int)(((long long)(rb + 1) * BR - 1) / group) + 1);
        return min(q.kv + last, w.capacity);
    }
    static __device__ __forceinline__ int blocks(const PagedSeq& q, int group) { return (q.rows * group + BR - 1) / BR; }

    // prefix[s]: units before sequence s, prefix[n_seqs]: all of them.  THREADS threads; ends with a barrier.
    template <int THREADS>
    static __device__ void count(const PagedView& w, int group, bool tree, u64* prefix) {
        __shared__ u64 warp_sums[THREADS / 32];
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
        u64 before = 0;
        for (int s0 = 0; s0 < w.n_seqs; s0 += THREADS) {
            const int s = s0 + tid;
            u64 n = 0;
            if (s < w.n_seqs) {
                const PagedSeq q = paged_seq(w, s);
                const int nb = blocks(q, group);
                for (int rb = 0; rb < nb; ++rb) n += (unsigned)(seen(w, q, rb, group, tree) + KEYS - 1) / KEYS;
                n *= w.heads;
            }
            u64 x = n;
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
        // unit < prefix[n_seqs]
        __device__ void seek(const PagedView& w, const u64* prefix, u64 unit, int group, bool tree) {
            int lo = 0, hi = w.n_seqs - 1;               // the last s with prefix[s] <= unit
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (prefix[mid] <= unit) lo = mid; else hi = mid - 1;
            }
            s = lo;
            q = paged_seq(w, s);
            u64 at = prefix[s];
            for (rb = 0;; ++rb) {
                block(w, group, tree);
                const u64 n = (u64)tiles * w.heads;
                if (unit < at + n) break;
                at += n;
            }
            h = (int)((unit - at) / tiles);
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
};

// CTA c of n takes units [run_begin(c), run_begin(c + 1)).
__device__ __forceinline__ u64 run_begin(u64 c, u64 units, unsigned n) { return c * units / n; }
// the CTA that has a unit
__device__ __forceinline__ int run_of(u64 unit, u64 units, unsigned n) { return (int)(((unit + 1) * n - 1) / units); }

}  // namespace csd
