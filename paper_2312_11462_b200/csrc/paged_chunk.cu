// Attention over the paged cache for chunks of many bf16 rows: prompts, and the chunks of long ones.
//
// What bounds it are the products, 4 d flops a (row, key, head), and the exponentials beside them.  A CTA takes blocks of 256 (row, query head)
// pairs, two accumulator halves of 128 rows, against tiles of 128 positions, in four groups of four warps:
//   0  warp 0 requests the pages of a tile by TMA (a box a page and 64 columns; 8-bit pages and their scales as they lie, one copy
//      each); warp 1 issues tcgen05.mma, scores S = Q K^T from shared memory and output O += P V with P from tensor memory; warps 2 and 3
//      gather the block's queries
//   1  widens 8-bit tiles to bf16 (value times scale is exact there), and puts bf16 tiles of values that not every row sees in order
//   2, 3  a half of the rows each, a thread a row: running maximum, exponentials, P as bf16 over the scores' columns.  They take most of
//      the registers.
// Tensor memory (512 columns): per half the scores of a tile, 128 columns that P overwrites, and the output.  All products of a CTA are
// issued by one thread and run in order, so when the scores of tile t + 1 are there, O += P V of tile t is done.  P goes out in two parts of 64
// positions; the first one's product runs under the other's exponentials.  A running maximum is only brought up when a score is above it by 2^16
// (bf16 and fp32 have room for that), so that hardly a tile after an item's first waits for its maximum or rescales the output.
// A row is divided by the sum of its weights in fp32; the products take them in bf16, off by 2^-9 of each at most and either way (the rounded ones' sum would
// cost an unpacking a weight).
//
// An item's rows that lie in several CTAs' runs leave as parts, which paged_join_kernel adds up.  Measured: 875 to 887 TFLOP/s of bf16 pages, 755 of 8-bit ones
// (592 heads of 64 rows behind 4288 positions, 128 dimensions), bounded by a half's chain of scores, exponentials and products: with a quarter of the
// exponentials as polynomials on the multipliers it is 3 to 5 % slower, so the special-function unit is not what holds it up.
//
// What lies behind a sequence's positions may be anything, and 0 x NaN is NaN: values behind the last position are zeroed, and so
// are infinities and NaN in positions that some of the block's rows do not see; rows that see them get them added at the end.
#include "paged_attention.cuh"
#include "tc_common.cuh"

namespace csd {

constexpr int CH_KEYS = 128, CH_ROWS = 256, CH_THREADS = 512;
constexpr int JOIN_MOST = 1024;                // CTAs at most
constexpr int CH_MORE = 136, CH_FEWER = 120;     // registers of a softmax thread and of the others: 512 threads are launched with 128 each
static_assert(256 * CH_MORE + 256 * CH_FEWER <= 512 * 128, "a setmaxnreg.inc beyond the launch's registers would wait for good");
// Where every item can have a CTA of its own, it gets one, and no parts are added up, if the longest is not this many units above the even share.  (Prompt
// of 1000 rows, 32 heads, 4 above: 32.7 us, 39.3 in even shares; 16 sequences of 16 rows behind 4000 positions, 5 above: 76 and 87; 8 behind 1000, 6: 27.5
// and 29.9; 5 of 64 rows behind 1500 on 16 heads of 64, 7: 34.1 and 33.0; 256 rows behind 1000, 9: 36.3 and 29.5.)
constexpr unsigned CH_ALONE = 6;
constexpr float CH_LATE = 16.f;                 // a running maximum may lag by this power of two (bf16 and fp32 have room for it)

template <int DH, bool E4M3> struct ChunkCfg {
    static constexpr int HALVES = DH / 64;                       // 64-column halves of a row, 128 bytes each
    static constexpr int TILE_BYTES = CH_KEYS * DH * 2;          // a tile of keys or of values
    static constexpr int SLOTS = DH == 64 ? 8 : E4M3 ? 4 : 5;
    static constexpr int RAW = E4M3 ? CH_KEYS * DH + CH_KEYS : 0;        // a tile as the pool has it, and its scales
    static constexpr int RAWS = E4M3 ? 2 : 0;
    static constexpr int Q_BYTES = CH_ROWS * DH * 2;
    static constexpr int SMEM = 1024 + Q_BYTES + SLOTS * TILE_BYTES + RAWS * RAW;
    static constexpr int PART = CH_ROWS * (DH + 2);              // floats of a part: [half][column][row], maxima, sums
    static constexpr int O_COL = 256;                            // tensor memory: S0, S1 (128 columns each), O0, O1
};

// An item whose parts lie in the workspace, by the CTA that has its first one; no part is looked at where `last` is below 0.
struct alignas(32) ChunkJoin { int last, start, head, p0, rows, _[3]; };
// (the workspace: the tickets of the other kernel, joins, parts)
__host__ __device__ __forceinline__ ChunkJoin* joins_of(const AttendArgs& a) { return (ChunkJoin*)((char*)a.tickets + PAGED_TICKET_BYTES); }

struct ChunkBars {
    uint64_t full[8], free_[8], landed[8], rawfull[2], rawfree[2], qfull, qfree, sfull[2], pready[2][2], firsthalf[2], ofull[2], ofree[2];
    uint32_t tmem;
    int abort_flag, longest;
    // of the run's last eight position tiles: groups of 16 without a page; positions with values that were taken out
    unsigned lost[8], odd[8][4];
};

// operand with 64 consecutive elements (of N) per 128-byte row and K down the rows: atoms of 8 rows 1024 bytes apart along K,
// the next 64 elements `next64` bytes on
__device__ __forceinline__ uint64_t smem_desc_sw128_mn(uint32_t addr, uint32_t next64) {
    uint64_t d = smem_desc_sw128(addr);
    d &= ~((uint64_t)0x3fff << 16);
    return d | (uint64_t)(next64 >> 4) << 16;
}
// A from tensor memory
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accum) : "memory");
}
__device__ __forceinline__ void tm_ld32(uint32_t addr, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]),
                   "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]),
                   "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(addr));
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
                   "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_st16(uint32_t addr, const float (&v)[16]) {
    uint32_t u[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) u[j] = __float_as_uint(v[j]);
    tm_st16(addr, u);
}
__device__ __forceinline__ void tm_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// pairs of fp32 numbers in one register pair
__device__ __forceinline__ u64 two(float x, float y) { u64 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y)); return r; }
__device__ __forceinline__ float low(u64 x) { return __uint_as_float((unsigned)x); }
__device__ __forceinline__ float high(u64 x) { return __uint_as_float((unsigned)(x >> 32)); }
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) { u64 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ u64 add2(u64 a, u64 b) { u64 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
// four e4m3 numbers times a power of two, `up` times `rest` less the 2^120 that the exponent fields lie apart, as two words of two bf16
__device__ __forceinline__ uint2 widen4(uint32_t w, uint32_t up, uint32_t rest, bool twice) {
    w = __byte_perm(w, 0, 0x3120);                               // numbers 0, 2, 1, 3 (never an infinity or NaN as they are put together here)
    uint32_t a = ((w << 4) & 0x07f007f0u) | ((w << 8) & 0x80008000u), b = ((w >> 4) & 0x07f007f0u) | (w & 0x80008000u);
    asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(up));
    asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(b) : "r"(up));
    if (twice) {
        asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(rest));
        asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(b) : "r"(rest));
    }
    return make_uint2(a, b);
}
// 2^e as two bf16 (a field of 8 exponent bits, e + 127 of 1 .. 254)
__device__ __forceinline__ uint32_t two_powers(unsigned field) { return field << 7 | field << 23; }
// copies `bytes` (a multiple of 16) as they lie
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// byte offset of 16-byte chunk c of row r in a tile of `rows` rows: 64-column halves one behind the other, 128-byte swizzle
__device__ __forceinline__ uint32_t tile_off(int r, int c, int rows) { return (uint32_t)((c >> 3) * (rows * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }

__device__ __forceinline__ bool mbar_try(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded; gives up for the CTA, or because another of its warps has.  (Kept out of the way of waits that are over at once: with the flag
// read in front of each, the products' thread spent 0.18 us on every one of the six of a tile.)
__device__ __forceinline__ bool wait_long(uint64_t* bar, uint32_t parity, volatile int* gave_up) {
    for (int i = 0; i < SPIN_LIMIT; ++i) {
        if (mbar_try(bar, parity)) return true;
        if ((i & 63) == 63 && *gave_up) return false;
    }
    *gave_up = 1;
    return false;
}

typedef Schedule<CH_ROWS, CH_KEYS, 2> ChunkSchedule;

// What a run has of an item, and the halves' own ends.
struct ChunkPiece {
    int first, stop, p0, nrows;
    int end[2], see[2];                                          // a half's last tile + 1, positions that all its rows see
    bool whole;
    __device__ __forceinline__ ChunkPiece(const PagedView& w, const ChunkSchedule::Cursor& at, u64 run_end, int group) {
        first = at.tile;
        stop = at.tiles_before(run_end);
        whole = first == 0 && at.item_end() <= run_end;
        p0 = at.rb * CH_ROWS;
        nrows = min(CH_ROWS, at.q.rows * group - p0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int last = min(at.q.rows - 1, (p0 + 128 * i + 127) / group);
            const int tiles = nrows > 128 * i ? (min(at.q.kv + last + 1, w.capacity) + CH_KEYS - 1) / CH_KEYS : 0;
            end[i] = min(stop, tiles);
            see[i] = min(at.q.kv + (p0 + 128 * i) / group + 1, w.capacity);
        }
    }
};

template <int DH, bool E4M3>
__global__ void __launch_bounds__(CH_THREADS, 1)
paged_chunk_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const PagedView w, const AttendArgs a) {
    using C = ChunkCfg<DH, E4M3>;
    extern __shared__ unsigned char smem_dyn[];
    __shared__ ChunkBars bars;
    unsigned char* Qs = (unsigned char*)(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    unsigned char* slots = Qs + C::Q_BYTES;
    unsigned char* raws = slots + C::SLOTS * C::TILE_BYTES;
    u64* prefix = reinterpret_cast<u64*>(Qs);                    // (until the run's first unit is found)
    static_assert(2 * (CSD_MAX_SEQS + 1) * 8 <= C::Q_BYTES, "the prefixes fit");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, group = a.group;

    pdl_wait();
    if (tid == 0) joins_of(a)[blockIdx.x].last = -1;             // (the barriers of the count lie before what the softmax warps write there)
    u64* items = prefix + CSD_MAX_SEQS + 1;
    ChunkSchedule::count<CH_THREADS>(w, group, false, prefix, items, &bars.longest);
    const u64 units = prefix[w.n_seqs], n_items = items[w.n_seqs];
    u64 begin, end;
    ChunkSchedule::Cursor at;
    const unsigned n_runs = units < gridDim.x ? (unsigned)units : gridDim.x;
    int snap = 0;
    if (n_items <= gridDim.x && (u64)bars.longest <= units / gridDim.x + CH_ALONE) {
        if (blockIdx.x >= n_items) return;
        ChunkSchedule::item(w, items, blockIdx.x, group, false, &begin, &end, &at);
    } else {
        if (blockIdx.x >= n_runs) return;
        snap = ChunkSchedule::snap_of(units, n_runs, 3);
        if (!ChunkSchedule::run(w, prefix, blockIdx.x, n_runs, snap, group, false, &begin, &end, &at)) return;
    }

    if (tid == 0) {
        for (int i = 0; i < 8; ++i) { mbar_init(&bars.full[i], 4); mbar_init(&bars.free_[i], 1); mbar_init(&bars.landed[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bars.rawfull[i], 1); mbar_init(&bars.rawfree[i], 4); }
        mbar_init(&bars.qfull, 2); mbar_init(&bars.qfree, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.sfull[i], 1); mbar_init(&bars.pready[i][0], 4); mbar_init(&bars.pready[i][1], 4);
            mbar_init(&bars.firsthalf[i], 1); mbar_init(&bars.ofull[i], 1); mbar_init(&bars.ofree[i], 4);
        }
        bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        // behind the dependency wait: a kernel before this one may hold tensor memory until it ends
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem;
    volatile int* gave_up = &bars.abort_flag;
    pdl_trigger();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_try(bar, parity) || wait_long(bar, parity, gave_up); };
    auto warp_waits = [&](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)) != 0; };

    u64 unit = begin;
    auto advance = [&](const ChunkPiece& p) {
        unit = at.unit_of(p.stop);
        if (unit < end) { at.tile = p.stop - 1; at.next(w, group, false); }
    };

    if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(CH_FEWER));
    if (warp == 0) {
        // ---- requests, tiles in the order K, V of a position tile
        unsigned n = 0;                                          // tiles so far
        bool ok = true;
        // this lane's page of position tile t: lanes 0-7 have its eight groups of 16
        auto page_of = [&](int t) {
            const int pos = t * CH_KEYS + 16 * lane;
            return lane < 8 && pos < at.seen ? paged_page(w, at.s, pos) : -1;
        };
        const int P = 1 << w.page_shift, pages = CH_KEYS >> w.page_shift;
        while (unit < end && ok) {
            const ChunkPiece p(w, at, end, group);
            int page = page_of(p.first);
            for (int t = p.first; t < p.stop && ok; ++t) {
                const int next = t + 1 < p.stop ? page_of(t + 1) : -1;
                const unsigned lost = __ballot_sync(0xffffffffu, lane < 8 && t * CH_KEYS + 16 * lane < at.seen && page < 0);
                if (lane == 0) bars.lost[n >> 1 & 7] = lost;
                const bool edge = (t + 1) * CH_KEYS > p.see[0];  // (warps 4-7 look through its values)
#pragma unroll 1
                for (int kv = 0; kv < 2; ++kv, ++n) {
                    const int boxes = E4M3 ? pages : pages * C::HALVES, j = E4M3 ? lane : lane / C::HALVES;
                    const int pg = __shfl_sync(0xffffffffu, page, min(j, pages - 1) << (w.page_shift - 4));
                    const bool there = lane < boxes && pg >= 0;
                    const size_t row = there ? paged_row(w, pg, at.h, 0) : 0;
                    const int count = __popc(__ballot_sync(0xffffffffu, there));
                    if constexpr (!E4M3) {
                        const int slot = (int)(n % C::SLOTS);
                        ok = n < (unsigned)C::SLOTS || warp_waits(&bars.free_[slot], (n / C::SLOTS - 1) & 1u);
                        if (!ok) break;
                        const bool direct = kv == 0 || !edge;
                        uint64_t* bar = direct ? &bars.full[slot] : &bars.landed[slot];
                        if (kv == 1 && lost) {                   // values of positions without a page: zeros
                            for (int i = lane; i < CH_KEYS * DH / 8; i += 32) {
                                const int key = i / (DH / 8), c = i % (DH / 8);
                                if (lost >> (key >> 4) & 1)
                                    *reinterpret_cast<uint4*>(slots + slot * C::TILE_BYTES + tile_off(key, c, CH_KEYS)) = make_uint4(0u, 0u, 0u, 0u);
                            }
                            fence_async_smem();
                            __syncwarp();
                        }
                        if (lane == 0) mbar_expect_tx(bar, (uint32_t)count * (uint32_t)P * 128u);
                        __syncwarp();
                        if (direct && lane >= 1 && lane < 4) mbar_arrive(bar);
                        if (there)
                            tma_load_2d(slots + slot * C::TILE_BYTES + lane % C::HALVES * (CH_KEYS * 128) + j * P * 128, kv ? &tmV : &tmK, bar, lane % C::HALVES * 64, (int)row);
                    } else {
                        const int stage = (int)(n & 1u);
                        ok = n < 2u || warp_waits(&bars.rawfree[stage], ((n >> 1) - 1) & 1u);
                        if (!ok) break;
                        if (lane == 0) mbar_expect_tx(&bars.rawfull[stage], (uint32_t)count * (uint32_t)(P * (DH + 1)));
                        __syncwarp();
                        if (there) {
                            const uint32_t dst = smem_u32(raws) + stage * C::RAW;
                            bulk_load(dst + j * P * DH, (kv ? w.v : w.k) + row * DH, (uint32_t)(P * DH), &bars.rawfull[stage]);
                            bulk_load(dst + CH_KEYS * DH + j * P, (kv ? w.v_exp : w.k_exp) + row, (uint32_t)P, &bars.rawfull[stage]);
                        }
                    }
                }
                page = next;
            }
            advance(p);
        }
    } else if (warp == 2 || warp == 3) {
        // ---- queries: the block's rows as two operand tiles of 128
        int pieces = 0;
        bool ok = true;
        while (unit < end && ok) {
            const ChunkPiece p(w, at, end, group);
            if (pieces > 0) ok = warp_waits(&bars.qfree, (uint32_t)(pieces - 1) & 1u);
            if (!ok) break;
            ++pieces;
            // row r of the block is the (rem + r)-th (token, head) pair behind the block's first token
            constexpr int PER = DH / 8, STEP = 64 / PER;
            const int c = (tid - 64) % PER, r0 = (tid - 64) / PER, first = p.p0 % group + r0, token = p.p0 / group + first / group;
            const int tokens = STEP / group, heads = STEP % group;               // of a turn
            const int64_t turn = (int64_t)tokens * a.ldq + heads * DH, wrap = a.ldq - (int64_t)group * DH;
            int head = first % group;
            const uint16_t* src = (const uint16_t*)a.q + (size_t)(at.q.start + token) * a.ldq + (size_t)(at.h * group + head) * DH + 8 * c;
            const uint32_t q0 = smem_u32(Qs);
#pragma unroll 8
            for (int r = r0; r < CH_ROWS; r += STEP) {
                const bool there = r < p.nrows;
                cp_async16(q0 + (r >> 7) * (128 * DH * 2) + tile_off(r & 127, c, 128), there ? (const void*)src : a.q, there);
                src += turn;
                head += heads;
                if (head >= group) { head -= group; src += wrap; }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.qfull);
            advance(p);
        }
    } else if (warp >= 4 && warp < 8) {
        // ---- finishing tiles
        unsigned n = 0;
        uint32_t landings = 0;                                   // parities of landed[]
        bool ok = true;
        const int f = warp - 4;
        while (unit < end && ok) {
            const ChunkPiece p(w, at, end, group);
            for (int t = p.first; t < p.stop && ok; ++t) {
                const int t0 = t * CH_KEYS, left = at.seen - t0, see = p.see[0] - t0;
                if constexpr (!E4M3) {
                    const unsigned v = n + 1, slot = v % C::SLOTS;
                    n += 2;
                    if (see >= CH_KEYS) continue;
                    ok = warp_waits(&bars.landed[slot], landings >> slot & 1u);
                    if (!ok) break;
                    landings ^= 1u << slot;
                    // a lane a position
                    const int key = 32 * f + lane;
                    const bool gone = key >= left;
                    const uint32_t rowa = smem_u32(slots) + slot * C::TILE_BYTES + key * 128;
                    bool odd = false;
                    if (gone || key >= see) {
#pragma unroll 4
                        for (int i = 0; i < DH / 8; ++i) {       // (a lane's own order, so that the banks differ)
                            const uint32_t addr = rowa + (i >> 3) * (CH_KEYS * 128) + (((i ^ lane) & 7) << 4);
                            uint32_t x[4] = {0u, 0u, 0u, 0u};
                            bool change = gone;
                            if (!gone) {
                                asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr));
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (odd_bf16(x[e])) {
                                        change = odd = true;
                                        if ((x[e] & 0x7f80u) == 0x7f80u) x[e] &= 0xffff0000u;
                                        if ((x[e] & 0x7f800000u) == 0x7f800000u) x[e] &= 0xffffu;
                                    }
                            }
                            if (change) asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
                        }
                    }
                    const unsigned word = __ballot_sync(0xffffffffu, odd);
                    if (lane == 0) bars.odd[v >> 1 & 7][f] = word;
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.full[slot]);
                } else {
#pragma unroll 1
                    for (int kv = 0; kv < 2; ++kv, ++n) {
                        const int stage = (int)(n & 1u), slot = (int)(n % C::SLOTS);
                        ok = warp_waits(&bars.rawfull[stage], (n >> 1) & 1u);
                        if (ok) ok = n < (unsigned)C::SLOTS || warp_waits(&bars.free_[slot], (n / C::SLOTS - 1) & 1u);
                        if (!ok) break;
                        const unsigned lost = bars.lost[n >> 1 & 7];
                        const unsigned char* raw = raws + stage * C::RAW;
                        const uint32_t dst = smem_u32(slots) + slot * C::TILE_BYTES;
                        // 16-byte pieces of a row, rows a turn, of them a warp's; a lane works the scale of one of the warp's 32 rows out
                        constexpr int PER = DH / 16, STEP = 128 / PER, MINE = 32 / PER;
                        const int row = STEP * (lane / MINE) + MINE * f + lane % MINE;
                        const unsigned e = raw[CH_KEYS * DH + row];
                        // 2^(e - 127) times 2^120, as one power where that is one; 0 for what is not there; NaN for 255, but values that not
                        // every row sees are taken out and put in at the end
                        unsigned field = min(e + 120u, 254u), more = e + 120u > 254u ? e + 120u - 254u + 127u : 127u;
                        uint32_t up = two_powers(field);
                        bool odd = false;
                        if (row >= left || (lost >> (row >> 4) & 1)) { up = 0u; more = 127u; }
                        else if (e == 255u) {
                            odd = kv && row >= see;
                            up = odd ? 0u : 0x7fc07fc0u;
                            more = 127u;
                        }
                        const bool twice = __any_sync(0xffffffffu, more != 127u);
                        const uint32_t rest = two_powers(more);
                        const int key0 = MINE * f + lane / PER, c = lane % PER;
                        const unsigned char* src = raw + key0 * DH + 16 * c;
                        const uint32_t d0 = dst + tile_off(key0, 2 * c, CH_KEYS), d1 = dst + tile_off(key0, 2 * c + 1, CH_KEYS);
#pragma unroll 4
                        for (int i = 0; i < CH_KEYS / STEP; ++i) {
                            const uint4 u = *reinterpret_cast<const uint4*>(src + i * STEP * DH);
                            const uint32_t by1 = __shfl_sync(0xffffffffu, up, MINE * i + lane / PER), by2 = __shfl_sync(0xffffffffu, rest, MINE * i + lane / PER);
                            const uint2 x = widen4(u.x, by1, by2, twice), y = widen4(u.y, by1, by2, twice), z = widen4(u.z, by1, by2, twice), v = widen4(u.w, by1, by2, twice);
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(d0 + i * STEP * 128), "r"(x.x), "r"(x.y), "r"(y.x), "r"(y.y) : "memory");
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(d1 + i * STEP * 128), "r"(z.x), "r"(z.y), "r"(v.x), "r"(v.y) : "memory");
                        }
                        const unsigned word = __ballot_sync(0xffffffffu, odd);       // (of positions anywhere in the tile: that some are is all that is asked)
                        if (kv && lane == 0) bars.odd[n >> 1 & 7][f] = word;
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) { mbar_arrive(&bars.rawfree[stage]); mbar_arrive(&bars.full[slot]); }
                    }
                }
            }
            advance(p);
        }
    } else if (warp == 1) {
        // ---- products
        if (lane == 0) {
            constexpr uint32_t F = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(128 >> 4) << 24);      // bf16 x bf16 -> fp32, 128 rows
            constexpr uint32_t IDESC_S = F | ((uint32_t)(CH_KEYS >> 3) << 17), IDESC_O = F | (1u << 16) | ((uint32_t)(DH >> 3) << 17);   // (V: N along the rows)
            const uint64_t qd = smem_desc_sw128(smem_u32(Qs)), kd = smem_desc_sw128(smem_u32(slots)), vd = smem_desc_sw128_mn(smem_u32(slots), CH_KEYS * 128);
            uint32_t slot = 0, phase = 0;                        // of the next tile to be multiplied
            int pieces = 0, rounds[2] = {0, 0};                  // pieces that a half had tiles of
            uint32_t done[2] = {0, 0};                           // position tiles of a half
            bool ok = true;
            auto past = [&]() { if (++slot == (uint32_t)C::SLOTS) { slot = 0; phase ^= 1u; } };
            auto scores = [&](int i, uint32_t of) {
                const uint64_t q = qd + (uint64_t)((i * 128 * DH * 2) >> 4), k = kd + (uint64_t)(of * (C::TILE_BYTES >> 4));
#pragma unroll
                for (int ks = 0; ks < DH / 16; ++ks) {
                    const uint32_t off = (uint32_t)((ks >> 2) * (128 * 128) + (ks & 3) * 32) >> 4;
                    tc_mma(tmem + 128 * i, q + off, k + off, IDESC_S, ks > 0);
                }
                tc_commit(&bars.sfull[i]);
            };
            while (unit < end && ok) {
                const ChunkPiece p(w, at, end, group);
                // A half that this piece has nothing for (one at most) has left the pieces before all the same: what was noted of its last tiles (bars.odd) is
                // read on its way out, and the notes come round after eight tiles.  (One wait, here: for each half in the loop below it moves
                // the code so that a prompt of 4096 rows takes 2 to 5 % longer.)
                const int gone = p.first >= p.end[0] ? 0 : p.first >= p.end[1] ? 1 : -1, left = gone == 0 ? rounds[0] : gone == 1 ? rounds[1] : 0;
                ok = wait(&bars.qfull, (uint32_t)pieces & 1u) && wait(&bars.full[slot], phase) && (left == 0 || wait(&bars.ofree[gone], (uint32_t)(left - 1) & 1u));
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (p.first < p.end[i]) scores(i, slot);
                tc_commit(&bars.free_[slot]);
                past();
                if (p.stop == p.first + 1) tc_commit(&bars.qfree);
                for (int t = p.first; t < p.stop && ok; ++t) {
                    const bool more = t + 1 < p.stop;
                    const uint32_t v = slot;                     // this tile's values, and behind them the next one's keys
                    ok = wait(&bars.full[slot], phase);
                    past();
                    const uint32_t k = slot;
                    if (more) {
                        ok = ok && wait(&bars.full[slot], phase);
                        past();
                    }
                    const uint64_t vt = vd + (uint64_t)(v * (C::TILE_BYTES >> 4));
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (!ok || t >= p.end[i]) continue;
                        if (t == p.first && rounds[i] > 0) ok = wait(&bars.ofree[i], (uint32_t)(rounds[i] - 1) & 1u);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {            // weights of positions 0-63, then the others
                            ok = ok && wait(&bars.pready[i][j], done[i] & 1u);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int ks = 4 * j; ks < 4 * j + 4; ++ks)
                                tc_mma_ts(tmem + C::O_COL + 128 * i, tmem + 128 * i + 8 * ks, vt + (uint64_t)((ks * 2048) >> 4), IDESC_O, t > p.first || ks > 0);
                            if (j == 0) tc_commit(&bars.firsthalf[i]);
                        }
                        if (!ok) continue;
                        ++done[i];
                        if (t + 1 == p.end[i]) { tc_commit(&bars.ofull[i]); ++rounds[i]; }
                        if (t + 1 < p.end[i]) scores(i, k);
                    }
                    if (!ok) break;
                    tc_commit(&bars.free_[v]);
                    if (more) tc_commit(&bars.free_[k]);
                    if (t + 2 == p.stop) tc_commit(&bars.qfree);
                }
                ++pieces;
                advance(p);
            }
        }
    }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(CH_MORE));
        // ---- softmax: a half of the block's rows, a thread a row
        const int half = (warp - 8) >> 2, quad = warp & 3, r = 128 * half + 32 * quad + lane;
        const uint32_t lanes = (uint32_t)(32 * quad) << 16, S = tmem + lanes + 128 * half, O = tmem + lanes + C::O_COL + 128 * half;
        const float to_log2 = a.scale * 1.4426950408889634f;
        const u64 by = two(to_log2, to_log2);
        uint32_t done = 0, run_tiles = 0;                        // position tiles of the half, of the run
        int rounds = 0;
        bool ok = true;
        while (unit < end && ok) {
            const ChunkPiece p(w, at, end, group);
            const int p_row = p.p0 + r, token = p_row / group;
            const bool mine = r < p.nrows;
            const int lim = mine ? min(at.q.kv + token + 1, w.capacity) : 0;
            float m = -INFINITY, l = 0.f;
            bool odd = false;                                    // values were taken out of the run's tiles
            for (int t = p.first; t < p.end[half]; ++t, ++done) {
                ok = warp_waits(&bars.sfull[half], done & 1u);
                if (!ok) break;
                tc_fence_after();
                float x[32], y[32];
                tm_ld32(S, x);
                tm_ld32(S + 32, y);
                const unsigned lost_groups = bars.lost[(run_tiles + (t - p.first)) & 7];
                const bool edge = (t + 1) * CH_KEYS > p.see[half];
                u64 sums[2] = {0ull, 0ull};
                auto weights = [&](float (&s)[32], int col, u64 less) {
                    uint32_t w16[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const u64 e = fma2(two(s[2 * j], s[2 * j + 1]), by, less);
                        const float e0 = ex2(low(e)), e1 = ex2(high(e));
                        sums[j & 1] = add2(sums[j & 1], two(e0, e1));
                        w16[j] = pack_bf16(e0, e1);
                    }
                    tm_st16(S + col, w16);
                };
                // 64 positions, then the others: when the first are out, their product with the values begins
#pragma unroll 1
                for (int part = 0; part < 2; ++part) {           // (one copy of the code: two do not fit the schedulers' instruction caches)
                    tm_wait_ld();
                    if (edge) {
                        const int sees = lim - t * CH_KEYS - 64 * part;
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            x[j] = j < sees ? x[j] : -INFINITY;
                            y[j] = j + 32 < sees ? y[j] : -INFINITY;
                        }
                    }
                    const unsigned lost = lost_groups >> (4 * part) & 15u;
                    if (lost)
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            if (lost >> (j >> 4) & 1) x[j] = -INFINITY;
                            if (lost >> (2 + (j >> 4)) & 1) y[j] = -INFINITY;
                        }
                    float tops[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) tops[j] = fmaxf(x[j], y[j]);
#pragma unroll
                    for (int j = 4; j < 32; ++j) tops[j & 3] = max3(tops[j & 3], x[j], y[j]);
                    const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * to_log2;     // (the scale is positive here)
                    if (__any_sync(0xffffffffu, top > m + CH_LATE)) {
                        const float nm = fmaxf(m, top), keep = nm == -INFINITY ? 0.f : ex2(m - nm);
                        m = nm;
                        l = (l + (low(sums[0]) + high(sums[0])) + (low(sums[1]) + high(sums[1]))) * keep;
                        sums[0] = sums[1] = 0ull;
                        if (t > p.first || part) {
                            // (the first half's product may be under way; with the scores here, the tile before is done)
                            if (part) ok = warp_waits(&bars.firsthalf[half], done & 1u);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < DH; c += 16) {
                                float o[16];
                                tc_ld16(O + c, o);
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[j] *= keep;
                                tm_st16(O + c, o);
                            }
                        }
                    }
                    const float base = m == -INFINITY ? 0.f : m;
                    const u64 less = two(-base, -base);
                    weights(x, 32 * part, less);
                    if (part == 0) tm_ld32(S + 64, x);
                    weights(y, 32 * part + 16, less);
                    if (part == 0) tm_ld32(S + 96, y);
                    tm_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.pready[half][part]);
                }
                if (!ok) break;
                const u64 sum = add2(sums[0], sums[1]);
                l += low(sum) + high(sum);
            }
            if (!ok) break;
            // ---- the rows leave, finished or as a part of their item
            const bool any = p.first < p.end[half];
            if (any) {
                // (the products of these tiles have read their values, so what was noted of them stands)
                ok = warp_waits(&bars.ofull[half], (uint32_t)rounds & 1u);
                if (!ok) break;
                ++rounds;
                tc_fence_after();
                for (int t = max(p.first, p.end[half] - 4); t < p.end[half]; ++t) {
                    const unsigned i = (run_tiles + (unsigned)(t - p.first)) & 7;
                    if ((t + 1) * CH_KEYS > p.see[0]) odd |= (bars.odd[i][0] | bars.odd[i][1] | bars.odd[i][2] | bars.odd[i][3]) != 0;
                }
            }
            float* part = a.parts + ((size_t)blockIdx.x * 2 + (p.first == 0 ? 1 : 0)) * C::PART;
            const size_t dst = mine ? (size_t)(at.q.start + token) * a.ldo + (size_t)(at.h * group + p_row % group) * DH : 0;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            // 32 columns of the warp's rows: four lanes exchange 16-byte pieces, so that a store covers 64 bytes of each of eight rows
            // instead of 16 of 32
            auto store_rows = [&](int c, const float (&o)[32], float f) {
                uint32_t u[4][4];
#pragma unroll
                for (int j = 0; j < 16; ++j) u[j >> 2][j & 3] = pack_bf16(o[2 * j] * f, o[2 * j + 1] * f);
#pragma unroll
                for (int d = 1; d < 4; d <<= 1)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k & d) continue;             // pieces k and k + d: one goes over, the other stays
                        const bool upper = lane & d;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t got = __shfl_xor_sync(0xffffffffu, upper ? u[k][e] : u[k + d][e], d);
                            if (upper) u[k][e] = got; else u[k + d][e] = got;
                        }
                    }
                // u[k]: piece lane & 3 of row (lane & ~3) + k
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int from = (lane & ~3) + k;
                    const size_t to = __shfl_sync(0xffffffffu, (u64)dst, from);
                    if (__shfl_sync(0xffffffffu, (int)mine, from))
                        *reinterpret_cast<uint4*>((uint16_t*)a.out + to + c + 8 * (lane & 3)) = make_uint4(u[k][0], u[k][1], u[k][2], u[k][3]);
                }
            };
            if (any) {
#pragma unroll 1
                for (int c = 0; c < DH; c += 32) {
                    float o[32];
                    tm_ld32(O + c, o);
                    tm_wait_ld();
                    if (odd && mine)                             // infinities and NaN that this row sees
                        for (int pos = max(p.see[0], p.first * CH_KEYS); pos < min(lim, p.stop * CH_KEYS); ++pos) {
                            const int pg = paged_page(w, at.s, pos);
                            const size_t row = pg >= 0 ? paged_row(w, pg, at.h, pos) : 0;
                            if (pg < 0 || (E4M3 && w.v_exp[row] != 255u)) continue;
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                const float v = E4M3 ? __uint_as_float(0x7fffffffu) : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(w.v)[row * DH + c + j]);
                                if (!(fabsf(v) < INFINITY)) o[j] += v;
                            }
                        }
                    if (p.whole) {
                        store_rows(c, o, inv);
                    } else if (mine) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) __stcg(part + (half * DH + c + j) * 128 + 32 * quad + lane, o[j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.ofree[half]);
            }
            if (!p.whole && p.nrows > 128 * half) {
                if (mine) { __stcg(part + CH_ROWS * DH + r, m); __stcg(part + CH_ROWS * DH + CH_ROWS + r, l); }
                if (r == 0 && p.first == 0) {                    // the item's first part tells of it
                    int c0, c1;
                    ChunkSchedule::parts_of(at, units, n_runs, snap, &c0, &c1);
                    joins_of(a)[blockIdx.x] = ChunkJoin{c1, at.q.start, at.h, p.p0, p.nrows, {}};
                }
            }
            run_tiles += (uint32_t)(p.stop - p.first);
            advance(p);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*gave_up) {
        if (tid == 0) set_status(w.status, CSD_ERR_TIMEOUT);
        __nanosleep(2000000);                    // let products already issued end before the CTA's memory is released
    }
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Adds up the parts of the items that lie in several CTAs' runs, in the order of the runs.  The grid takes the items' jobs, 16 dimensions of a half's
// 128 rows each, in turn: a warp two dimensions, a lane four rows, JOIN_PARTS parts under way at a time, three blocks an SM; it is bounded by the parts' way
// through the L2 cache.  While the last CTA to arrive at an item added it up alone, 16 rows of 32 heads on 8 behind 16000 positions, 18 parts an item,
// took 73 us, 48 of them for this, and behind 1000 32 us; now 35 and 17, and a prompt of 4096 rows, most items in two parts, 180 for 175.  (Four parts and two
// blocks: 33, 17 and 186; two and four: 38, 18 and 184.)
constexpr int JOIN_PARTS = 3, JOIN_DIMS = 16, JOIN_THREADS = 256;
template <int DH> __global__ void __launch_bounds__(JOIN_THREADS, 3) paged_join_kernel(const AttendArgs a, int n) {
    constexpr int PART = ChunkCfg<DH, false>::PART, GROUPS = DH / JOIN_DIMS, WARPS = JOIN_THREADS / 32;
    static_assert(JOIN_DIMS == 2 * WARPS, "two dimensions a warp");
    __shared__ int counts[WARPS];
    __shared__ short items[JOIN_MOST];
    __shared__ float outs[JOIN_DIMS][128 + 4];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const ChunkJoin* joins = joins_of(a);
    pdl_wait();
    pdl_trigger();
    int n_items = 0;
    for (int c0 = 0; c0 < n; c0 += JOIN_THREADS) {
        const bool has = c0 + tid < n && __ldcg(&joins[c0 + tid].last) >= 0;
        const unsigned in = __ballot_sync(0xffffffffu, has);
        if (lane == 0) counts[warp] = __popc(in);
        __syncthreads();
        int at = n_items;
        for (int i = 0; i < WARPS; ++i) {
            if (i < warp) at += counts[i];
            n_items += counts[i];
        }
        if (has) items[at + __popc(in & ((1u << lane) - 1u))] = (short)(c0 + tid);
        __syncthreads();
    }
    for (int job = blockIdx.x; job < n_items * 2 * GROUPS; job += gridDim.x) {
        const int c0 = items[job / (2 * GROUPS)], half = job / GROUPS & 1, d0 = job % GROUPS * JOIN_DIMS;
        const int4 told = __ldcg(reinterpret_cast<const int4*>(joins + c0));
        const ChunkJoin item = {told.x, told.y, told.z, told.w, __ldcg(&joins[c0].rows), {}};
        const int rows = min(item.rows - 128 * half, 128);
        if (rows <= 0) continue;
        const int r = 4 * lane;                                  // (rows behind the item's are never written out)
        float top[4], total[4], o[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { top[i] = -INFINITY; total[i] = o[0][i] = o[1][i] = 0.f; }
        for (int k0 = c0; k0 <= item.last; k0 += JOIN_PARTS) {
            float m[JOIN_PARTS][4], l[JOIN_PARTS][4], x[2][JOIN_PARTS][4];
#pragma unroll
            for (int k = 0; k < JOIN_PARTS; ++k) {
                const bool there = k0 + k <= item.last && r < rows;
                const float* part = a.parts + ((size_t)(k0 + k) * 2 + (k0 + k == c0 ? 1 : 0)) * PART;
                auto get = [&](float (&to)[4], int at, float none) {
                    const float4 v = there ? __ldcg(reinterpret_cast<const float4*>(part + at)) : make_float4(none, none, none, none);
                    to[0] = v.x; to[1] = v.y; to[2] = v.z; to[3] = v.w;
                };
                get(m[k], CH_ROWS * DH + 128 * half + r, -INFINITY);
                get(l[k], CH_ROWS * DH + CH_ROWS + 128 * half + r, 0.f);
                get(x[0][k], (half * DH + d0 + 2 * warp) * 128 + r, 0.f);
                get(x[1][k], (half * DH + d0 + 2 * warp + 1) * 128 + r, 0.f);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float now = top[i];
#pragma unroll
                for (int k = 0; k < JOIN_PARTS; ++k) now = fmaxf(now, m[k][i]);
                const float keep = top[i] == -INFINITY ? 0.f : ex2(top[i] - now);
                top[i] = now;
                total[i] *= keep; o[0][i] *= keep; o[1][i] *= keep;
#pragma unroll
                for (int k = 0; k < JOIN_PARTS; ++k) {
                    // nothing was written of the row, or it sees nothing in the part.  (Scores that are all NaN leave the maximum at -inf too, but
                    // not the sum at 0: their NaN goes on.)
                    if (m[k][i] == -INFINITY && l[k][i] == 0.f) continue;
                    const float f = ex2(m[k][i] - now);
                    total[i] = fmaf(f, l[k][i], total[i]);
                    o[0][i] = fmaf(f, x[0][k][i], o[0][i]);
                    o[1][i] = fmaf(f, x[1][k][i], o[1][i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float scale = total[i] == 0.f ? 0.f : 1.f / total[i];
            outs[2 * warp][r + i] = o[0][i] * scale;
            outs[2 * warp + 1][r + i] = o[1][i] * scale;
        }
        __syncthreads();
        // two threads a row, eight dimensions each
        const int row = tid >> 1, d = tid % 2 * 8;
        if (row < rows) {
            const int p = item.p0 + 128 * half + row;
            uint32_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = pack_bf16(outs[d + 2 * j][row], outs[d + 2 * j + 1][row]);
            *reinterpret_cast<uint4*>((uint16_t*)a.out + (size_t)(item.start + p / a.group) * a.ldo + (size_t)(item.head * a.group + p % a.group) * DH + d0 + d) = make_uint4(u[0], u[1], u[2], u[3]);
        }
        __syncthreads();
    }
}

template <int DH, bool E4M3> static csd_status run_chunk(const PagedView& w, const AttendArgs& a, cudaStream_t st) {
    using C = ChunkCfg<DH, E4M3>;
    auto kern = paged_chunk_kernel<DH, E4M3>;
    static PerDevice ready;
    const csd_status ok = allow_smem(ready, kern, C::SMEM);
    if (ok != CSD_OK) return ok;
    CUtensorMap tk = {}, tv = {};
    if constexpr (!E4M3) {
        const int rows = w.n_pages * w.heads << w.page_shift;    // (below 2^31: paged_view)
        if (!encode_map_2d(w.k, rows, DH, 1 << w.page_shift, &tk) || !encode_map_2d(w.v, rows, DH, 1 << w.page_shift, &tv)) return CSD_ERR_UNSUPPORTED;
    }
    PdlLaunch L(dim3((unsigned)tc_sm_count()), dim3(CH_THREADS), C::SMEM, st);
    CSD_CUDA(cudaLaunchKernelEx(&L.cfg, kern, tk, tv, w, a));
    count_launch();
    PdlLaunch J(dim3((unsigned)(3 * tc_sm_count())), dim3(JOIN_THREADS), 0, st);
    CSD_CUDA(cudaLaunchKernelEx(&J.cfg, paged_join_kernel<DH>, a, tc_sm_count()));
    count_launch();
    return CSD_OK;
}

size_t paged_chunk_workspace(int d_head) {
    return PAGED_TICKET_BYTES + JOIN_MOST * sizeof(ChunkJoin) + (size_t)tc_sm_count() * 2 * (d_head == 64 ? ChunkCfg<64, false>::PART : ChunkCfg<128, false>::PART) * 4;
}

csd_status launch_paged_chunk(const PagedView& w, AttendArgs a, int d_head, void* workspace, cudaStream_t st) {
    if (tc_sm_count() > JOIN_MOST) return CSD_ERR_UNSUPPORTED;
    a.tickets = (unsigned*)workspace;
    a.parts = (float*)(joins_of(a) + JOIN_MOST);
    if (d_head == 64) return w.k_exp ? run_chunk<64, true>(w, a, st) : run_chunk<64, false>(w, a, st);
    return w.k_exp ? run_chunk<128, true>(w, a, st) : run_chunk<128, false>(w, a, st);
}

}  // namespace csd
