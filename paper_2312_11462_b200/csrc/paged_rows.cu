// Attention over the paged cache for few rows a sequence: decode, reviews of drafted blocks and trees (and fp32 rows of any number).
//
// What bounds it is the cache: each visible page is read once per block of 16 or 32 (row, query head) pairs.  A CTA has twelve
// or eight warps, one CTA an SM.  A key tile is one or two groups of 16 positions a warp, a group always inside one page; each warp
// stages its own keys and values with cp.async, across the ends of items, one tile ahead where twelve warps have tiles of 8 KB each and two to four elsewhere,
// and never waits for another warp until an item ends: it keeps its own running maximum, sum and output, which the CTA's warps add up through shared memory.
// An SM has 96 to 146 KB in flight that way (fp32 rows of 64 over 8 bits, more than 16 of them: 65), up to three times what the memory's latency asks for.
// Measured: bf16 rows of 128 at 6.5 TB/s, the copy rate; 8-bit ones at 4.5 (issuing in 59 % of the cycles, most of it to widen them).
//
// Scores and outputs are mma.sync products (m16n8k16): at 16 rows a tile's products take a sixth of its loading time, and the
// operands' layout leaves the scores' accumulators as the operands of the second product.  Rows in bf16 enter as they are, their weights as
// bf16.  Rows in fp32 enter as three bf16 terms (24 bits), and so do their weights.
//
// The parts of an item in several runs are added up by the last CTA to arrive, 16 loads of a thread under way (32 rows behind 16000 positions, 18
// parts: 43 us with four, 38).
//
// 8-bit rows are widened in registers.  Keys: e4m3 is a subset of fp16, so the conversion is one instruction for
// two; the query then enters in fp16 too, each row times a power of two that puts its largest entry at 2^13 (entries down to 2^-27 of
// it stay exact; fp32 rows as two terms, 22 bits).  Values: to bf16 by shifting the exponent field and a multiplication by 2^120, as the
// weights times the rows' scales need bf16's range.
#include "attention_mma.cuh"
#include "paged_attention.cuh"
#include <cuda_fp16.h>
#include <type_traits>

namespace csd {

constexpr int PSMEM = 227 * 1024;
constexpr float LATE = 8.f;                     // a running maximum may lag by this power of two (weights of up to 2^8)

constexpr int most_dims(int rows, int dims, int bytes) { return rows * dims * 4 <= bytes ? dims : most_dims(rows, dims / 2, bytes); }

template <int DH, int MT, bool ROWS16, bool E4M3> struct PagedRowsCfg {
    static constexpr int BR = 16 * MT;
    // warps of a CTA: three to a scheduler hide one another's chains where their registers fit (296 heads of 16384 positions, four rows
    // each: bf16 451 us with eight, 381 with twelve; 8 bits 356 and 270)
    static constexpr int PW = MT == 1 ? 12 : 8;
    static constexpr int RB = E4M3 ? DH : 2 * DH;                        // bytes of a cache row
    static constexpr int QT = ROWS16 ? 1 : E4M3 ? 2 : 3;                 // terms of a query entry
    static constexpr int PT = ROWS16 ? 1 : 3;                            // of a weight
    // groups of 16 positions that a warp takes of a tile: two where rows are short, whose loading time one group's chain of
    // products, maxima and exponentials exceeds (8-bit rows of 128, 296 heads of 16384 positions: 390 us with one)
    static constexpr int GK = RB <= 128 && (MT == 1 || ROWS16) ? 2 : 1, WK = 16 * GK, KEYS = WK * PW;
    static constexpr int STAGE = 2 * WK * RB + (E4M3 ? 2 * WK : 0);      // a warp's keys, values and scales of a tile
    static constexpr int DIMS = most_dims(BR, DH, STAGE);                // dimensions of the rows that a stage has room for in fp32
    static constexpr int Q = QT * BR * DH * 2, ROWF = (2 * PW + 3) * BR * 4;
    static constexpr int FIXED = Q + ROWF;
    static constexpr int FIT = (PSMEM - FIXED - 512) / (PW * STAGE), STAGES = FIT > 5 ? 5 : FIT;
    static_assert(STAGES >= 2 && STAGES * PW * STAGE >= (CSD_MAX_SEQS + 1) * 8, "two tiles in flight, room for the prefix");
    static constexpr int SMEM = FIXED + STAGES * PW * STAGE;
    static constexpr int PART = BR * (DH + 2);                           // floats of a part: rows, maxima, sums (paged_rows_workspace)
};

__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t e4m3_to_f16(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((unsigned short)two));
    return r;
}
// bytes 0 and 2 (odd: 1 and 3) of four e4m3 numbers as bf16 (a number's exponent field lands 120 below where bf16 has it)
__device__ __forceinline__ uint32_t e4m3_to_bf16(uint32_t w, bool odd) {
    uint32_t r = odd ? ((w >> 4) & 0x07f007f0u) | (w & 0x80008000u) : ((w << 4) & 0x07f007f0u) | ((w << 8) & 0x80008000u);
    asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(0x7b807b80u));
    return r;
}
// byte offset of 16-byte chunk c of row j, so that ldmatrix reads eight rows without conflict
template <int RB> __device__ __forceinline__ uint32_t stage_off(int j, int c) {
    return (uint32_t)(j * RB + ((RB >= 128 ? c ^ (j & 7) : c ^ ((j >> 1) & 3)) << 4));
}

template <int DH, int MT, bool ROWS16, bool E4M3>
__global__ void __launch_bounds__(32 * PagedRowsCfg<DH, MT, ROWS16, E4M3>::PW, 1)
paged_rows_kernel(const PagedView w, const AttendArgs a) {
    using C = PagedRowsCfg<DH, MT, ROWS16, E4M3>;
    using S = Schedule<C::BR, C::KEYS, 1>;
    constexpr int BR = C::BR, PW = C::PW, KS = DH / 16, NS = C::STAGES, GK = C::GK, WK = C::WK, RB = C::RB;
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* Qs = smem;
    u64* prefix = reinterpret_cast<u64*>(smem + C::FIXED);               // (until the run's first unit is found)
    float* row_m = reinterpret_cast<float*>(Qs + C::Q);  // [warp][row], then the item's [row]
    float* row_l = row_m + PW * BR;
    float* row_f = row_l + PW * BR;                      // [3][row]
    __shared__ int s_last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    unsigned char* stages = smem + C::FIXED + warp * (NS * C::STAGE);
    const uint32_t st0 = smem_u32(stages), qs0 = smem_u32(Qs);

    pdl_wait();
    pdl_trigger();
    S::template count<32 * PW>(w, a.group, a.tree != nullptr, prefix);
    const u64 units = prefix[w.n_seqs];
    const unsigned n_runs = units < gridDim.x ? (unsigned)units : gridDim.x;
    if (blockIdx.x >= n_runs) return;
    const int snap = S::snap_of(units, n_runs, 16);
    const bool tree = a.tree != nullptr;
    const float to_log2 = a.scale * 1.4426950408889634f;

    typename S::Cursor ld, at;                           // the tile to request next, the tile to multiply
    u64 begin, end;
    if (!S::run(w, prefix, blockIdx.x, n_runs, snap, a.group, tree, &begin, &end, &at)) return;
    __syncthreads();                                     // (the stages take the prefix's place)
    ld = at;
    unsigned lost = 0;                                   // GK bits a stage: groups that have no positions or no page
    // Pages of this warp's groups, a lane a group: of tiles paged .. of the item at ld (what is found is checked when it is used)
    int pages = -1, paged = 0;
    auto look_up = [&]() {
        paged = ld.tile;
        const int t0 = (ld.tile + lane / GK) * C::KEYS + WK * warp + 16 * (lane % GK);
        pages = t0 < ld.seen ? w.table[(size_t)ld.s * w.max_pages + (t0 >> w.page_shift)] : -1;
    };
    look_up();
    // Requests the positions of the tile at ld into a stage.
    auto request = [&](int slot) {
        if (ld.unit_of(ld.tile) < end) {
            const uint32_t dst = st0 + slot * C::STAGE;
            lost &= ~(((1u << GK) - 1) << (slot * GK));
#pragma unroll
            for (int q = 0; q < GK; ++q) {
                const int t0 = ld.tile * C::KEYS + WK * warp + 16 * q, n = ld.seen - t0, page = __shfl_sync(0xffffffffu, pages, (ld.tile - paged) * GK + q);
                const bool is = page >= 0 && page < w.n_pages;
                if (n > 0 && !is) set_status(w.status, CSD_ERR_BAD_PAGE);
                if (!is) lost |= 1u << (slot * GK + q);
                const size_t row = is ? paged_row(w, page, ld.h, t0) : 0;
                const unsigned char* ks = w.k + row * RB + lane * 16;
                const unsigned char* vs = w.v + row * RB + lane * 16;
                constexpr int PER = RB / 16;             // 16-byte chunks of a row
#pragma unroll
                for (int i = 0; i < RB / 32; ++i) {
                    const int c = i * 32 + lane, j = c / PER, cc = c % PER;
                    const bool there = is && j < n;
                    cp_async16(dst + stage_off<RB>(16 * q + j, cc), ks + i * 512, there);
                    cp_async16(dst + WK * RB + stage_off<RB>(16 * q + j, cc), vs + i * 512, there);
                }
                if (E4M3 && lane < 2) cp_async16(dst + 2 * WK * RB + 16 * q + WK * lane, (lane ? w.v_exp : w.k_exp) + row, is);
            }
            // (behind the run's last tile the cursor stays on it, one tile too far)
            if (ld.tile + 1 < ld.tiles || ld.item_end() < end) ld.next(w, a.group, tree); else ++ld.tile;
            if (ld.unit_of(ld.tile) < end && ld.tile < ld.tiles) {
                if (ld.tile == 0 || ld.tile == paged + 32 / GK) look_up();
            }
        }
        cp_async_commit();
    };
#pragma unroll 1
    for (int i = 0; i < NS - 1; ++i) request(i);

    int slot = 0;
    u64 unit = begin;
    while (unit < end) {
        // ---- an item, or the part of it that this run has
        const u64 item_end = at.item_end();
        const int first_tile = at.tile, stop = at.tiles_before(end);
        const int p0 = at.rb * BR, nrows = min(BR, at.q.rows * a.group - p0);
        __syncthreads();                                 // (the item before has left Qs and the row arrays)
        {   // the block's queries as operand rows
            constexpr int PER = DH / 8;
            for (int i = tid; i < BR * PER; i += 32 * PW) {
                const int r = i / PER, c = i % PER, p = p0 + r;
                float x[8] = {};
                if (r < nrows) {
                    const size_t src = (size_t)(at.q.start + p / a.group) * a.ldq + (size_t)(at.h * a.group + p % a.group) * DH + 8 * c;
                    if constexpr (ROWS16) {
                        const uint4 u = *reinterpret_cast<const uint4*>((const uint16_t*)a.q + src);
                        x[0] = bf16lo(u.x); x[1] = bf16hi(u.x); x[2] = bf16lo(u.y); x[3] = bf16hi(u.y);
                        x[4] = bf16lo(u.z); x[5] = bf16hi(u.z); x[6] = bf16lo(u.w); x[7] = bf16hi(u.w);
                    } else {
                        const float4 u = *reinterpret_cast<const float4*>((const float*)a.q + src), v = *reinterpret_cast<const float4*>((const float*)a.q + src + 4);
                        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
                        if (a.rope.cos) {
                            const float* far = (const float*)a.q + src + (8 * c < DH / 2 ? DH / 2 : -DH / 2);
                            const float4 y = *reinterpret_cast<const float4*>(far), z = *reinterpret_cast<const float4*>(far + 4);
                            const float other[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
                            const int i = p / a.group;
                            rope8(a.rope, rope_position(w, a.rope, at.q.kv, i, at.q.rows, a.tree ? a.tree + at.q.start + i : nullptr), DH / 2, 8 * c, x, other);
                        }
                    }
                }
                if constexpr (!E4M3) {
#pragma unroll
                    for (int t = 0; t < C::QT; ++t) {
                        uint32_t u[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            u[j] = pack_bf16(x[2 * j], x[2 * j + 1]);
                            x[2 * j] -= bf16lo(u[j]); x[2 * j + 1] -= bf16hi(u[j]);
                        }
                        *reinterpret_cast<uint4*>(Qs + (size_t)t * BR * DH * 2 + stage_off<2 * DH>(r, c)) = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                } else {
                    float top = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[j]));
#pragma unroll
                    for (int o = PER / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    // 2^(13 - exponent of the largest entry); the row's scores are multiplied by its inverse
                    const int e = min(max((int)(__float_as_uint(top) >> 23), 20), 250);
                    const float up = __uint_as_float((unsigned)(267 - e) << 23), down = __uint_as_float((unsigned)(e - 13) << 23);
                    if (c == 0) row_f[2 * BR + r] = down;
                    // dimension 16 s + 4 c + r of a row stands where a thread's four bytes of a key row put it: r = 0, 1 in the first
                    // half of an operand's 16, r = 2, 3 in the second
#pragma unroll
                    for (int t = 0; t < C::QT; ++t)
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            const __half2 hh = __floats2half2_rn(x[j] * up, x[j + 1] * up);
                            const float2 f = __half22float2(hh);
                            x[j] -= f.x * down; x[j + 1] -= f.y * down;
                            const int d = 8 * c + j, within = d & 15, k = (within & 2 ? 8 : 0) + 2 * (within >> 2);
                            *reinterpret_cast<__half2*>(Qs + (size_t)t * BR * DH * 2 + stage_off<2 * DH>(r, (d >> 4) * 2 + (k >> 3)) + 2 * (k & 7)) = hh;
                        }
                }
            }
        }
        // what this thread's rows see: 16 mt + lane / 4 (+ 8)
        int lim[MT][2];
        u64 bits[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int hr = 0; hr < 2; ++hr) {
                const int r = 16 * mt + (lane >> 2) + 8 * hr, i = (p0 + r) / a.group;
                lim[mt][hr] = r < nrows ? min(at.q.kv + (tree ? 0 : i + 1), w.capacity) : 0;
                bits[mt][hr] = tree && r < nrows ? a.tree[at.q.start + i] : 0ull;
            }
        const int all_see = min(at.q.kv + (tree ? 0 : p0 / a.group + 1), w.capacity);   // positions that every row sees
        __syncthreads();
        float q_scale[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int hr = 0; hr < 2; ++hr) q_scale[mt][hr] = E4M3 ? to_log2 * row_f[2 * BR + 16 * mt + (lane >> 2) + 8 * hr] : to_log2;

        float o[MT][DH / 8][4], m[MT][2], l[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt][0] = m[mt][1] = -INFINITY;
            l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
            for (int t = 0; t < DH / 8; ++t) o[mt][t][0] = o[mt][t][1] = o[mt][t][2] = o[mt][t][3] = 0.f;
        }
#pragma unroll 1
        for (int tile = first_tile; tile < stop; ++tile) {
            cp_async_wait<NS - 2>();
            __syncwarp();                                // the stage has landed for all lanes, and all have read the one before
            const int t0 = tile * C::KEYS + WK * warp;
            const uint32_t Kt = st0 + slot * C::STAGE, Vt = Kt + WK * RB;
            const unsigned gone = lost >> (slot * GK) & ((1u << GK) - 1);
            request(slot == 0 ? NS - 1 : slot - 1);
            if (gone != (1u << GK) - 1) {
                // ---- scores: 16 rows a block against the warp's positions in blocks of 8, the smallest terms first
                constexpr int NG = 2 * GK, CH = GK == 1 ? 2 : 1;         // (of one group two chains, even and odd steps of 16 dimensions)
                float s[MT][NG][4], more[CH][MT][NG][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[mt][g][e] = more[CH - 1][mt][g][e] = 0.f;
                const int key = (lane >> 4) * 8 + (lane & 7);
#pragma unroll
                for (int k2 = 0; k2 < KS; k2 += 2) {
                    uint32_t kb[2][GK][4];               // [16 dimensions][group][keys 0-7: two halves, keys 8-15: two halves]
#pragma unroll
                    for (int q = 0; q < GK; ++q) {
                        if constexpr (E4M3) {
                            uint32_t raw[4];
                            ldsm_x4(Kt + stage_off<RB>(16 * q + key, k2 + ((lane >> 3) & 1)), raw);
#pragma unroll
                            for (int u = 0; u < 2; ++u)
#pragma unroll
                                for (int g = 0; g < 2; ++g) {
                                    kb[u][q][2 * g] = e4m3_to_f16(raw[2 * g + u] & 0xffffu);
                                    kb[u][q][2 * g + 1] = e4m3_to_f16(raw[2 * g + u] >> 16);
                                }
                        } else {
#pragma unroll
                            for (int u = 0; u < 2; ++u) ldsm_x4(Kt + stage_off<RB>(16 * q + key, 2 * (k2 + u) + ((lane >> 3) & 1)), kb[u][q]);
                        }
                    }
#pragma unroll
                    for (int t = C::QT - 1; t >= 0; --t)
#pragma unroll
                        for (int u = 0; u < 2; ++u)
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                uint32_t qa[4];
                                ldsm_x4(qs0 + t * BR * DH * 2 + stage_off<2 * DH>(16 * mt + (lane & 15), 2 * (k2 + u) + (lane >> 4)), qa);
#pragma unroll
                                for (int g = 0; g < NG; ++g) {
                                    float (&acc)[4] = CH == 2 && u ? more[CH - 1][mt][g] : s[mt][g];
                                    const uint32_t (&kk)[4] = kb[u][g >> 1];
                                    if constexpr (E4M3) mma_f16(acc, qa, kk[2 * (g & 1)], kk[2 * (g & 1) + 1]);
                                    else mma_bf16(acc, qa, kk[2 * (g & 1)], kk[2 * (g & 1) + 1]);
                                }
                            }
                }
                float kscale[NG][2], vscale[NG][2];      // [8 keys][this lane's two]
                if constexpr (E4M3) {
                    const unsigned char* ex = stages + slot * C::STAGE + 2 * WK * RB;
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const uint32_t ke = *reinterpret_cast<const uint16_t*>(ex + 8 * g + 2 * (lane & 3));
                        const uint32_t ve = *reinterpret_cast<const uint16_t*>(ex + WK + 8 * g + 2 * (lane & 3));
                        kscale[g][0] = row_scale(ke & 255u); kscale[g][1] = row_scale(ke >> 8);
                        vscale[g][0] = row_scale(ve & 255u); vscale[g][1] = row_scale(ve >> 8);
                    }
                }
                // ---- scale and mask; the warp's own running maxima
                const bool edge = t0 + WK > all_see || gone;
                float mx[MT][2];
                bool grown = false, nan = false;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int hr = 0; hr < 2; ++hr) {
#pragma unroll
                        for (int g = 0; g < NG; ++g)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float& x = s[mt][g][2 * hr + e];
                                if constexpr (CH == 2) x += more[CH - 1][mt][g][2 * hr + e];
                                if constexpr (E4M3) x *= kscale[g][e];
                                x *= q_scale[mt][hr];
                                if (edge) {
                                    const int t = t0 + 8 * g + 2 * (lane & 3) + e, back = t - at.q.kv;
                                    const bool sees = t < lim[mt][hr] || (back >= 0 && back < 64 && t < at.seen && (bits[mt][hr] >> back & 1));
                                    if (!sees || (gone >> (g >> 1) & 1)) x = -INFINITY;
                                }
                                nan |= x != x;
                            }
                    }
                // An infinite entry of a key times a query's smaller terms, 0 or of the other sign, is NaN or the other infinity: of fp32 rows
                // the scores that are NaN are formed anew, each query entry as one number
                if constexpr (!ROWS16 && !E4M3) {
                    if (__any_sync(0xffffffffu, nan)) {
                        const unsigned char* kt = stages + slot * C::STAGE;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int hr = 0; hr < 2; ++hr)
#pragma unroll
                                for (int g = 0; g < NG; ++g)
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        float& x = s[mt][g][2 * hr + e];
                                        if (x == x) continue;
                                        const int r = 16 * mt + (lane >> 2) + 8 * hr, k = 8 * g + 2 * (lane & 3) + e;
                                        x = 0.f;
#pragma unroll 1
                                        for (int d = 0; d < DH; ++d) {
                                            float y = 0.f;
#pragma unroll
                                            for (int t = 0; t < C::QT; ++t)
                                                y += bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(Qs + (size_t)t * BR * DH * 2 + stage_off<2 * DH>(r, d >> 3) + 2 * (d & 7)));
                                            x = fmaf(y, bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(kt + stage_off<RB>(k, d >> 3) + 2 * (d & 7))), x);
                                        }
                                        x *= q_scale[mt][hr];
                                    }
                    }
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int hr = 0; hr < 2; ++hr) {
                        float top = -INFINITY;
#pragma unroll
                        for (int g = 0; g < NG; ++g) top = fmaxf(top, fmaxf(s[mt][g][2 * hr], s[mt][g][2 * hr + 1]));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        mx[mt][hr] = top;
                        grown |= top > m[mt][hr] + LATE;                 // (from -inf: any score)
                    }
                if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int hr = 0; hr < 2; ++hr) {
                            const float nm = fmaxf(m[mt][hr], mx[mt][hr]);
                            const float keep = nm == -INFINITY ? 0.f : ex2(m[mt][hr] - nm);
                            m[mt][hr] = nm;
                            l[mt][hr] *= keep;
#pragma unroll
                            for (int t = 0; t < DH / 8; ++t) { o[mt][t][2 * hr] *= keep; o[mt][t][2 * hr + 1] *= keep; }
                        }
                }
                // ---- weights as operand rows; the sums run over the weights as the products see them
                uint32_t pa[MT][GK][C::PT][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int q = 0; q < GK; ++q)
#pragma unroll
                        for (int f = 0; f < 4; ++f) {                    // rows lane / 4 + 8 (f & 1), keys 8 (f >> 1) + this lane's two
                            const int hr = f & 1, g = 2 * q + (f >> 1);
                            const float base = m[mt][hr] == -INFINITY ? 0.f : m[mt][hr];
                            const float x0 = ex2(s[mt][g][2 * hr] - base), y0 = ex2(s[mt][g][2 * hr + 1] - base);
                            float x = x0, y = y0, sum = 0.f;
#pragma unroll
                            for (int t = 0; t < C::PT; ++t) {
                                uint32_t u = pack_bf16(x, y);
                                const float xr = bf16lo(u), yr = bf16hi(u);
                                x -= xr; y -= yr;
                                sum += xr + yr;
                                // (a power of two: exact; a position that nobody sees may have any scale, of one that all see a NaN counts even
                                // where the weight is below fp32's range)
                                if constexpr (E4M3) u = pack_bf16(edge && x0 == 0.f ? 0.f : xr * vscale[g][0], edge && y0 == 0.f ? 0.f : yr * vscale[g][1]);
                                pa[mt][q][t][f] = u;
                            }
                            l[mt][hr] += sum;
                        }
                // ---- output += weights . values.  0 x NaN is NaN: where some rows do not see all of the positions, infinities and NaN
                //      among their values send the warp through them one by one (fp32 rows everywhere: an infinity times a weight's
                //      terms is one less another)
                bool odd = false;
                if (edge || !ROWS16) {
                    if constexpr (E4M3) {
                        odd = lane < WK && t0 + lane < at.seen && (stages + slot * C::STAGE + 2 * WK * RB)[WK + lane] == 255u;
                    } else {
#pragma unroll
                        for (int i = 0; i < WK * RB / 512; ++i) {
                            const uint4 u = *reinterpret_cast<const uint4*>(stages + slot * C::STAGE + WK * RB + (i * 32 + lane) * 16);
                            odd |= odd_bf16(u.x) || odd_bf16(u.y) || odd_bf16(u.z) || odd_bf16(u.w);
                        }
                    }
                }
                if (__any_sync(0xffffffffu, odd)) {
                    const unsigned char* vt = stages + slot * C::STAGE + WK * RB;
#pragma unroll 1
                    for (int k = 0; k < WK; ++k) {
                        const int from = (lane & ~3) | ((k & 7) >> 1);
                        const float vs = E4M3 ? row_scale(vt[WK * RB + WK + k]) : 1.f;
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int hr = 0; hr < 2; ++hr) {
                                float x = 0.f;
#pragma unroll
                                for (int g = 0; g < NG; ++g) {
                                    const float even = s[mt][g][2 * hr], uneven = s[mt][g][2 * hr + 1];
                                    x = (k & ~6) == 8 * g ? even : x;
                                    x = (k & ~6) == 8 * g + 1 ? uneven : x;
                                }
                                x = __shfl_sync(0xffffffffu, x, from);
                                // not seen, or a score of -inf: no weight, but what it sees that is not finite counts
                                const int t1 = t0 + k, back = t1 - at.q.kv;
                                const bool sees = t1 < lim[mt][hr] || (back >= 0 && back < 64 && t1 < at.seen && (bits[mt][hr] >> back & 1));
                                if (x == -INFINITY && (!sees || (gone >> (k >> 4) & 1))) continue;
                                const float weight = ex2(x - (m[mt][hr] == -INFINITY ? 0.f : m[mt][hr]));
#pragma unroll
                                for (int t = 0; t < DH / 8; ++t)
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        float v;
                                        if constexpr (E4M3)
                                            v = __half2float(__ushort_as_half((unsigned short)e4m3_to_f16(vt[stage_off<RB>(k, t >> 1) + 4 * (lane & 3) + 2 * e + (t & 1)]))) * vs;
                                        else
                                            v = bf16_bits_to_float(*reinterpret_cast<const uint16_t*>(vt + stage_off<RB>(k, t) + 2 * (2 * (lane & 3) + e)));
                                        o[mt][t][2 * hr + e] = fmaf(weight, v, o[mt][t][2 * hr + e]);
                                    }
                            }
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < GK; ++q)
#pragma unroll
                        for (int j = 0; j < RB / 32; ++j) {
                            uint32_t vb[4];
                            ldsm_x4_t(Vt + stage_off<RB>(16 * q + (lane & 15), 2 * j + (lane >> 4)), vb);
                            if constexpr (E4M3) {
#pragma unroll
                                for (int u = 0; u < 2; ++u)              // 16 dimensions, the even ones and the odd ones
#pragma unroll
                                    for (int b = 0; b < 2; ++b) {
                                        const uint32_t b0 = e4m3_to_bf16(vb[2 * u], b), b1 = e4m3_to_bf16(vb[2 * u + 1], b);
#pragma unroll
                                        for (int t = C::PT - 1; t >= 0; --t)
#pragma unroll
                                            for (int mt = 0; mt < MT; ++mt) mma_bf16(o[mt][4 * j + 2 * u + b], pa[mt][q][t], b0, b1);
                                    }
                            } else {
#pragma unroll
                                for (int t = C::PT - 1; t >= 0; --t)
#pragma unroll
                                    for (int mt = 0; mt < MT; ++mt) {
                                        mma_bf16(o[mt][2 * j], pa[mt][q][t], vb[0], vb[1]);
                                        mma_bf16(o[mt][2 * j + 1], pa[mt][q][t], vb[2], vb[3]);
                                    }
                            }
                        }
                }
            }
            slot = slot + 1 == NS ? 0 : slot + 1;
        }
        // ---- the item's rows over the warps: maxima and sums first, then MC dimensions at a time
        const int head0 = at.h * a.group;
        const bool whole = first_tile == 0 && item_end <= end;
        float* part = a.parts + ((size_t)blockIdx.x * 2 + (first_tile == 0 ? 1 : 0)) * C::PART;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int hr = 0; hr < 2; ++hr) {
                float sum = l[mt][hr];
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if ((lane & 3) == 0) {
                    const int r = 16 * mt + (lane >> 2) + 8 * hr;
                    row_m[warp * BR + r] = m[mt][hr];
                    row_l[warp * BR + r] = sum;
                }
            }
        __syncthreads();
        if (tid < BR) {
            float top = -INFINITY, sum = 0.f;
            for (int i = 0; i < PW; ++i) top = fmaxf(top, row_m[i * BR + tid]);
            for (int i = 0; i < PW; ++i) {
                const float f = top == -INFINITY ? 0.f : ex2(row_m[i * BR + tid] - top);
                sum += f * row_l[i * BR + tid];
                row_m[i * BR + tid] = f;                 // from here on: the warp's share of the item's rows
            }
            row_f[tid] = sum == 0.f ? 0.f : 1.f / sum;   // (a row that sees nothing is 0; NaN stays)
            if (!whole) { __stcg(part + BR * DH + tid, top); __stcg(part + BR * DH + BR + tid, sum); }
        }
        __syncthreads();
        auto put = [&](int r, int d, float4 v) {         // four neighbouring dimensions of the finished row r
            const int p = p0 + r;
            const size_t dst = (size_t)(at.q.start + p / a.group) * a.ldo + (size_t)(head0 + p % a.group) * DH + d;
            if constexpr (ROWS16) *reinterpret_cast<uint2*>((uint16_t*)a.out + dst) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
            else *reinterpret_cast<float4*>((float*)a.out + dst) = v;
        };
        // DIMS dimensions of the valid rows at a time, every warp's in its stage of the item's last tile, which the next request fills
        constexpr int DIMS = C::DIMS;
        unsigned char* const spare = smem + C::FIXED + (slot == 0 ? NS - 1 : slot - 1) * C::STAGE;
        auto rows_of = [&](int j) { return reinterpret_cast<float*>(spare + j * (NS * C::STAGE)); };
#pragma unroll
        for (int d0 = 0; d0 < DH; d0 += DIMS) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int hr = 0; hr < 2; ++hr) {
                    const int r = 16 * mt + (lane >> 2) + 8 * hr;
                    if (r >= nrows) continue;
                    const float f = row_m[warp * BR + r];
                    float* dst = rows_of(warp) + r * DIMS;
#pragma unroll
                    for (int t = d0 / 8; t < (d0 + DIMS) / 8; t += 2) {
                        const float a0 = o[mt][t][2 * hr] * f, a1 = o[mt][t][2 * hr + 1] * f, b0 = o[mt][t + 1][2 * hr] * f, b1 = o[mt][t + 1][2 * hr + 1] * f;
                        if constexpr (E4M3) {            // (accumulators t and t + 1: the even and the odd ones of 16)
                            *reinterpret_cast<float4*>(dst + 8 * t - d0 + 4 * (lane & 3)) = make_float4(a0, b0, a1, b1);
                        } else {
                            *reinterpret_cast<float2*>(dst + 8 * t - d0 + 2 * (lane & 3)) = make_float2(a0, a1);
                            *reinterpret_cast<float2*>(dst + 8 * t + 8 - d0 + 2 * (lane & 3)) = make_float2(b0, b1);
                        }
                    }
                }
            __syncthreads();
            constexpr int PER = DIMS / 4;
            for (int i = tid; i < nrows * PER; i += 32 * PW) {
                const int r = i / PER, c = i % PER * 4;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int j = 0; j < PW; ++j) {
                    const float4 x = *reinterpret_cast<const float4*>(rows_of(j) + r * DIMS + c);
                    v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
                }
                if (whole) {
                    const float f = row_f[r];
                    put(r, d0 + c, make_float4(v.x * f, v.y * f, v.z * f, v.w * f));
                } else {
                    __stcg(reinterpret_cast<float4*>(part + r * DH + d0 + c), v);
                }
            }
            if (d0 + DIMS < DH) __syncthreads();
        }
        if (!whole) {
            // ---- the last of the item's parts to arrive adds them up, in the order of their runs
            int c0, c1;
            S::parts_of(at, units, n_runs, snap, &c0, &c1);
            __threadfence();
            __syncthreads();
            if (tid == 0) s_last = atomicInc(a.tickets + c0, (unsigned)(c1 - c0)) == (unsigned)(c1 - c0);
            __syncthreads();
            if (s_last) {
                __threadfence();
                auto of = [&](int c) { return a.parts + ((size_t)c * 2 + (c == c0 ? 1 : 0)) * C::PART; };
                const int n_parts = c1 - c0 + 1;
                // a warp a row, a lane a part: the row's maximum and sum; then what each part counts, in a stage
                constexpr int MOST = DIMS;                       // parts at a time
                float* share = rows_of(0);
                for (int r = warp; r < nrows; r += PW) {
                    float top = -INFINITY, sum = 0.f;
                    for (int c = lane; c < n_parts; c += 32) top = fmaxf(top, __ldcg(of(c0 + c) + BR * DH + r));
                    top = warp_max(top);
                    if (top == -INFINITY) top = 0.f;
                    for (int c = lane; c < n_parts; c += 32) sum += ex2(__ldcg(of(c0 + c) + BR * DH + r) - top) * __ldcg(of(c0 + c) + BR * DH + BR + r);
                    sum = warp_sum(sum);
                    if (lane == 0) {
                        row_f[r] = sum == 0.f ? 0.f : 1.f / sum;
                        row_f[BR + r] = top;
                    }
                }
                constexpr int PER = DH / 4, EACH = (BR * PER + 32 * PW - 1) / (32 * PW);
                float4 v[EACH] = {};
                for (int b0 = 0; b0 < n_parts; b0 += MOST) {
                    const int nb = min(MOST, n_parts - b0);
                    __syncthreads();
                    for (int i = tid; i < nrows * nb; i += 32 * PW) {
                        const int r = i / nb, c = i % nb;
                        share[r * MOST + c] = ex2(__ldcg(of(c0 + b0 + c) + BR * DH + r) - row_f[BR + r]);
                    }
                    __syncthreads();
#pragma unroll (16 / EACH)
                    for (int c = 0; c < nb; ++c)                 // (16 loads of a thread under way)
#pragma unroll
                        for (int e = 0; e < EACH; ++e) {
                            const int i = tid + e * 32 * PW, r = i / PER, d = i % PER * 4;
                            if (i >= nrows * PER) continue;
                            const float f = share[r * MOST + c];
                            const float4 x = __ldcg(reinterpret_cast<const float4*>(of(c0 + b0 + c) + r * DH + d));
                            v[e].x += f * x.x; v[e].y += f * x.y; v[e].z += f * x.z; v[e].w += f * x.w;
                        }
                }
#pragma unroll
                for (int e = 0; e < EACH; ++e) {
                    const int i = tid + e * 32 * PW, r = i / PER, d = i % PER * 4;
                    if (i >= nrows * PER) continue;
                    const float f = row_f[r];
                    put(r, d, make_float4(v[e].x * f, v[e].y * f, v[e].z * f, v[e].w * f));
                }
            }
        }
        unit = at.unit_of(stop);
        if (unit < end) {
            at.tile = stop - 1;
            at.next(w, a.group, tree);
        }
    }
    cp_async_wait<0>();
}

template <int DH, int MT, bool ROWS16, bool E4M3>
static csd_status run_rows(const PagedView& w, const AttendArgs& a, cudaStream_t st) {
    using C = PagedRowsCfg<DH, MT, ROWS16, E4M3>;
    auto kern = paged_rows_kernel<DH, MT, ROWS16, E4M3>;
    static PerDevice ready;
    const csd_status ok = allow_smem(ready, kern, C::SMEM);
    if (ok != CSD_OK) return ok;
    PdlLaunch L(dim3((unsigned)tc_sm_count()), dim3(32 * C::PW), C::SMEM, st);
    CSD_CUDA(cudaLaunchKernelEx(&L.cfg, kern, w, a));
    count_launch();
    return CSD_OK;
}

// Which of them serves a call, by its sizes: f(integral constants DH, MT, ROWS16, E4M3).
template <class F> static auto pick_rows(int d_head, int packed_rows, int row_type, bool e4m3, F f) {
    auto four = [&](auto dh, auto mt) {
        constexpr int D = decltype(dh)::value, M = decltype(mt)::value;
        if (row_type == CSD_BF16) return e4m3 ? f.template operator()<D, M, true, true>() : f.template operator()<D, M, true, false>();
        return e4m3 ? f.template operator()<D, M, false, true>() : f.template operator()<D, M, false, false>();
    };
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    if (d_head == 64) return packed_rows <= 16 ? four(std::integral_constant<int, 64>(), One()) : four(std::integral_constant<int, 64>(), Two());
    return packed_rows <= 16 ? four(std::integral_constant<int, 128>(), One()) : four(std::integral_constant<int, 128>(), Two());
}

struct RowsRun {
    const PagedView& w; const AttendArgs& a; cudaStream_t st;
    template <int D, int M, bool R, bool E> csd_status operator()() const { return run_rows<D, M, R, E>(w, a, st); }
};

// (room for blocks of 32 rows, whichever a call takes: callers keep one workspace for batches of all lengths)
size_t paged_rows_workspace(int d_head) { return PAGED_TICKET_BYTES + (size_t)tc_sm_count() * 2 * 32 * (d_head + 2) * 4; }

csd_status launch_paged_rows(const PagedView& w, AttendArgs a, int d_head, int packed_rows, int row_type, void* workspace, cudaStream_t st) {
    a.tickets = (unsigned*)workspace;
    a.parts = (float*)((char*)workspace + PAGED_TICKET_BYTES);
    return pick_rows(d_head, packed_rows, row_type, w.k_exp != nullptr, RowsRun{w, a, st});
}

}  // namespace csd
