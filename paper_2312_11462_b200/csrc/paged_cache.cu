// Writing rows into the paged cache, in 16 or 8 bits, and reading them back.
//
// A row of one position and head is quantised by the lanes that hold it: max|x| by a shuffle among them, the scale's exponent
// from the maximum's bits (of finite entries; max|x| = m * 2^x with m in [1, 2): 448 = 1.75 * 2^8, so e = x - 8, one more where m > 1.75), then
// rn_e4m3(x * 2^-e).  The scale is a power of two, so x * 2^-e is exact and the result does not depend on how it is formed.
//
// A thread holds 8 neighbouring elements of one row, d_head / 8 threads a row, K and V of a head side by side; a warp belongs to
// one position and looks it up once.  What bounds both directions is the row traffic: some 10500 positions of 32 heads x 128, bf16 to 8 bits and
// back, 103 us, 77 % of the copy rate; reading 37500 positions of 8 heads alone 40 us, 88 %.
#include "paged_attention.cuh"
#include "tc_common.cuh"
#include <cuda_fp8.h>

namespace csd {

struct RowsView {
    const void* k; const void* v; long long ld;
    RopeView rope; const unsigned long long* tree;       // (append alone, fp32 rows: the model's keys are turned on their way)
};

// Sequence that row r of the batch belongs to, and the row's position (and its number in the chunk and the chunk's rows); false: to none.  Whole warps.
__device__ __forceinline__ bool find_row(const PagedView& w, int r, int* seq, int* pos, int* row = nullptr, int* rows = nullptr) {
    const int lane = threadIdx.x & 31;
    int s = 0;
    for (int b = 0; b < w.n_seqs; b += 32) {
        const bool past = b + lane < w.n_seqs && w.row_start[b + lane + 1] <= r;
        const int n = __popc(__ballot_sync(0xffffffffu, past));
        s += n;
        if (n < 32) break;
    }
    if (s >= w.n_seqs) return false;
    const PagedSeq q = paged_seq(w, s);
    *seq = s; *pos = q.kv + r - q.start;
    if (row) { *row = r - q.start; *rows = q.rows; }
    return r >= q.start && r - q.start < q.rows;
}

template <bool BF16>
__device__ __forceinline__ void load8(const void* p, float* x) {
    if constexpr (BF16) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        x[0] = bf16lo(u.x); x[1] = bf16hi(u.x); x[2] = bf16lo(u.y); x[3] = bf16hi(u.y);
        x[4] = bf16lo(u.z); x[5] = bf16hi(u.z); x[6] = bf16lo(u.w); x[7] = bf16hi(u.w);
    } else {
        const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}

__device__ __forceinline__ uint4 pack8_bf16(const float* x) {
    auto two = [](float a, float b) { return (uint32_t)float_to_bf16_bits(a) | (uint32_t)float_to_bf16_bits(b) << 16; };
    return make_uint4(two(x[0], x[1]), two(x[2], x[3]), two(x[4], x[5]), two(x[6], x[7]));
}

template <bool BF16>
__device__ __forceinline__ void store8(void* p, const float* x) {
    if constexpr (BF16) {
        *reinterpret_cast<uint4*>(p) = pack8_bf16(x);
    } else {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// A position's pieces of eight elements: [head][K, V][column], a stretch of 32 a warp and turn.  `split` warps share a position, each
// takes every split-th stretch, BATCH of them at a time with their loads in flight together.  A lane keeps its half and column and
// moves from head to head.
constexpr int BATCH = 4;
template <int DH> struct Lane {
    static constexpr int PER = DH / 8, HEADS = 32 / (2 * PER);           // lanes of a row, heads of a stretch
    int which, col, head;
    __device__ __forceinline__ Lane(int lane, int stretch) : which(lane / PER & 1), col(lane % PER * 8), head(stretch * HEADS + lane / (2 * PER)) {}
};

__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

template <int DH, bool ROWS16, bool E4M3>
__global__ void __launch_bounds__(256)
paged_append_kernel(const PagedView w, const RowsView src, int split) {
    pdl_wait();
    pdl_trigger();
    const int gw = (int)(blockIdx.x * 8 + (threadIdx.x >> 5)), r = gw / split, lane = threadIdx.x & 31;
    if (r >= w.total_rows) return;
    const Lane<DH> p(lane, gw % split);
    const int next = split * Lane<DH>::HEADS;                            // heads from one of the warp's stretches to its next
    constexpr int SIZE = ROWS16 ? 2 : 4;
    const char* from = (const char*)(p.which ? src.v : src.k) + ((size_t)r * src.ld + (size_t)p.head * DH + p.col) * SIZE;
    unsigned char* to = nullptr;
    uint8_t* to_exp = nullptr;
    int turn = 0;
    bool looked = false;
    for (int h0 = 0; h0 + gw % split * Lane<DH>::HEADS < w.heads; h0 += BATCH * next) {
        float x[BATCH][8] = {};
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (h0 + b * next + p.head < w.heads) load8<ROWS16>(from + (size_t)(h0 + b * next) * DH * SIZE, x[b]);
        if (!looked) {                                               // (the first loads are under way)
            int seq, pos, i, rows;
            if (!find_row(w, r, &seq, &pos, &i, &rows)) return;
            if (!ROWS16 && src.rope.cos) turn = rope_position(w, src.rope, pos - i, i, rows, src.tree ? src.tree + r : nullptr);
            const int page = paged_page(w, seq, pos);
            if (page < 0) return;
            const size_t row = paged_row(w, page, p.head, pos);      // (of a head that may not exist: not written)
            to = const_cast<unsigned char*>(p.which ? w.v : w.k) + (row * DH + p.col) * (E4M3 ? 1 : 2);
            if (E4M3) to_exp = const_cast<uint8_t*>(p.which ? w.v_exp : w.k_exp) + row;
            looked = true;
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const bool live = h0 + b * next + p.head < w.heads;
            const size_t on = (size_t)(h0 + b * next) << w.page_shift;           // rows of the pool from the lane's first head
            if (!ROWS16 && src.rope.cos) {                           // (the dimensions half a row away are DH / 16 lanes on)
                float other[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) other[i] = __shfl_xor_sync(0xffffffffu, x[b][i], DH / 16);
                if (live && !p.which) rope8(src.rope, turn, DH / 2, p.col, x[b], other);
            }
            if constexpr (!E4M3) {
                if (live) *reinterpret_cast<uint4*>(to + on * (DH * 2)) = pack8_bf16(x[b]);
            } else {
                float top = fabsf(x[b][0]);
#pragma unroll
                for (int i = 1; i < 8; ++i) top = max_nan(top, fabsf(x[b][i]));
#pragma unroll
                for (int o = DH / 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
                if (__any_sync(0xffffffffu, top == INFINITY)) {      // the largest finite entry counts
                    float finite = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) finite = fmaxf(finite, fabsf(x[b][i]) < INFINITY ? fabsf(x[b][i]) : 0.f);
#pragma unroll
                    for (int o = DH / 16; o > 0; o >>= 1) finite = fmaxf(finite, __shfl_xor_sync(0xffffffffu, finite, o));
                    if (top == INFINITY) top = finite;
                }
                const unsigned bits = __float_as_uint(top);
                const bool nan = top != top;
                const int e = nan ? 127 : max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 27);        // exponent of the scale + 127
                if (e == 247) {                                      // (up to 240 * 2^120: the next number, 2^128, is none in fp32)
                    const float most = __uint_as_float(0x7f700000u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[b][i] = x[b][i] > most ? most : x[b][i] < -most ? -most : x[b][i];
                }
                const float inv = __uint_as_float((unsigned)(254 - e) << 23);
                uint32_t out[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float* y = x[b] + 4 * i;
                    const __nv_fp8x2_storage_t f = __nv_cvt_float2_to_fp8x2(make_float2(y[0] * inv, y[1] * inv), __NV_SATFINITE, __NV_E4M3);
                    const __nv_fp8x2_storage_t g = __nv_cvt_float2_to_fp8x2(make_float2(y[2] * inv, y[3] * inv), __NV_SATFINITE, __NV_E4M3);
                    out[i] = (uint32_t)f | (uint32_t)g << 16;
                }
                if (live) {
                    *reinterpret_cast<uint2*>(to + on * DH) = make_uint2(out[0], out[1]);
                    if (p.col == 0) to_exp[on] = (uint8_t)(nan ? 255 : e);
                }
            }
        }
    }
}

template <int DH, bool ROWS16, bool E4M3>
__global__ void __launch_bounds__(256)
paged_read_kernel(const PagedView w, const RowsView dst, int split) {
    pdl_wait();
    pdl_trigger();
    const int gw = (int)(blockIdx.x * 8 + (threadIdx.x >> 5)), r = gw / split, lane = threadIdx.x & 31;
    if (r >= w.total_rows) return;
    const Lane<DH> p(lane, gw % split);
    const int next = split * Lane<DH>::HEADS;
    constexpr int SIZE = ROWS16 ? 2 : 4;
    char* to = (char*)const_cast<void*>(p.which ? dst.v : dst.k) + ((size_t)r * dst.ld + (size_t)p.head * DH + p.col) * SIZE;
    int seq, pos;
    if (!find_row(w, r, &seq, &pos)) return;
    const int page = paged_page(w, seq, pos);
    const size_t row = page >= 0 ? paged_row(w, page, p.head, pos) : 0;
    const unsigned char* from = (p.which ? w.v : w.k) + (row * DH + p.col) * (E4M3 ? 1 : 2);
    const uint8_t* from_exp = E4M3 ? (p.which ? w.v_exp : w.k_exp) + row : nullptr;
    for (int h0 = 0; h0 + p.head < w.heads; h0 += BATCH * next) {
        uint4 raw[BATCH];
        unsigned e[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            raw[b] = make_uint4(0u, 0u, 0u, 0u);
            e[b] = 127u;
            if (h0 + b * next + p.head >= w.heads || page < 0) continue;
            const size_t on = (size_t)(h0 + b * next) << w.page_shift;
            if constexpr (E4M3) {
                const uint2 u = *reinterpret_cast<const uint2*>(from + on * DH);
                raw[b].x = u.x; raw[b].y = u.y;
                e[b] = from_exp[on];
            } else {
                raw[b] = *reinterpret_cast<const uint4*>(from + on * (DH * 2));
            }
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            if (h0 + b * next + p.head >= w.heads) continue;
            float x[8];
            if constexpr (E4M3) {
                const float scale = row_scale(e[b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __half2 h(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((i < 2 ? raw[b].x : raw[b].y) >> 16 * (i & 1)), __NV_E4M3));
                    const float2 f = __half22float2(h);
                    x[2 * i] = f.x * scale; x[2 * i + 1] = f.y * scale;
                }
            } else {
                load8<true>(&raw[b], x);
            }
            store8<ROWS16>(to + (size_t)(h0 + b * next) * DH * SIZE, x);
        }
    }
}

template <template <int, bool, bool> class Pick>
static csd_status launch_cache(const PagedView& w, const RowsView& rows, int d_head, bool rows16, cudaStream_t st) {
    // warps a position: all its stretches at once while that leaves SMs idle, down to one, which looks up where the position lies
    // once for all of them (10500 positions of 32 heads x 128, bf16 to 8 bits and back: 184 us with a warp a stretch, 149 so)
    const int stretches = (2 * w.heads * (d_head / 8) + 31) / 32;
    int split = stretches;
    while (split > 1 && (long long)w.total_rows * ((split + 1) / 2) >= 48ll * tc_sm_count()) split = (split + 1) / 2;
    const long long warps = (long long)w.total_rows * split, blocks = (warps + 7) / 8;
    if (warps >= 1ll << 31) return CSD_ERR_INVALID_ARG;
    PdlLaunch L(dim3((unsigned)blocks), dim3(256), 0, st);
    auto go = [&](auto kern) { return cudaLaunchKernelEx(&L.cfg, kern, w, rows, split); };
    const bool e4m3 = w.k_exp != nullptr;
    cudaError_t e;
    if (d_head == 64)
        e = rows16 ? (e4m3 ? go(Pick<64, true, true>::kernel) : go(Pick<64, true, false>::kernel))
                   : (e4m3 ? go(Pick<64, false, true>::kernel) : go(Pick<64, false, false>::kernel));
    else
        e = rows16 ? (e4m3 ? go(Pick<128, true, true>::kernel) : go(Pick<128, true, false>::kernel))
                   : (e4m3 ? go(Pick<128, false, true>::kernel) : go(Pick<128, false, false>::kernel));
    CSD_CUDA(e);
    count_launch();
    return CSD_OK;
}

template <int DH, bool R, bool E> struct AppendPick { static constexpr auto kernel = paged_append_kernel<DH, R, E>; };
template <int DH, bool R, bool E> struct ReadPick { static constexpr auto kernel = paged_read_kernel<DH, R, E>; };

template <template <int, bool, bool> class Pick>
static csd_status run_cache(const csd_kv_pool* pool, const csd_paged_batch* batch, const void* k, const void* v, int64_t ld,
                            int row_type, const RopeView& rope, const unsigned long long* tree, void* stream) {
    PagedView w;
    const csd_status ok = paged_view(pool, batch, &w);
    if (ok != CSD_OK) return ok;
    const int64_t width = (int64_t)pool->n_kv_heads * pool->d_head;
    if (row_type != CSD_F32 && row_type != CSD_BF16) return CSD_ERR_INVALID_ARG;
    if (w.total_rows == 0) return CSD_OK;
    if (!paged_rows_ok(k, ld, width) || !paged_rows_ok(v, ld, width)) return CSD_ERR_INVALID_ARG;
    w.status = status_word_device();
    if (!w.status) return CSD_ERR_CUDA;
    return launch_cache<Pick>(w, RowsView{k, v, ld, rope, tree}, pool->d_head, row_type == CSD_BF16, (cudaStream_t)stream);
}

csd_status paged_append_turned(const csd_kv_pool* pool, const csd_paged_batch* batch, const float* k, const float* v, int64_t ld, const RopeView& rope,
                               const unsigned long long* tree, void* stream) {
    return run_cache<AppendPick>(pool, batch, k, v, ld, CSD_F32, rope, tree, stream);
}

}  // namespace csd

using namespace csd;

extern "C" csd_status csd_paged_append(const csd_kv_pool* pool, const csd_paged_batch* batch, const void* k_dev, const void* v_dev,
                                       int64_t ld, int row_type, void* stream) {
    return run_cache<AppendPick>(pool, batch, k_dev, v_dev, ld, row_type, RopeView{}, nullptr, stream);
}

extern "C" csd_status csd_paged_read(const csd_kv_pool* pool, const csd_paged_batch* batch, void* k_dev, void* v_dev, int64_t ld,
                                     int row_type, void* stream) {
    return run_cache<ReadPick>(pool, batch, k_dev, v_dev, ld, row_type, RopeView{}, nullptr, stream);
}
