// Verification of drafted tokens against given probabilities with given random numbers.
//
// A row needs 2 k numbers for its tests and then one law, or two, of V entries: what is left of p after a rejection, max(0, p - q),
// summed in fp64 (the differences of fp32 numbers are exact there, and so are most sums), and the entry in which u of the
// whole falls.  A cluster of up to eight CTAs takes a row.  Every CTA makes the row's tests (a warp, a lane a draft), each warp sums a
// contiguous piece of the law, the warps' sums go to all CTAs through distributed shared memory, and the warp whose piece holds
// the target goes through it once more (from L2): lanes' stretches, then the stretch.  No workspace, one launch.
//
// What bounds it: many rows, the laws' bytes (256 rows of 128256 fp32 entries, most with a refused draft: 46 us, 77 % of the copy rate); one row, the
// chain of tests, sums, exchange and second look (32000 entries 6.0 us).
#include "tc_common.cuh"

namespace csd {

struct VerifyArgs {
    const void* p; const void* q; const int32_t* tokens; const int32_t* n_drafts; const float* u;
    int32_t* accepted; int32_t* out; int* status;
    long long ldp, ldq;
    int k, V;
};

constexpr int VW = 8, VMAX = 8;            // warps of a CTA, CTAs of a cluster at most
constexpr int VSUMS = VW * VMAX;

template <bool LAW16> __device__ __forceinline__ float law_at(const void* law, size_t i) {
    return LAW16 ? bf16_bits_to_float(((const uint16_t*)law)[i]) : ((const float*)law)[i];
}
// What is left of an entry, max(0, p - q), as a difference d in fp32 and what its rounding lost, e, so that d + e is exact: with
// y = min(p, max(q, 0)) the subtraction of the smaller from the larger leaves an error that (p - d) - y gives exactly.  Negative
// numbers and NaN count as 0.
struct Left { float d, e; };
__device__ __forceinline__ Left left_of(float p, float q) {
    const float x = fmaxf(p, 0.f), y = fminf(x, fmaxf(q, 0.f)), d = x - y;
    return Left{d, (x - d) - y};
}
// A lane's sum: the differences in fp64, their errors (2^-24 of them) in fp32.  Nine instructions an entry; with both numbers
// converted, or in pairs of fp32, the arithmetic bounds the pass.
struct Sum {
    double d = 0.0; float e = 0.f;
    __device__ __forceinline__ void add(const Left& x) { d += (double)x.d; e += x.e; }
    __device__ __forceinline__ double value() const { return d + (double)e; }
};

__device__ __forceinline__ double warp_scan(double x, int lane) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

template <bool LAW16>
__global__ void __launch_bounds__(32 * VW, 4)
verify_kernel(const VerifyArgs a) {
    __shared__ double sums[2][VSUMS];      // of both forms of the law: the warps of the cluster in their order
    __shared__ double stretch[VW];
    __shared__ int s_at, s_n;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, V = a.V, k = a.k;
    int ctas, rank;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ctas));
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int row = blockIdx.x / ctas;
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");      // (waited for before the first store to another CTA: all have begun)
    pdl_wait();
    pdl_trigger();
    const int32_t* tokens = a.tokens + (size_t)row * k;
    const float* uniforms = a.u + (size_t)row * (k + 1);
    auto uniform = [&](int i, bool tell) {
        const float u = uniforms[i];
        if (u >= 0.f && u < 1.f) return u;
        if (tell) set_status(a.status, CSD_ERR_INVALID_ARG);
        return u >= 1.f ? 0.99999994f : 0.f;
    };
    if (warp == 0) {
        int n = a.n_drafts ? a.n_drafts[row] : k;
        if (n < 0 || n > k) { set_status(a.status, CSD_ERR_INVALID_ARG); n = min(max(n, 0), k); }
        int at = n;
        for (int i0 = 0; i0 < n && at == n; i0 += 32) {
            const int i = i0 + lane;
            bool stop = false;
            if (i < n) {
                const int x = tokens[i];
                if (x < 0 || x >= V) {
                    stop = true;
                } else {
                    const float px = fmaxf(law_at<LAW16>(a.p, ((size_t)row * (k + 1) + i) * a.ldp + x), 0.f);      // (negative numbers and NaN: 0)
                    const float qx = a.q ? fmaxf(law_at<LAW16>(a.q, ((size_t)row * k + i) * a.ldq + x), 0.f) : 1.f;
                    stop = !((double)uniform(i, true) * (double)qx < (double)px);
                }
            }
            const unsigned any = __ballot_sync(0xffffffffu, stop);
            if (any) at = i0 + __ffs(any) - 1;
        }
        if (lane == 0) {
            s_at = at; s_n = n;
            if (at < n && (tokens[at] < 0 || tokens[at] >= V)) set_status(a.status, CSD_ERR_BAD_TOKEN);
        }
    }
    __syncthreads();
    const int at = s_at, n = s_n;
    const size_t prow = ((size_t)row * (k + 1) + at) * a.ldp, qrow = ((size_t)row * k + at) * a.ldq;
    const int drop = at < n ? tokens[at] : -1;
    const double u = (double)uniform(k, tid == 0);
    // this warp's piece of the vocabulary: warps of the cluster in order, pieces from multiples of 8 entries on
    const int all = ctas * VW, mine = rank * VW + warp;
    auto piece = [&](int i) { return i >= all ? V : (int)((long long)i * V / all) & ~7; };
    const int lo = piece(mine), hi = piece(mine + 1);
    int32_t* out = a.out + (size_t)row * (k + 1);
    if (rank == 0) {
        if (tid <= k && tid != at) out[tid] = tid < at ? tokens[tid] : -1;
        if (tid == 0) a.accepted[row] = at;
    }
    asm volatile("barrier.cluster.wait;" ::: "memory");
    for (int mode = at < n ? (a.q ? 0 : 1) : 2;; mode = 2) {     // p less q, p without the draft, p
        // eight entries from `first` on, `step` apart, those before `end`; infinities carry nothing
        auto eight = [&](int first, int step, int end, double (&v)[8]) {
            float p[8], q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = first + i * step;
                p[i] = j < end ? law_at<LAW16>(a.p, prow + j) : 0.f;
                q[i] = mode == 0 && j < end ? law_at<LAW16>(a.q, qrow + j) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = p[i] < INFINITY && !(mode == 1 && first + i * step == drop) ? p[i] : 0.f;
                const Left l = left_of(x, q[i]);
                v[i] = (double)l.d + (double)l.e;
            }
        };
        // 16 bytes a lane and load where both laws lie on such boundaries, four loads of each in flight
        constexpr int EACH = LAW16 ? 8 : 4, SIZE = LAW16 ? 2 : 4;
        Sum part;
        int from = lo;
        const char* pw = (const char*)a.p + (prow + lo) * SIZE;
        const char* qw = mode == 0 ? (const char*)a.q + (qrow + lo) * SIZE : pw;
        if (((((uintptr_t)pw) | ((uintptr_t)qw)) & 15) == 0) {
            const int loads = (hi - lo) / (128 * EACH) * 4;
#pragma unroll 1
            for (int b0 = 0; b0 < loads; b0 += 4) {
                uint4 p[4], q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = __ldg(reinterpret_cast<const uint4*>(pw) + (b0 + i) * 32 + lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = mode == 0 ? __ldg(reinterpret_cast<const uint4*>(qw) + (b0 + i) * 32 + lane) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int first = lo + ((b0 + i) * 32 + lane) * EACH;
                    const uint32_t x[4] = {p[i].x, p[i].y, p[i].z, p[i].w}, y[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
                    if (mode == 1 && (unsigned)(drop - first) < (unsigned)EACH) continue;        // (added below, without the draft)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (LAW16) {
                            part.add(left_of(bf16lo(x[e]), bf16lo(y[e])));
                            part.add(left_of(bf16hi(x[e]), bf16hi(y[e])));
                        } else {
                            part.add(left_of(__uint_as_float(x[e]), __uint_as_float(y[e])));
                        }
                    }
                }
            }
            from += loads * 32 * EACH;
        }
        double mass = part.value();
        auto add_up = [&](int first, int end) {
            for (int j = first + lane; j < end; j += 256) {
                double v[8];
                eight(j, 32, end, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) mass += v[i];
            }
        };
        if (mode == 1 && drop >= lo && drop < from) {                    // the load that was left out
            const int first = lo + (drop - lo) / EACH * EACH;
            add_up(first, first + EACH);
        }
        add_up(from, hi);
        double sum = warp_sum(mass);
        if (!(sum < INFINITY)) {                                         // an infinite entry
            mass = 0.0;
            add_up(lo, hi);
            sum = warp_sum(mass);
        }
        const int form = mode == 2 ? 1 : 0;
        if (lane < ctas) {
            const uint32_t there = map_to_cta(smem_u32(&sums[form][mine]), (uint32_t)lane);
            asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(there), "d"(sum) : "memory");
        }
        cluster_barrier();
        // every warp: where the pieces begin, two a lane, the whole, and the piece that holds the target: the last one with any mass that begins
        // at or before it.  (Pieces that end before the target would do if sums were exact.  But a lane adds to the scan's
        // sum, and the scan's next sum is added up in another order: the end of an empty piece can lie a rounding above the one before, and
        // with the target between the two nothing would be chosen.)
        double start[VSUMS / 32], run = 0.0;
        bool some_of[VSUMS / 32];
#pragma unroll
        for (int i = 0; i < VSUMS / 32; ++i) {
            const int w = lane * (VSUMS / 32) + i;
            const double x = w < all ? sums[form][w] : 0.0;
            some_of[i] = x > 0.0;
            start[i] = run;
            run += x;
        }
        const double upto = warp_scan(run, lane), before = __shfl_up_sync(0xffffffffu, upto, 1);
        const double base = lane ? before : 0.0;
        const double total = __shfl_sync(0xffffffffu, base + run, 31);
        if (!(total > 0.0)) {
            if (mode != 2) continue;                 // nothing is left: the target's own law
            if (rank == 0 && tid == 0) out[at] = 0;
            break;
        }
        const double target = u * total;
        int chosen = 0;                              // (the first piece with mass begins at 0)
#pragma unroll
        for (int i = 0; i < VSUMS / 32; ++i) {
            start[i] += base;
            if (some_of[i] && start[i] <= target) chosen = lane * (VSUMS / 32) + i;
        }
        chosen = __reduce_max_sync(0xffffffffu, chosen);
        if (chosen / VW != rank) break;              // (the same for all warps of a CTA)
        double left = 0.0;                           // in front of the piece
#pragma unroll
        for (int i = 0; i < VSUMS / 32; ++i) {
            const double e = __shfl_sync(0xffffffffu, start[i], chosen / (VSUMS / 32));
            if (chosen % (VSUMS / 32) == i) left = e;
        }
        // The CTA's warps take a stretch of that piece each, in up to 32 blocks: a block's entries are summed side by side, lane b
        // keeps the sum of block b.  Then the block that holds the target, a few neighbours a lane.  Where another order of the sums leaves
        // the target behind the last entry, it is the last entry that carries anything.
        const int f0 = piece(chosen), len = piece(chosen + 1) - f0;
        const int g0 = f0 + (int)((long long)warp * len / VW), g1 = f0 + (int)((long long)(warp + 1) * len / VW);
        const int block = ((g1 - g0 + 8191) / 8192) * 256;
        double s = 0.0;
        for (int b = 0; g0 + b * block < g1; ++b) {
            mass = 0.0;
            add_up(g0 + b * block, min(g0 + (b + 1) * block, g1));
            const double x = warp_sum(mass);
            if (lane == b) s = x;
        }
        double upto_block = warp_scan(s, lane);
        if (lane == 31) stretch[warp] = upto_block;
        __syncthreads();
        double want = target - left;
        int pick = -1, some = 0;
        for (int i = 0; i < VW; ++i) {
            const double x = stretch[i];
            if (x > 0.0) some = i;
            if (pick < 0) {
                if (x > want) pick = i; else want -= x;
            }
        }
        if (pick < 0) { pick = some; want = INFINITY; }
        if (pick != warp) break;
        auto choose = [&](double upto_lane, double mine_sum) {           // the lane whose share holds the target, and what lies in front of it
            const unsigned here = __ballot_sync(0xffffffffu, upto_lane > want && mine_sum > 0.0), any = __ballot_sync(0xffffffffu, mine_sum > 0.0);
            const int winner = here ? __ffs(here) - 1 : 31 - __clz(any);
            if (!here) want = INFINITY;
            want -= __shfl_sync(0xffffffffu, upto_lane - mine_sum, winner);
            return winner;
        };
        const int b = choose(upto_block, s), h0 = g0 + b * block, h1 = min(h0 + block, g1);
        const int b0 = min(h0 + lane * (block / 32), h1), b1 = min(b0 + block / 32, h1);
        s = 0.0;
        double v[8];
        for (int i = b0; i < b1; i += 8) {
            eight(i, 1, b1, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[e];
        }
        const int winner = choose(warp_scan(s, lane), s);
        if (lane == winner) {
            double reached = 0.0;
            int token = b0;
            bool found = false;
            for (int i = b0; i < b1 && !found; i += 8) {
                eight(i, 1, b1, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (found || !(v[e] > 0.0)) continue;
                    token = i + e;
                    reached += v[e];
                    found = reached > want;
                }
            }
            out[at] = token;
        }
        break;
    }
}

// CTAs a row: as many as the vocabulary fills (2048 entries each) and as leave every row of the call resident at four CTAs an SM.
static int verify_cluster(int rows, int V) {
    int n = 1;
    while (n < VMAX && n * 2048 < V && (long long)rows * n * 2 <= 4ll * tc_sm_count()) n *= 2;
    return n;
}

template <bool LAW16> static csd_status launch_verify(const VerifyArgs& a, int rows, cudaStream_t st) {
    const int ctas = verify_cluster(rows, a.V);
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)rows * ctas); cfg.blockDim = dim3(32 * VW); cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    CSD_CUDA(cudaLaunchKernelEx(&cfg, verify_kernel<LAW16>, a));
    count_launch();
    return CSD_OK;
}

}  // namespace csd

using namespace csd;

extern "C" csd_status csd_spec_verify(const void* target_probs_dev, int64_t ld_p, const void* draft_probs_dev, int64_t ld_q, int prob_type,
                                      const int32_t* draft_tokens_dev, const int32_t* n_drafts_dev, const float* uniforms_dev, int rows,
                                      int k, int V, int32_t* n_accepted_dev, int32_t* tokens_dev, void* stream) {
    if (rows < 0 || rows > 1 << 24 || k < 0 || k > 64 || V < 1 || V > 1 << 30 || (prob_type != CSD_F32 && prob_type != CSD_BF16)) return CSD_ERR_INVALID_ARG;
    if (rows == 0) return CSD_OK;
    if (!target_probs_dev || (k > 0 && !draft_tokens_dev) || !uniforms_dev || !n_accepted_dev || !tokens_dev) return CSD_ERR_INVALID_ARG;
    if (ld_p < V || (draft_probs_dev && ld_q < V)) return CSD_ERR_INVALID_ARG;
    if (((uintptr_t)target_probs_dev | (uintptr_t)draft_probs_dev) & (prob_type == CSD_BF16 ? 1 : 3)) return CSD_ERR_INVALID_ARG;
    VerifyArgs a{target_probs_dev, draft_probs_dev, draft_tokens_dev, n_drafts_dev, uniforms_dev, n_accepted_dev, tokens_dev,
                 status_word_device(), ld_p, ld_q, k, V};
    if (!a.status) return CSD_ERR_CUDA;
    return prob_type == CSD_BF16 ? launch_verify<true>(a, rows, (cudaStream_t)stream) : launch_verify<false>(a, rows, (cudaStream_t)stream);
}
