// Verification of drafted tokens against given probabilities with given random numbers: a CTA a row.
#include "common.cuh"

namespace csd {

struct VerifyArgs {
    const void* p; const void* q; const int32_t* tokens; const int32_t* n_drafts; const float* u;
    int32_t* accepted; int32_t* out; int* status;
    long long ldp, ldq;
    int k, V;
};

template <bool LAW16>
__device__ __forceinline__ float law_at(const void* law, size_t i) {
    return LAW16 ? bf16_bits_to_float(((const uint16_t*)law)[i]) : ((const float*)law)[i];
}

// what an entry carries: positive finite numbers only
__device__ __forceinline__ double mass_of(double x) { return x > 0.0 && x < INFINITY ? x : 0.0; }
// entry j of what is left of p after a rejection
__device__ __forceinline__ double left_of(float p, float q) { return fmax(mass_of(p) - mass_of(q), 0.0); }

constexpr int VT = 1024;

template <bool LAW16>
__global__ void __launch_bounds__(VT)
verify_kernel(const VerifyArgs a) {
    __shared__ double part[VT];
    __shared__ double s_total;
    __shared__ int s_token;
    const int row = blockIdx.x, tid = threadIdx.x, V = a.V;
    int n = a.n_drafts ? a.n_drafts[row] : a.k;
    if (n < 0 || n > a.k) { if (tid == 0) set_status(a.status, CSD_ERR_INVALID_ARG); n = min(max(n, 0), a.k); }
    auto uniform = [&](int i) {
        const float u = a.u[(size_t)row * (a.k + 1) + i];
        if (!(u >= 0.f && u < 1.f)) { if (tid == 0) set_status(a.status, CSD_ERR_INVALID_ARG); return u >= 1.f ? 0.99999994f : 0.f; }
        return u;
    };
    int at = 0;
    for (; at < n; ++at) {
        const int x = a.tokens[(size_t)row * a.k + at];
        if (x < 0 || x >= V) { if (tid == 0) set_status(a.status, CSD_ERR_BAD_TOKEN); break; }
        const float px = law_at<LAW16>(a.p, ((size_t)row * (a.k + 1) + at) * a.ldp + x);
        const float qx = a.q ? law_at<LAW16>(a.q, ((size_t)row * a.k + at) * a.ldq + x) : 1.f;
        if (!((double)uniform(at) * (double)qx < (double)px)) break;
    }
    const size_t prow = ((size_t)row * (a.k + 1) + at) * a.ldp, qrow = ((size_t)row * a.k + at) * a.ldq;
    const int drop = at < n ? a.tokens[(size_t)row * a.k + at] : -1;
    const double u = uniform(a.k);
    const int per = (V + VT - 1) / VT, lo = min(tid * per, V), hi = min(lo + per, V);
    int token = 0;
    for (int mode = at < n ? 0 : 1; mode < 2; ++mode) {        // 0: what is left after a rejection, 1: the target's law
        auto entry = [&](int j) {
            const float p = law_at<LAW16>(a.p, prow + j);
            if (mode == 1) return mass_of(p);
            return a.q ? left_of(p, law_at<LAW16>(a.q, qrow + j)) : (j == drop ? 0.0 : mass_of(p));
        };
        double s = 0.0;
        for (int j = lo; j < hi; ++j) s += entry(j);
        part[tid] = s;
        if (tid == 0) s_token = 0;
        __syncthreads();
        if (tid == 0) {
            double run = 0.0;
            for (int i = 0; i < VT; ++i) { const double x = part[i]; part[i] = run; run += x; }
            s_total = run;
        }
        __syncthreads();
        if (s_total > 0.0) {
            const double target = u * s_total;
            double run = part[tid];
            if (run <= target && run + s > target)
                for (int j = lo; j < hi; ++j) {
                    run += entry(j);
                    if (run > target) { s_token = j; break; }
                }
            __syncthreads();
            token = s_token;
            break;
        }
        __syncthreads();
    }
    if (tid <= a.k) a.out[(size_t)row * (a.k + 1) + tid] = tid < at ? a.tokens[(size_t)row * a.k + tid] : tid == at ? token : -1;
    if (tid == 0) a.accepted[row] = at;
}

}  // namespace csd

using namespace csd;

extern "C" csd_status csd_spec_verify(const void* target_probs_dev, int64_t ld_p, const void* draft_probs_dev, int64_t ld_q, int prob_type,
                                      const int32_t* draft_tokens_dev, const int32_t* n_drafts_dev, const float* uniforms_dev, int rows,
                                      int k, int V, int32_t* n_accepted_dev, int32_t* tokens_dev, void* stream) {
    if (rows < 0 || k < 0 || k > 64 || V < 1 || (prob_type != CSD_F32 && prob_type != CSD_BF16)) return CSD_ERR_INVALID_ARG;
    if (rows == 0) return CSD_OK;
    if (!target_probs_dev || (k > 0 && !draft_tokens_dev) || !uniforms_dev || !n_accepted_dev || !tokens_dev) return CSD_ERR_INVALID_ARG;
    if (ld_p < V || (draft_probs_dev && ld_q < V)) return CSD_ERR_INVALID_ARG;
    VerifyArgs a{target_probs_dev, draft_probs_dev, draft_tokens_dev, n_drafts_dev, uniforms_dev, n_accepted_dev, tokens_dev,
                 status_word_device(), ld_p, ld_q, k, V};
    if (!a.status) return CSD_ERR_CUDA;
    if (prob_type == CSD_BF16) verify_kernel<true><<<rows, VT, 0, (cudaStream_t)stream>>>(a);
    else verify_kernel<false><<<rows, VT, 0, (cudaStream_t)stream>>>(a);
    CSD_CUDA(cudaGetLastError());
    count_launch();
    return CSD_OK;
}
