// Layer norm of rows, forward and backward, with the reduction of the gradients of weight and bias.
#include "common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRowBlocks = 65536;   // workgroups of the row kernels; more rows go round

// Sum over the workgroup, on every thread; `red` holds kThreads / kWave floats and is free again after the
// next barrier that the caller passes.
__device__ __forceinline__ float block_sum(float v, float *red) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    float s = red[0];
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) s += red[w];
    return s;
}

// One workgroup per row: mean, then the squares around it, then the row's values; the row is read three
// times, from the caches after the first.
template <typename TH, typename TX>
__global__ __launch_bounds__(kThreads) void k_ln_fwd(int64_t B, int64_t F, const TH *H, int64_t ldh,
                                                     const float *__restrict__ weight, const float *__restrict__ bias,
                                                     float eps, TX *X, int64_t ldx, float *__restrict__ mean,
                                                     float *__restrict__ rstd) {
    __shared__ float red[kThreads / kWave];
    for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
        const TH *h = H + b * ldh;
        TX *x = X + b * ldx;
        float s = 0.0f;
        for (int64_t f = threadIdx.x; f < F; f += kThreads) s += load_f32(h, f);
        const float mu = block_sum(s, red) / (float)F;
        float q = 0.0f;
        for (int64_t f = threadIdx.x; f < F; f += kThreads) {
            const float d = load_f32(h, f) - mu;
            q = __fmaf_rn(d, d, q);
        }
        const float rs = 1.0f / sqrtf(block_sum(q, red) / (float)F + eps);
        for (int64_t f = threadIdx.x; f < F; f += kThreads)
            store_out(x, f, __fmaf_rn((load_f32(h, f) - mu) * rs, weight ? weight[f] : 1.0f, bias ? bias[f] : 0.0f));
        if (mean && threadIdx.x == 0) {
            mean[b] = mu;
            rstd[b] = rs;
        }
    }
}

// One workgroup per row: both sums of the row, then its gradient.
template <typename TH, typename TD>
__global__ __launch_bounds__(kThreads) void k_ln_bwd(int64_t B, int64_t F, const TH *__restrict__ H, int64_t ldh,
                                                     const float *__restrict__ weight, const float *__restrict__ mean,
                                                     const float *__restrict__ rstd, const TD *dX, int64_t lddx, TH *dH,
                                                     int64_t lddh) {
    __shared__ float red[kThreads / kWave];
    for (int64_t b = blockIdx.x; b < B; b += gridDim.x) {
        const TH *h = H + b * ldh;
        const TD *d = dX + b * lddx;
        const float mu = mean[b], rs = rstd[b];
        float s = 0.0f, t = 0.0f;
        for (int64_t f = threadIdx.x; f < F; f += kThreads) {
            const float q = load_f32(d, f) * (weight ? weight[f] : 1.0f);
            s += q;
            t = __fmaf_rn(q, (load_f32(h, f) - mu) * rs, t);
        }
        s = block_sum(s, red) / (float)F;
        t = block_sum(t, red) / (float)F;
        for (int64_t f = threadIdx.x; f < F; f += kThreads) {
            const float q = load_f32(d, f) * (weight ? weight[f] : 1.0f), xh = (load_f32(h, f) - mu) * rs;
            store_out(dH + b * lddh, f, (q - s - xh * t) * rs);
        }
    }
}

// The rows are cut into `parts` runs; part[p][0][f] and part[p][1][f] are run p's sums of dX xh and of dX.  A
// workgroup takes 64 features of one run, each of its waves every fourth row.
template <typename TH, typename TD>
__global__ __launch_bounds__(kThreads) void k_ln_wgrad(int64_t B, int64_t F, const TH *__restrict__ H, int64_t ldh,
                                                       const float *__restrict__ mean, const float *__restrict__ rstd,
                                                       const TD *__restrict__ dX, int64_t lddx, int64_t per_part,
                                                       float *__restrict__ part) {
    __shared__ float sw[kThreads], sb[kThreads];
    const int64_t f = (int64_t)blockIdx.x * kWave + (threadIdx.x & (kWave - 1)), p = blockIdx.y;
    const int64_t b1 = (p + 1) * per_part < B ? (p + 1) * per_part : B;
    float w = 0.0f, c = 0.0f;
    if (f < F)
        for (int64_t b = p * per_part + threadIdx.x / kWave; b < b1; b += kThreads / kWave) {
            const float d = load_f32(dX + b * lddx, f);
            w = __fmaf_rn(d, (load_f32(H + b * ldh, f) - mean[b]) * rstd[b], w);
            c += d;
        }
    sw[threadIdx.x] = w;
    sb[threadIdx.x] = c;
    __syncthreads();
    if (threadIdx.x < kWave && f < F) {
#pragma unroll
        for (int r = 1; r < kThreads / kWave; ++r) {
            w += sw[threadIdx.x + r * kWave];
            c += sb[threadIdx.x + r * kWave];
        }
        part[(2 * p) * F + f] = w;
        part[(2 * p + 1) * F + f] = c;
    }
}

// dweight, dbias (either may be NULL) from the runs' sums, in ascending order
__global__ __launch_bounds__(kThreads) void k_ln_wsum(const float *__restrict__ part, int64_t parts, int64_t F,
                                                      float *__restrict__ dweight, float *__restrict__ dbias, int beta) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= 2 * F) return;
    float *out = i < F ? dweight : dbias;
    if (!out) return;
    out += i < F ? i : i - F;
    float s = 0.0f;
    for (int64_t p = 0; p < parts; ++p) s += part[p * 2 * F + i];
    *out = beta ? *out + s : s;
}

int64_t ln_parts(int64_t B) {
    const int64_t n = haste::cdiv(B, 64);
    return n < 256 ? n : 256;
}

// f(a value of the type that a dtype stands for)
template <typename F>
void with_type(int32_t dtype, F &&f) {
    if (dtype == HASTE_DTYPE_BF16) f(bf16_t{});
    else f(float{});
}

}  // namespace

namespace haste {

hipError_t ln_fwd(int64_t B, int64_t F, int32_t dtype_h, const void *H, int64_t ldh, const float *weight,
                  const float *bias, float eps, int32_t dtype_x, void *X, int64_t ldx, float *mean, float *rstd,
                  hipStream_t s) {
    const dim3 grid((unsigned)(B < kMaxRowBlocks ? B : kMaxRowBlocks));
    with_type(dtype_h, [&](auto th) {
        with_type(dtype_x, [&](auto tx) {
            typedef decltype(th) TH;
            typedef decltype(tx) TX;
            hipLaunchKernelGGL((k_ln_fwd<TH, TX>), grid, dim3(kThreads), 0, s, B, F, (const TH *)H, ldh, weight, bias, eps,
                               (TX *)X, ldx, mean, rstd);
        });
    });
    return hipGetLastError();
}

size_t ln_bwd_ws(int64_t B, int64_t F) { return (size_t)(ln_parts(B) * 2 * F * 4); }

hipError_t ln_bwd(int64_t B, int64_t F, int32_t dtype_h, const void *H, int64_t ldh, const float *weight,
                  const float *mean, const float *rstd, int32_t dtype_dx, const void *dX, int64_t lddx, void *dH,
                  int64_t lddh, float *dweight, float *dbias, int beta, void *ws, hipStream_t s) {
    const int64_t parts = ln_parts(B), per_part = cdiv(B, parts);
    float *part = (float *)ws;
    // the sums over rows first: dH may take dX's place
    with_type(dtype_h, [&](auto th) {
        with_type(dtype_dx, [&](auto td) {
            typedef decltype(th) TH;
            typedef decltype(td) TD;
            if (dweight || dbias) {
                hipLaunchKernelGGL((k_ln_wgrad<TH, TD>), dim3((unsigned)cdiv(F, kWave), (unsigned)parts), dim3(kThreads), 0,
                                   s, B, F, (const TH *)H, ldh, mean, rstd, (const TD *)dX, lddx, per_part, part);
                hipLaunchKernelGGL(k_ln_wsum, dim3((unsigned)cdiv(2 * F, kThreads)), dim3(kThreads), 0, s, part, parts, F,
                                   dweight, dbias, beta);
            }
            if (dH)
                hipLaunchKernelGGL((k_ln_bwd<TH, TD>), dim3((unsigned)(B < kMaxRowBlocks ? B : kMaxRowBlocks)),
                                   dim3(kThreads), 0, s, B, F, (const TH *)H, ldh, weight, mean, rstd, (const TD *)dX, lddx,
                                   (TH *)dH, lddh);
        });
    });
    return hipGetLastError();
}

}  // namespace haste
