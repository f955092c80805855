// Layer norm of rows, forward and backward, with the reduction of the gradients of weight and bias.
//
// A row belongs to a team of 16, 64, 256 or 1024 threads, which hold it in registers: every value is read once
// and every sum is taken from the registers, the squares around the row's mean.  A thread holds NC runs of
// four consecutive values, TEAM runs apart.  Rows wider than kWideF go through a loop that reads them again.
#include "common.hpp"

namespace {

// ---- four consecutive values, at any alignment of their elements ----------------------------------
template <typename T>
struct Raw4 {
    uint32_t w[sizeof(T)];
};
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
// (the hardware takes vector accesses at any element's address)
typedef u32x4_t u32x4_el_t __attribute__((aligned(4)));
typedef u32x2_t u32x2_el_t __attribute__((aligned(2)));

// n values of the four are there; the others read as zero
__device__ __forceinline__ Raw4<float> load4(const float *p, int64_t n) {
    Raw4<float> r = {};
    if (n >= 4) {
        const u32x4_t v = *reinterpret_cast<const u32x4_el_t *>(p);
        r.w[0] = v.x, r.w[1] = v.y, r.w[2] = v.z, r.w[3] = v.w;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) r.w[j] = __float_as_uint(p[j]);
    }
    return r;
}
__device__ __forceinline__ Raw4<bf16_t> load4(const bf16_t *p, int64_t n) {
    Raw4<bf16_t> r = {};
    if (n >= 4) {
        const u32x2_t v = *reinterpret_cast<const u32x2_el_t *>(p);
        r.w[0] = v.x, r.w[1] = v.y;
    } else {
        if (n > 0) r.w[0] = p[0];
        if (n > 1) r.w[0] |= (uint32_t)p[1] << 16;
        if (n > 2) r.w[1] = p[2];
    }
    return r;
}
__device__ __forceinline__ void unpack4(const Raw4<float> &r, float (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(r.w[j]);
}
__device__ __forceinline__ void unpack4(const Raw4<bf16_t> &r, float (&v)[4]) {
    v[0] = __uint_as_float(r.w[0] << 16), v[1] = __uint_as_float(r.w[0] & 0xffff0000u);
    v[2] = __uint_as_float(r.w[1] << 16), v[3] = __uint_as_float(r.w[1] & 0xffff0000u);
}
__device__ __forceinline__ void store4(float *p, const float (&v)[4], int64_t n) {
    if (n >= 4) {
        const u32x4_t w = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        *reinterpret_cast<u32x4_el_t *>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) p[j] = v[j];
    }
}
__device__ __forceinline__ void store4(bf16_t *p, const float (&v)[4], int64_t n) {
    if (n >= 4) {
        const u32x2_t w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        *reinterpret_cast<u32x2_el_t *>(p) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) p[j] = f32_to_bf16(v[j]);
    }
}

// ---- sums over a team -------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    const int s = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true);
    return v + __builtin_bit_cast(float, s);
}
// over 16 lanes, on each of them: neighbours, pairs, then the halves and quarters mirrored
__device__ __forceinline__ float sum16(float v) {
    v = dpp_add<0xB1>(v);    // lanes 1 0 3 2
    v = dpp_add<0x4E>(v);    // lanes 2 3 0 1
    v = dpp_add<0x141>(v);   // mirrored in 8
    return dpp_add<0x140>(v);   // mirrored in 16
}
__device__ __forceinline__ float sum64(float v) {
    const int r = __builtin_bit_cast(int, sum16(v));
    const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(r, 0));
    const float b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(r, 16));
    const float c = __builtin_bit_cast(float, __builtin_amdgcn_readlane(r, 32));
    const float d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(r, 48));
    return (a + b) + (c + d);
}

// N sums at once.  Teams of more than one wave meet in LDS, in `red` ([2][16][N] floats a workgroup), whose
// halves are used in turn (`turn`), so that one barrier a call is enough; every thread of the workgroup calls.
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float *red, int &turn) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = TEAM == 16 ? sum16(v[k]) : sum64(v[k]);
    if constexpr (TEAM > kWave) {
        constexpr int W = TEAM / kWave;
        const int wave = threadIdx.x / kWave, first = wave / W * W;
        float *half = red + turn * 16 * N;
        turn ^= 1;
        if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) half[wave * N + k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = half[first * N + k];
#pragma unroll
            for (int w = 1; w < W; ++w) v[k] += half[(first + w) * N + k];
        }
    }
}

// ---- forward ----------------------------------------------------------------------------------------
template <typename TH, typename TX, int TEAM, int NC>
__global__ __launch_bounds__(TEAM > 256 ? TEAM : 256) void k_ln_fwd(int64_t B, int F, const TH *H, int64_t ldh,
                                                                    const float *__restrict__ weight,
                                                                    const float *__restrict__ bias, float eps, TX *X,
                                                                    int64_t ldx, float *__restrict__ mean,
                                                                    float *__restrict__ rstd) {
    __shared__ float red[2 * 16];
    int turn = 0;
    const int t = threadIdx.x % TEAM;
    const int64_t teams = blockDim.x / TEAM;
    float w[NC][4], c[NC][4];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int f = 4 * (i * TEAM + t);
        unpack4(load4(weight + f, weight ? F - f : 0), w[i]);
        unpack4(load4(bias + f, bias ? F - f : 0), c[i]);
        if (!weight)
            for (int j = 0; j < 4; ++j) w[i][j] = 1.0f;
    }
    // every team of a workgroup goes round as often as the first one, for the barriers
    for (int64_t b0 = blockIdx.x * teams; b0 < B; b0 += gridDim.x * teams) {
        const int64_t b = b0 + threadIdx.x / TEAM;
        const bool in = b < B;
        const TH *h = H + (in ? b : b0) * ldh;
        float v[NC][4], s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int f = 4 * (i * TEAM + t);
            unpack4(load4(h + f, F - f), v[i]);
        }
#pragma unroll
        for (int i = 0; i < NC; ++i) s[0] += (v[i][0] + v[i][1]) + (v[i][2] + v[i][3]);
        team_sum<TEAM>(s, red, turn);
        const float mu = s[0] / (float)F;
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int f = 4 * (i * TEAM + t);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[i][j] = f + j < F ? v[i][j] - mu : 0.0f;
                s[0] = __fmaf_rn(v[i][j], v[i][j], s[0]);
            }
        }
        team_sum<TEAM>(s, red, turn);
        const float rs = 1.0f / sqrtf(s[0] / (float)F + eps);
        if (in) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int f = 4 * (i * TEAM + t);
                float o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = __fmaf_rn(v[i][j] * rs, w[i][j], c[i][j]);
                store4(X + b * ldx + f, o, F - f);
            }
            if (mean && t == 0) {
                mean[b] = mu;
                rstd[b] = rs;
            }
        }
    }
}

// ---- backward ---------------------------------------------------------------------------------------
// Both sums of a row and its gradient from one read of H and dX; where the gradients of weight and bias are
// asked for (WG), every thread adds its values' terms over the team's rows in registers, the teams of a
// workgroup are added in LDS, and part[workgroup][0][f] and part[workgroup][1][f] are its sums.
template <typename TH, typename TD, int TEAM, int NC, bool WG>
__global__ __launch_bounds__(1024) void k_ln_bwd(int64_t B, int F, const TH *__restrict__ H, int64_t ldh,
                                                 const float *__restrict__ weight, const float *__restrict__ mean,
                                                 const float *__restrict__ rstd, const TD *dX, int64_t lddx, TH *dH,
                                                 int64_t lddh, float *__restrict__ part) {
    __shared__ float red[2 * 16 * 2];
    extern __shared__ float4 lds[];             // [teams][F] floats, rows of whole float4
    int turn = 0;
    const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM, teams = blockDim.x / TEAM;
    float w[NC][4], aw[NC][4], ab[NC][4];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int f = 4 * (i * TEAM + t);
        unpack4(load4(weight + f, weight ? F - f : 0), w[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (!weight) w[i][j] = 1.0f;
            aw[i][j] = ab[i][j] = 0.0f;
        }
    }
    for (int64_t b0 = (int64_t)blockIdx.x * teams; b0 < B; b0 += (int64_t)gridDim.x * teams) {
        const bool in = b0 + team < B;
        const int64_t b = in ? b0 + team : b0;
        const TH *h = H + b * ldh;
        const TD *d = dX + b * lddx;
        float x[NC][4], g[NC][4];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int f = 4 * (i * TEAM + t);
            unpack4(load4(h + f, F - f), x[i]);
            unpack4(load4(d + f, in ? F - f : 0), g[i]);      // a row that is not there adds zeros
        }
        const float mu = mean[b], rs = rstd[b];
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[i][j] = (x[i][j] - mu) * rs;
                if constexpr (WG) {
                    aw[i][j] = in ? __fmaf_rn(g[i][j], x[i][j], aw[i][j]) : aw[i][j];
                    ab[i][j] += g[i][j];
                }
                g[i][j] *= w[i][j];
                s[0] += g[i][j];
                s[1] = 4 * (i * TEAM + t) + j < F ? __fmaf_rn(g[i][j], x[i][j], s[1]) : s[1];
            }
        if (!dH) continue;
        team_sum<TEAM>(s, red, turn);
        const float m0 = s[0] / (float)F, m1 = s[1] / (float)F;
        if (in) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int f = 4 * (i * TEAM + t);
                float o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = (g[i][j] - m0 - x[i][j] * m1) * rs;
                store4(dH + b * lddh + f, o, F - f);
            }
        }
    }
    if constexpr (WG) {
        const int F4 = (F + 3) / 4;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float *out = part + (2 * (int64_t)blockIdx.x + k) * F;
            if (teams == 1) {
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const int f = 4 * (i * TEAM + t);
                    store4(out + f, k ? ab[i] : aw[i], F - f);
                }
                continue;
            }
            if (k) __syncthreads();
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int q = i * TEAM + t;
                const float *v = k ? ab[i] : aw[i];
                if (q < F4) lds[team * F4 + q] = make_float4(v[0], v[1], v[2], v[3]);
            }
            __syncthreads();
            for (int q = threadIdx.x; q < F4; q += blockDim.x) {
                float4 a = lds[q];
                for (int r = 1; r < teams; ++r) {
                    const float4 v = lds[r * F4 + q];
                    a.x += v.x, a.y += v.y, a.z += v.z, a.w += v.w;
                }
                const float v[4] = {a.x, a.y, a.z, a.w};
                store4(out + 4 * q, v, F - 4 * q);
            }
        }
    }
}

// dweight, dbias (either may be NULL) from the workgroups' sums: 64 columns a workgroup, its sixteen waves a
// sixteenth of the sums each, in ascending order, and the waves' sums in order.
__global__ __launch_bounds__(1024) void k_ln_wsum(const float *__restrict__ part, int64_t parts, int64_t F,
                                                  float *__restrict__ dweight, float *__restrict__ dbias, int beta) {
    __shared__ float red[1024];
    const int64_t i = (int64_t)blockIdx.x * kWave + (threadIdx.x & (kWave - 1));
    const int64_t run = (parts + 15) / 16, p0 = threadIdx.x / kWave * run, p1 = p0 + run < parts ? p0 + run : parts;
    float s = 0.0f;
    if (i < 2 * F) {
        const float *p = part + i;
#pragma unroll 8
        for (int64_t k = p0; k < p1; ++k) s += p[k * 2 * F];
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x >= kWave || i >= 2 * F) return;
    float *out = i < F ? dweight : dbias;
    if (!out) return;
    out += i < F ? i : i - F;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += red[threadIdx.x + w * kWave];
    *out = beta ? *out + s : s;
}

// ---- rows of any width ------------------------------------------------------------------------------
constexpr int kThreads = 256;

// Sum over the workgroup, on every thread.
__device__ __forceinline__ float block_sum(float v, float *red) {
    v = sum64(v);
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// One workgroup per row: mean, then the squares around it, then the row's values; the row is read three
// times, from the caches after the first.
template <typename TH, typename TX>
__global__ __launch_bounds__(kThreads) void k_ln_fwd_wide(int64_t B, int64_t F, const TH *H, int64_t ldh,
                                                          const float *__restrict__ weight,
                                                          const float *__restrict__ bias, float eps, TX *X, int64_t ldx,
                                                          float *__restrict__ mean, float *__restrict__ rstd) {
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
__global__ __launch_bounds__(kThreads) void k_ln_bwd_wide(int64_t B, int64_t F, const TH *__restrict__ H, int64_t ldh,
                                                          const float *__restrict__ weight,
                                                          const float *__restrict__ mean, const float *__restrict__ rstd,
                                                          const TD *dX, int64_t lddx, TH *dH, int64_t lddh) {
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

// part[p][0][f] and part[p][1][f]: the sums of dX xh and of dX over run p of the rows.  A workgroup takes 64
// columns of a run, each of its waves every fourth row.
template <typename TH, typename TD>
__global__ __launch_bounds__(kThreads) void k_ln_wgrad_wide(int64_t B, int64_t F, const TH *__restrict__ H, int64_t ldh,
                                                            const float *__restrict__ mean,
                                                            const float *__restrict__ rstd, const TD *__restrict__ dX,
                                                            int64_t lddx, int64_t per_part, float *__restrict__ part) {
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

// ---- which team takes a row ---------------------------------------------------------------------------
constexpr int64_t kWideF = 8192;       // rows beyond it are not held in registers
constexpr int kMaxRowBlocks = 65536;   // workgroups of the kernels for them; more rows go round

int team_of(int64_t F) { return F <= 256 ? 16 : F <= 1024 ? 64 : F <= 2048 ? 256 : 1024; }

// f(team, runs of four values a thread) for rows of F <= kWideF values
template <typename F>
void with_team(int64_t width, F &&f) {
    auto go = [&](auto team, auto most) {
        const int64_t n = haste::cdiv(width, 4 * team);
        if (n <= 1) f(team, std::integral_constant<int, 1>{});
        else if (n == 2) f(team, std::integral_constant<int, 2>{});
        if constexpr (most > 2) {
            if (n == 3) f(team, std::integral_constant<int, 3>{});
            else if (n == 4) f(team, std::integral_constant<int, 4>{});
        }
    };
    typedef std::integral_constant<int, 2> two;
    typedef std::integral_constant<int, 4> four;
    switch (team_of(width)) {
    case 16: go(std::integral_constant<int, 16>{}, four{}); break;
    case 64: go(std::integral_constant<int, 64>{}, four{}); break;
    case 256: go(std::integral_constant<int, 256>{}, two{}); break;
    default: go(std::integral_constant<int, 1024>{}, two{});
    }
}

// The backward kernel's workgroups.  Each leaves one row of sums, so many rows take 1024 threads a workgroup and
// no more workgroups than CUs; few rows take 256 threads, to spread over the CUs.
struct BwdShape {
    int threads;
    int64_t blocks;
};
BwdShape bwd_shape(int64_t B, int64_t F) {
    const int team = team_of(F);
    const int threads = team > 256 || B * team >= (int64_t)2 * 256 * 1024 ? 1024 : 256;
    const int64_t want = haste::cdiv(B, threads / team), most = 256 * (1024 / threads);
    return {threads, want < most ? want : most};
}

int64_t wide_parts(int64_t B) {
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
    with_type(dtype_h, [&](auto th) {
        with_type(dtype_x, [&](auto tx) {
            typedef decltype(th) TH;
            typedef decltype(tx) TX;
            if (F > kWideF) {
                hipLaunchKernelGGL((k_ln_fwd_wide<TH, TX>), dim3((unsigned)(B < kMaxRowBlocks ? B : kMaxRowBlocks)),
                                   dim3(kThreads), 0, s, B, F, (const TH *)H, ldh, weight, bias, eps, (TX *)X, ldx, mean, rstd);
                return;
            }
            with_team(F, [&](auto team, auto nc) {
                const int threads = team > 256 ? (int)team : 256;
                const int64_t want = cdiv(B, threads / team), most = 256 * (2048 / threads);
                hipLaunchKernelGGL((k_ln_fwd<TH, TX, team, nc>), dim3((unsigned)(want < most ? want : most)), dim3(threads), 0,
                                   s, B, (int)F, (const TH *)H, ldh, weight, bias, eps, (TX *)X, ldx, mean, rstd);
            });
        });
    });
    return hipGetLastError();
}

size_t ln_bwd_ws(int64_t B, int64_t F) {
    return (size_t)((F > kWideF ? wide_parts(B) : bwd_shape(B, F).blocks) * 2 * F * 4);
}

hipError_t ln_bwd(int64_t B, int64_t F, int32_t dtype_h, const void *H, int64_t ldh, const float *weight,
                  const float *mean, const float *rstd, int32_t dtype_dx, const void *dX, int64_t lddx, void *dH,
                  int64_t lddh, float *dweight, float *dbias, int beta, void *ws, hipStream_t s) {
    float *part = (float *)ws;
    const bool wg = dweight || dbias;
    const BwdShape n = bwd_shape(B, F);
    const int64_t parts = F > kWideF ? wide_parts(B) : n.blocks;
    with_type(dtype_h, [&](auto th) {
        with_type(dtype_dx, [&](auto td) {
            typedef decltype(th) TH;
            typedef decltype(td) TD;
            if (F > kWideF) {
                // the sums over rows first: dH may take dX's place
                if (wg)
                    hipLaunchKernelGGL((k_ln_wgrad_wide<TH, TD>), dim3((unsigned)cdiv(F, kWave), (unsigned)parts),
                                       dim3(kThreads), 0, s, B, F, (const TH *)H, ldh, mean, rstd, (const TD *)dX, lddx,
                                       cdiv(B, parts), part);
                if (dH)
                    hipLaunchKernelGGL((k_ln_bwd_wide<TH, TD>), dim3((unsigned)(B < kMaxRowBlocks ? B : kMaxRowBlocks)),
                                       dim3(kThreads), 0, s, B, F, (const TH *)H, ldh, weight, mean, rstd, (const TD *)dX,
                                       lddx, (TH *)dH, lddh);
                return;
            }
            with_team(F, [&](auto team, auto nc) {
                const int teams = n.threads / team;
                const size_t lds = wg && teams > 1 ? (size_t)teams * cdiv(F, 4) * 16 : 0;
                if (wg)
                    hipLaunchKernelGGL((k_ln_bwd<TH, TD, team, nc, true>), dim3((unsigned)n.blocks), dim3(n.threads), lds, s, B,
                                       (int)F, (const TH *)H, ldh, weight, mean, rstd, (const TD *)dX, lddx, (TH *)dH, lddh, part);
                else
                    hipLaunchKernelGGL((k_ln_bwd<TH, TD, team, nc, false>), dim3((unsigned)n.blocks), dim3(n.threads), lds, s, B,
                                       (int)F, (const TH *)H, ldh, weight, mean, rstd, (const TD *)dX, lddx, (TH *)dH, lddh, part);
            });
        });
    });
    if (wg)
        hipLaunchKernelGGL(k_ln_wsum, dim3((unsigned)cdiv(2 * F, kWave)), dim3(1024), 0, s, part, parts, F, dweight, dbias, beta);
    return hipGetLastError();
}

}  // namespace haste
