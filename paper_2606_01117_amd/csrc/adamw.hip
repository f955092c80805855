// The norm of a list of gradients with the factor that clips it, and one step of AdamW over a list of
// tensors, with moments in 32 or in 8 bits.
//
// A list reaches the GPU in the kernel's own arguments, kListMax tensors a launch: no table to copy, and a
// captured graph holds it by value.  A workgroup takes kChunk consecutive values of one tensor; `start` holds
// the number of each tensor's first workgroup.
#include "common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;     // values under one scale of an 8-bit moment

// The tensor that a workgroup belongs to: the last one whose first workgroup is not beyond it.  Every lane
// compares one tensor's, so the search waits for memory once.
__device__ __forceinline__ int tensor_of(const uint32_t *start, int count, uint32_t block) {
    const int lane = threadIdx.x & (kWave - 1);
    const bool before = lane < count && start[lane < count ? lane : 0] <= block;
    return __popcll(__ballot(before)) - 1;
}

// ---- the norm ---------------------------------------------------------------------------------
constexpr int kNormMax = 64;
constexpr int64_t kNormChunk = 8192;

struct NormList {
    const void *grad[kNormMax];
    int64_t n[kNormMax];
    uint32_t start[kNormMax];
    uint64_t bf16;              // bit k: tensor k's gradient is bf16
    int32_t count;
};

// the sum over the workgroup's threads, in thread 0
__device__ __forceinline__ double block_sum(double v, double *red) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    double s = red[0];
    for (int w = 1; w < (int)blockDim.x / kWave; ++w) s += red[w];
    return s;
}

template <typename T>
__device__ __forceinline__ double sum_squares(const T *g, int64_t n) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kThreads) {
        const double x = (double)load_f32(g, i);
        s = __fma_rn(x, x, s);
    }
    return s;
}

// part[workgroup] = the sum of its values' squares, in 64 bits (fp32's range ends at 1.8e19 for a square)
__global__ __launch_bounds__(kThreads) void k_gn_part(NormList l, double *__restrict__ part) {
    __shared__ double red[kThreads / kWave];
    const int k = tensor_of(l.start, l.count, blockIdx.x);
    const int64_t i0 = (int64_t)(blockIdx.x - l.start[k]) * kNormChunk;
    const int64_t n = l.n[k] - i0 < kNormChunk ? l.n[k] - i0 : kNormChunk;
    const double s = block_sum((l.bf16 >> k) & 1 ? sum_squares((const bf16_t *)l.grad[k] + i0, n)
                                                 : sum_squares((const float *)l.grad[k] + i0, n), red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void k_gn_final(const double *__restrict__ part, int64_t parts, float max_norm,
                                                   float *__restrict__ out) {
    __shared__ double red[1024 / kWave];
    double s = 0.0;
    for (int64_t p = threadIdx.x; p < parts; p += 1024) s += part[p];
    s = block_sum(s, red);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        out[0] = (float)norm;
        out[1] = !(norm < (double)INFINITY) ? NAN : norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
    }
}

// ---- the step ---------------------------------------------------------------------------------
constexpr int kListMax = 52;          // the arguments of a kernel have 4096 bytes
constexpr int64_t kChunk = 1024;

struct StepTensor {
    void *W;
    float *W32;
    const void *grad;
    void *m, *v;
    uint8_t *scale;
    int64_t n;
    float lr_scale, weight_decay;
    int32_t kind;                     // kBf16 | kMaster | kGradBf16 | kBits8
};
constexpr int kBf16 = 1, kMaster = 2, kGradBf16 = 4, kBits8 = 8;

struct StepList {
    StepTensor t[kListMax];
    uint32_t start[kListMax];
    int32_t count;
    uint32_t first;                   // number of t[0] in the caller's list (for the draws)
    float b1, c1, b2, c2, eps;        // betas, 1 - betas
    float lr, rbc1, rbc2;             // 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    uint64_t seed;                    // + step, where that is known on the host
    double beta1, beta2;
    const float *lr_dev;
    const int64_t *step_dev;
    const float *grad_scale;
};
static_assert(sizeof(StepList) <= 4096, "kernel arguments");

__device__ __forceinline__ uint64_t splitmix64_at(uint64_t s, uint64_t i) {
    uint64_t z = s + (i + 1) * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// 1 - beta^t by squaring, as the host's pow gives it to 1e-10
__device__ __forceinline__ double bias_correction(double beta, int64_t t) {
    double p = 1.0, b = beta;
    for (; t > 0; t >>= 1) {
        if (t & 1) p *= b;
        if (p < 1e-30) break;
        b *= b;
    }
    return 1.0 - p;
}

// What the kernels take from the options: fixed by the host, or read here where they are on the device.
struct Scalars {
    float lr, rbc1, rbc2, gs;
    uint64_t key;
};

// E4M3 magnitude as it is stored: x is scaled so that E4M3's exponent and mantissa are the upper bits of
// fp32's own (its lowest exponents, and below them its denormals, are E4M3's), so rounding by the draw d is an
// addition to the 20 bits below them.  Infinities and NaN come out as 127, NaN.
__device__ __forceinline__ uint32_t store_e4m3(float x, int shift, uint32_t d) {
    const uint32_t q = (__float_as_uint(ldexpf(x, shift)) + (d << 4)) >> 20;
    return q < 127u ? q : 127u;
}

__device__ __forceinline__ float load_e4m3(uint8_t q, uint8_t scale) {
    return __builtin_amdgcn_cvt_f32_fp8((int)q, 0) * __uint_as_float((uint32_t)scale << 23);
}

// largest finite magnitude of the 32 lanes' values -> their scale
__device__ __forceinline__ uint32_t block_scale(float x) {
    uint32_t e = __float_as_uint(x) & 0x7fffffffu;
    e = e < 0x7f800000u ? e : 0u;
#pragma unroll
    for (int o = kBlock / 2; o > 0; o >>= 1) {
        const uint32_t y = __shfl_xor(e, o);
        e = e > y ? e : y;
    }
    e >>= 23;
    return (e < 23u ? 23u : e) - 7u;
}

template <int KIND>
__device__ __forceinline__ void step_chunk(const StepTensor &t, const StepList &l, const Scalars &c, uint32_t k, int64_t i0) {
    typedef std::conditional_t<(KIND & kBf16) != 0, bf16_t, float> TW;
    typedef std::conditional_t<(KIND & kGradBf16) != 0, bf16_t, float> TG;
    const float lr = c.lr * t.lr_scale;
    for (int64_t j = threadIdx.x; j < kChunk; j += kThreads) {
        const int64_t i = i0 + j;
        const bool in = i < t.n;      // whole blocks of 32 lanes go on together
        const float g = in ? load_f32((const TG *)t.grad, i) * c.gs : 0.0f;
        float m = 0.0f, v = 0.0f;
        if (in) {
            if constexpr (KIND & kBits8) {
                const uint8_t *sc = t.scale + i / kBlock * 2;
                m = load_e4m3(((const uint8_t *)t.m)[i], sc[0]);
                v = load_e4m3(((const uint8_t *)t.v)[i], sc[1]);
                v = __fmul_rn(v, v);
            } else {
                m = ((const float *)t.m)[i];
                v = ((const float *)t.v)[i];
            }
        }
        m = __fmaf_rn(l.b1, m, __fmul_rn(l.c1, g));
        v = __fmaf_rn(l.b2, v, __fmul_rn(__fmul_rn(l.c2, g), g));
        const float r = __fsqrt_rn(v);
        if (in) {
            float w = KIND & kMaster ? t.W32[i] : load_f32((const TW *)t.W, i);
            const float u = m * c.rbc1 / __fmaf_rn(r, c.rbc2, l.eps);
            w = __fmaf_rn(-lr, __fmaf_rn(t.weight_decay, w, u), w);
            if constexpr (KIND & kMaster) t.W32[i] = w;
            store_out((TW *)t.W, i, w);
        }
        if constexpr (KIND & kBits8) {
            const uint32_t sm = block_scale(m), sv = block_scale(r);
            if (in) {
                const uint32_t d = (uint32_t)(splitmix64_at(c.key, ((uint64_t)k << 40) + (uint64_t)(i >> 2)) >>
                                              (16 * (i & 3))) & 0xffffu;
                const uint32_t qm = store_e4m3(fabsf(m), 7 - (int)sm, d);
                uint32_t qv = store_e4m3(r, 7 - (int)sv, 0xffffu - d);
                if (r > 0.0f && qv == 0u) qv = 1u;
                ((uint8_t *)t.m)[i] = (uint8_t)(qm | (__float_as_uint(m) >> 31 << 7));
                ((uint8_t *)t.v)[i] = (uint8_t)qv;
                if (i % kBlock == 0) {
                    t.scale[i / kBlock * 2] = (uint8_t)sm;
                    t.scale[i / kBlock * 2 + 1] = (uint8_t)sv;
                }
            }
        } else if (in) {
            ((float *)t.m)[i] = m;
            ((float *)t.v)[i] = v;
        }
    }
}

__global__ __launch_bounds__(kThreads) void k_adamw(StepList l) {
    Scalars c = {l.lr, l.rbc1, l.rbc2, 1.0f, 0};
    if (l.grad_scale) {
        c.gs = *l.grad_scale;
        if (!(fabsf(c.gs) < INFINITY)) return;     // the whole grid: the gradients overflowed
    }
    if (l.lr_dev) c.lr = *l.lr_dev;
    uint64_t seed = l.seed;
    if (l.step_dev) {
        const int64_t t = *l.step_dev;
        c.rbc1 = (float)(1.0 / bias_correction(l.beta1, t));
        c.rbc2 = (float)(1.0 / sqrt(bias_correction(l.beta2, t)));
        seed += (uint64_t)t;
    }
    c.key = splitmix64_at(seed, 0);
    const int k = tensor_of(l.start, l.count, blockIdx.x);
    const StepTensor &t = l.t[k];
    const int64_t i0 = (int64_t)(blockIdx.x - l.start[k]) * kChunk;
    const uint32_t no = l.first + (uint32_t)k;
    switch (t.kind) {
    case 0: step_chunk<0>(t, l, c, no, i0); break;
    case kBf16: step_chunk<kBf16>(t, l, c, no, i0); break;
    case kBf16 | kMaster: step_chunk<kBf16 | kMaster>(t, l, c, no, i0); break;
    case kGradBf16: step_chunk<kGradBf16>(t, l, c, no, i0); break;
    case kGradBf16 | kBf16: step_chunk<kGradBf16 | kBf16>(t, l, c, no, i0); break;
    case kGradBf16 | kBf16 | kMaster: step_chunk<kGradBf16 | kBf16 | kMaster>(t, l, c, no, i0); break;
    case kBits8: step_chunk<kBits8>(t, l, c, no, i0); break;
    case kBits8 | kBf16: step_chunk<kBits8 | kBf16>(t, l, c, no, i0); break;
    case kBits8 | kBf16 | kMaster: step_chunk<kBits8 | kBf16 | kMaster>(t, l, c, no, i0); break;
    case kBits8 | kGradBf16: step_chunk<kBits8 | kGradBf16>(t, l, c, no, i0); break;
    case kBits8 | kGradBf16 | kBf16: step_chunk<kBits8 | kGradBf16 | kBf16>(t, l, c, no, i0); break;
    case kBits8 | kGradBf16 | kBf16 | kMaster:
        step_chunk<kBits8 | kGradBf16 | kBf16 | kMaster>(t, l, c, no, i0);
        break;
    }
}

// workgroups of a launch (which has fewer than 2^32 threads); the largest tensor fits one
constexpr int64_t kMaxGrid = (int64_t)1 << 23;
static_assert(haste::kParamValuesMax / kChunk <= kMaxGrid && kMaxGrid * kThreads < ((int64_t)1 << 32), "one launch");

}  // namespace

namespace haste {

size_t grad_norm_ws(const haste_param_t *p, int64_t n) {
    int64_t parts = 0;
    for (int64_t k = 0; k < n; ++k) parts += cdiv(p[k].n, kNormChunk);
    return (size_t)(parts > 0 ? parts : 1) * 8;
}

hipError_t grad_norm(const haste_param_t *p, int64_t n, float max_norm, float *out, void *ws, hipStream_t s) {
    double *part = (double *)ws;
    int64_t parts = 0;
    NormList l;
    l.count = 0;
    l.bf16 = 0;
    int64_t grid = 0;
    for (int64_t k = 0; k <= n; ++k) {
        if (k < n && p[k].n == 0) continue;
        const int64_t c = k < n ? cdiv(p[k].n, kNormChunk) : 0;
        if (l.count > 0 && (k == n || l.count == kNormMax || grid + c > kMaxGrid)) {
            hipLaunchKernelGGL(k_gn_part, dim3((unsigned)grid), dim3(kThreads), 0, s, l, part + parts);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            parts += grid;
            grid = 0;
            l.count = 0;
            l.bf16 = 0;
        }
        if (k == n) break;
        l.grad[l.count] = p[k].grad;
        l.n[l.count] = p[k].n;
        l.start[l.count] = (uint32_t)grid;
        if (p[k].grad_dtype == HASTE_DTYPE_BF16) l.bf16 |= 1ull << l.count;
        ++l.count;
        grid += c;
    }
    hipLaunchKernelGGL(k_gn_final, dim3(1), dim3(1024), 0, s, part, parts, max_norm, out);
    return hipGetLastError();
}

// The updated arrays' addresses in an open hash table on the stack: 512 tensors go in, the ones behind them are
// only looked up, then the next 512 go in.
int64_t adamw_repeated(const haste_param_t *p, int64_t n) {
    constexpr int kWindow = 512, kSlots = 4096;      // 5 addresses a tensor
    const void *slot[kSlots];
    for (int64_t w = 0; w < n; w += kWindow) {
        const int64_t w1 = w + kWindow < n ? w + kWindow : n;
        for (int i = 0; i < kSlots; ++i) slot[i] = nullptr;
        for (int64_t k = w; k < n; ++k) {
            if (p[k].n == 0) continue;
            const void *a[5] = {p[k].W, p[k].W32, p[k].m, p[k].v, p[k].state_bits == 8 ? p[k].scale : nullptr};
            for (const void *x : a) {
                if (!x) continue;
                uint32_t h = (uint32_t)(((uint64_t)(uintptr_t)x * 0x9E3779B97F4A7C15ull) >> 52);
                while (slot[h] && slot[h] != x) h = (h + 1) & (kSlots - 1);
                if (slot[h]) return k;
                if (k < w1) slot[h] = x;
            }
        }
    }
    return -1;
}

hipError_t adamw(const haste_param_t *p, int64_t n, const haste_adamw_opts_t &o, hipStream_t s) {
    StepList l;
    l.b1 = (float)o.beta1;
    l.c1 = (float)(1.0 - o.beta1);
    l.b2 = (float)o.beta2;
    l.c2 = (float)(1.0 - o.beta2);
    l.eps = (float)o.eps;
    l.lr = (float)o.lr;
    l.rbc1 = l.rbc2 = 1.0f;
    l.seed = o.seed;
    if (!o.step_dev) {
        l.rbc1 = (float)(1.0 / (1.0 - pow(o.beta1, (double)o.step)));
        l.rbc2 = (float)(1.0 / sqrt(1.0 - pow(o.beta2, (double)o.step)));
        l.seed += (uint64_t)o.step;
    }
    l.beta1 = o.beta1;
    l.beta2 = o.beta2;
    l.lr_dev = o.lr_dev;
    l.step_dev = o.step_dev;
    l.grad_scale = o.grad_scale;
    l.count = 0;
    int64_t grid = 0;
    for (int64_t k = 0; k <= n; ++k) {
        // a run's tensors have consecutive numbers, so one of no values keeps its slot in it
        const int64_t c = k < n ? cdiv(p[k].n, kChunk) : 0;
        if (l.count > 0 && (k == n || l.count == kListMax || grid + c > kMaxGrid)) {
            if (grid > 0) hipLaunchKernelGGL(k_adamw, dim3((unsigned)grid), dim3(kThreads), 0, s, l);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            grid = 0;
            l.count = 0;
        }
        if (k == n) break;
        if (l.count == 0) l.first = (uint32_t)k;
        StepTensor &t = l.t[l.count];
        t.W = p[k].W;
        t.W32 = p[k].W32;
        t.grad = p[k].grad;
        t.m = p[k].m;
        t.v = p[k].v;
        t.scale = p[k].scale;
        t.n = p[k].n;
        t.lr_scale = p[k].lr_scale;
        t.weight_decay = p[k].weight_decay;
        t.kind = (p[k].dtype == HASTE_DTYPE_BF16 ? kBf16 : 0) | (p[k].W32 ? kMaster : 0) |
                 (p[k].grad_dtype == HASTE_DTYPE_BF16 ? kGradBf16 : 0) | (p[k].state_bits == 8 ? kBits8 : 0);
        l.start[l.count] = (uint32_t)grid;
        ++l.count;
        grid += c;
    }
    return hipSuccess;
}

}  // namespace haste
