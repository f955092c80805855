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
// compares MAX / 64 tensors', so the search waits for memory once.
template <int MAX>
__device__ __forceinline__ int tensor_of(const uint32_t (&start)[MAX], int count, uint32_t block) {
    const int lane = threadIdx.x & (kWave - 1);
    int k = -1;
#pragma unroll
    for (int j = 0; j < (MAX + kWave - 1) / kWave; ++j) {
        const int i = j * kWave + lane;
        k += __popcll(__ballot(i < count && start[i < count ? i : 0] <= block));
    }
    return k;
}

// ---- the norm ---------------------------------------------------------------------------------
constexpr int kNormMax = 192;
constexpr int64_t kNormChunk = 16384;

struct NormList {
    const void *grad[kNormMax];
    int64_t n[kNormMax];
    uint32_t start[kNormMax];
    uint64_t bf16[kNormMax / 64];   // bit k: tensor k's gradient is bf16
    int32_t count;
};
static_assert(sizeof(NormList) <= 4096 - 16, "kernel arguments");

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

__device__ __forceinline__ double square(float x, double s) { return __fma_rn((double)x, (double)x, s); }

// Four sums a thread, each of a 16-byte load in a round of four; the loads of a round go out together.
template <typename T>
__device__ __forceinline__ double sum_squares(const T *g, int n) {
    constexpr int V = 16 / sizeof(T), R = 4;
    double s[R] = {};
    const int whole = n / (V * kThreads * R) * (V * kThreads * R);
    for (int i = V * (int)threadIdx.x; i < whole; i += V * kThreads * R) {
        uint4 v[R];
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = *reinterpret_cast<const uint4 *>(g + i + r * V * kThreads);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t w[4] = {v[r].x, v[r].y, v[r].z, v[r].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (sizeof(T) == 2) {
                    s[r] = square(__uint_as_float(w[j] << 16), s[r]);
                    s[r] = square(__uint_as_float(w[j] & 0xffff0000u), s[r]);
                } else {
                    s[r] = square(__uint_as_float(w[j]), s[r]);
                }
            }
        }
    }
#pragma unroll 4
    for (int i = whole + (int)threadIdx.x; i < n; i += kThreads) s[0] = square(load_f32(g, i), s[0]);
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// part[workgroup] = the sum of its values' squares, in 64 bits (fp32's range ends at 1.8e19 for a square)
__global__ __launch_bounds__(kThreads) void k_gn_part(NormList l, double *__restrict__ part) {
    __shared__ double red[kThreads / kWave];
    const int k = tensor_of(l.start, l.count, blockIdx.x);
    const int64_t i0 = (int64_t)(blockIdx.x - l.start[k]) * kNormChunk;
    const int n = (int)(l.n[k] - i0 < kNormChunk ? l.n[k] - i0 : kNormChunk);
    const double s = block_sum((l.bf16[k / 64] >> (k % 64)) & 1 ? sum_squares((const bf16_t *)l.grad[k] + i0, n)
                                                                : sum_squares((const float *)l.grad[k] + i0, n), red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void k_gn_final(const double *__restrict__ part, int64_t parts, float max_norm,
                                                   float *__restrict__ out) {
    __shared__ double red[1024 / kWave];
    double s = 0.0;
#pragma unroll 4
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
constexpr int64_t kChunk = 4096;

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

// What a step takes from the options: fixed by the host, or read here where they are on the device.
struct Scalars {
    float lr, rbc1, rbc2, gs;
    uint64_t key;
};

// ---- eight consecutive values ---------------------------------------------------------------------
// n of them are there (16-byte accesses where all are), the others read as zero
__device__ __forceinline__ void load8(const float *p, int n, float (&v)[8]) {
    if (n == 8) {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const bf16_t *p, int n, float (&v)[8]) {
    if (n == 8) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) v[2 * j] = __uint_as_float(w[j] << 16), v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? bf16_to_f32(p[j]) : 0.0f;
    }
}
__device__ __forceinline__ uint2 load8(const uint8_t *p, int n) {
    if (n == 8) return *reinterpret_cast<const uint2 *>(p);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < n) w[j / 4] |= (uint32_t)p[j] << (8 * (j % 4));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store8(float *p, int n, const float (&v)[8]) {
    if (n == 8) {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = v[j];
    }
}
__device__ __forceinline__ void store8(bf16_t *p, int n, const float (&v)[8]) {
    if (n == 8) {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                                                   pack_bf16(v[6], v[7]));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = f32_to_bf16(v[j]);
    }
}
__device__ __forceinline__ void store8(uint8_t *p, int n, uint2 q) {
    if (n == 8) {
        *reinterpret_cast<uint2 *>(p) = q;
    } else {
        const uint32_t w[2] = {q.x, q.y};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
    }
}

// ---- moments in 8 bits ------------------------------------------------------------------------------
// E4M3 bytes times their block's scale
__device__ __forceinline__ void load_e4m3(uint2 q, uint32_t scale, float (&v)[8]) {
    const float s = __uint_as_float(scale << 23);
    const uint32_t w[2] = {q.x, q.y};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
        v[4 * j] = a.x * s, v[4 * j + 1] = a.y * s, v[4 * j + 2] = b.x * s, v[4 * j + 3] = b.y * s;
    }
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return o > v ? o : v;
}

// The scale of a block from the magnitudes of its 32 values, eight on each of four neighbouring lanes.
__device__ __forceinline__ uint32_t block_scale(const float (&x)[8]) {
    uint32_t e = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(x[j]) & 0x7fffffffu;
        e = b > e ? b : e;
    }
    if (__ballot(e >= 0x7f800000u)) {       // an infinity or a NaN among the wave's values: they do not count
        e = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = __float_as_uint(x[j]) & 0x7fffffffu;
            e = b < 0x7f800000u && b > e ? b : e;
        }
    }
    e = dpp_max<0x4E>(dpp_max<0xB1>(e)) >> 23;
    return (e < 23u ? 23u : e) - 7u;
}

// E4M3 magnitude as it is stored: x is scaled so that E4M3's exponent and mantissa are the upper bits of
// fp32's own (its lowest exponents, and below them its denormals, are E4M3's), so rounding by the draw d is an
// addition to the 20 bits below them.  Infinities and NaN come out as 127, NaN.
__device__ __forceinline__ uint32_t store_e4m3(float x, int shift, uint32_t d) {
    const uint32_t q = (__float_as_uint(ldexpf(x, shift)) + (d << 4)) >> 20;
    return q < 127u ? q : 127u;
}

// draws z[0] for the first four values, z[1] for the others, 16 bits each; ROOT: not negative, at least 1 above zero
template <bool ROOT>
__device__ __forceinline__ uint2 store_block(const float (&x)[8], uint32_t scale, const uint64_t (&z)[2]) {
    const int shift = 7 - (int)scale;
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t d = (uint32_t)(z[j / 4] >> (16 * (j % 4))) & 0xffffu;
        uint32_t q = store_e4m3(fabsf(x[j]), shift, d);
        if constexpr (ROOT) q = x[j] > 0.0f && q == 0u ? 1u : q;
        else q |= __float_as_uint(x[j]) >> 31 << 7;
        w[j / 4] |= q << (8 * (j % 4));
    }
    return make_uint2(w[0], w[1]);
}

// Values i0 .. i0 + kChunk of tensor t (number k of the list), eight a thread at a time.
template <int KIND>
__device__ __forceinline__ void step_chunk(const StepTensor &t, const StepList &l, const Scalars &c, uint32_t k, int64_t i0) {
    typedef std::conditional_t<(KIND & kBf16) != 0, bf16_t, float> TW;
    typedef std::conditional_t<(KIND & kGradBf16) != 0, bf16_t, float> TG;
    const float lr = c.lr * t.lr_scale, wd = t.weight_decay;
    for (int64_t b = i0; b < i0 + kChunk && b < t.n; b += 8 * kThreads) {
        const int64_t i = b + 8 * threadIdx.x;
        const int n = t.n - i >= 8 ? 8 : t.n - i > 0 ? (int)(t.n - i) : 0;
        float w[8], g[8], m[8], v[8], r[8];
        uint2 qm, qv;
        uint32_t sc = 0;
        load8((const TG *)t.grad + i, n, g);
        if constexpr (KIND & kBits8) {
            qm = load8((const uint8_t *)t.m + i, n);
            qv = load8((const uint8_t *)t.v + i, n);
            if (n > 0) sc = ((const uint16_t *)t.scale)[i / kBlock];
        } else {
            load8((const float *)t.m + i, n, m);
            load8((const float *)t.v + i, n, v);
        }
        if constexpr (KIND & kMaster) load8(t.W32 + i, n, w);
        else load8((const TW *)t.W + i, n, w);
        if constexpr (KIND & kBits8) {
            load_e4m3(qm, sc & 0xffu, m);
            load_e4m3(qv, sc >> 8, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (KIND & kBits8) v[j] = __fmul_rn(v[j], v[j]);
            const float x = __fmul_rn(g[j], c.gs);
            m[j] = __fmaf_rn(l.b1, m[j], __fmul_rn(l.c1, x));
            v[j] = __fmaf_rn(l.b2, v[j], __fmul_rn(__fmul_rn(l.c2, x), x));
            r[j] = __fsqrt_rn(v[j]);
            const float u = m[j] * c.rbc1 * __builtin_amdgcn_rcpf(__fmaf_rn(r[j], c.rbc2, l.eps));
            w[j] = __fmaf_rn(-lr, __fmaf_rn(wd, w[j], u), w[j]);
        }
        if constexpr (KIND & kMaster) store8(t.W32 + i, n, w);
        store8((TW *)t.W + i, n, w);
        if constexpr (KIND & kBits8) {
            const uint32_t sm = block_scale(m), sv = block_scale(r);
            const uint64_t first = ((uint64_t)k << 40) + (uint64_t)(i >> 2);
            uint64_t z[2] = {splitmix64_at(c.key, first), splitmix64_at(c.key, first + 1)};
            store8((uint8_t *)t.m + i, n, store_block<false>(m, sm, z));
            z[0] = ~z[0], z[1] = ~z[1];
            store8((uint8_t *)t.v + i, n, store_block<true>(r, sv, z));
            if (n > 0 && (threadIdx.x & 3) == 0) ((uint16_t *)t.scale)[i / kBlock] = (uint16_t)(sm | sv << 8);
        } else {
            store8((float *)t.m + i, n, m);
            store8((float *)t.v + i, n, v);
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
    l.bf16[0] = l.bf16[1] = l.bf16[2] = 0;
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
            l.bf16[0] = l.bf16[1] = l.bf16[2] = 0;
        }
        if (k == n) break;
        l.grad[l.count] = p[k].grad;
        l.n[l.count] = p[k].n;
        l.start[l.count] = (uint32_t)grid;
        if (p[k].grad_dtype == HASTE_DTYPE_BF16) l.bf16[l.count / 64] |= 1ull << (l.count % 64);
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
