// The norm of a list of gradients with the factor that clips it, and one step of AdamW over a list of
// tensors, with moments in 32 or in 8 bits.
//
// A list reaches the GPU in the kernel's own arguments, kListMax tensors a launch: no table to copy, and a
// captured graph holds it by value.  A workgroup takes a chunk of consecutive values of one tensor; `start`
// holds the number of each tensor's first workgroup.
#include "common.hpp"

#include <cstdlib>

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 32;     // values under one scale of an 8-bit moment

// The tensor that a workgroup belongs to: the last one whose first workgroup is not beyond it.  Every lane
// compares MAX / 64 tensors', so the search waits for memory once.
template <int MAX, int N>
__device__ __forceinline__ int tensor_of(const uint32_t (&start)[N], int count, uint32_t block) {
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

// Values of a workgroup: enough to read ahead; of short lists one round of loads a thread at most, or they would run on few
// CUs (135K values: 4.4 us with 16384 a workgroup, 3.9 with 4096; 58M take 42 with 16384, 5.5 TB/s).
int64_t norm_chunk(const haste_param_t *p, int64_t n) {
    int64_t total = 0;
    for (int64_t k = 0; k < n; ++k) total += p[k].n;
    return total <= ((int64_t)1 << 22) ? 4096 : 16384;
}

struct NormList {
    const void *grad[kNormMax];
    int64_t n[kNormMax];
    uint32_t start[kNormMax];
    uint64_t bf16[kNormMax / 64];   // bit k: tensor k's gradient is bf16
    int32_t count, chunk;
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

// the squares of a 16-byte load's values, added to s
template <typename T>
__device__ __forceinline__ double squares(const uint4 &v, double s) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) {
            s = square(__uint_as_float(w[j] << 16), s);
            s = square(__uint_as_float(w[j] & 0xffff0000u), s);
        } else {
            s = square(__uint_as_float(w[j]), s);
        }
    }
    return s;
}

// Four sums a thread, each of a 16-byte load in a round of four; the loads of a round go out together.  The last,
// partial round's loads do so too: one past the whole vectors reads the round's first and does not count.  (Both launches
// of a norm, one value a load there and so: 190 tensors of 40768 bf16 values 10.4 and 8.9 us; 211 odd tensors of 3M
// values 10.7 and 9.6, in fp32 13.5 and 11.5.)
template <typename T>
__device__ __forceinline__ double sum_squares(const T *g, int n) {
    constexpr int V = 16 / sizeof(T), R = 4;
    double s[R] = {};
    const int whole = n / (V * kThreads * R) * (V * kThreads * R), vectors = n / V * V;
    for (int i = V * (int)threadIdx.x; i < whole; i += V * kThreads * R) {
        uint4 v[R];
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = *reinterpret_cast<const uint4 *>(g + i + r * V * kThreads);
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = squares<T>(v[r], s[r]);
    }
    if (whole < vectors) {
        const int i = whole + V * (int)threadIdx.x;
        uint4 v[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int at = i + r * V * kThreads;
            v[r] = *reinterpret_cast<const uint4 *>(g + (at < vectors ? at : whole));
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (i + r * V * kThreads < vectors) s[r] = squares<T>(v[r], s[r]);
    }
    const int i = vectors + (int)threadIdx.x;
    if (i < n) s[0] = square(load_f32(g, i), s[0]);
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// part[workgroup] = the sum of its values' squares, in 64 bits (fp32's range ends at 1.8e19 for a square)
__global__ __launch_bounds__(kThreads) void k_gn_part(NormList l, double *__restrict__ part) {
    __shared__ double red[kThreads / kWave];
    const int k = tensor_of<kNormMax>(l.start, l.count, blockIdx.x);
    const int64_t i0 = (int64_t)(blockIdx.x - l.start[k]) * l.chunk;
    const int n = (int)(l.n[k] - i0 < l.chunk ? l.n[k] - i0 : l.chunk);
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
constexpr int kListMax = 76;          // the arguments of a kernel have 4096 bytes
constexpr int kStepThreads = 128;
constexpr int64_t kChunk = 1024;
constexpr int kBf16 = 1, kMaster = 2, kGradBf16 = 4, kBits8 = 8;

// A tensor in 48 bytes, its addresses in 48 bits each, its size by its number of chunks and the values in the last.
struct StepTensor {
    uint32_t lo[6], hi[3];            // of W, W32, grad, m, v, scale
    uint32_t last;                    // values of the last chunk, and 65536 times the kind (kBf16 | ...)
    float lr_scale, weight_decay;
    template <typename T>
    __device__ __forceinline__ T *at(int k) const {
        return reinterpret_cast<T *>((uint64_t)lo[k] | (uint64_t)((hi[k / 2] >> (16 * (k & 1))) & 0xffffu) << 32);
    }
    void put(int k, const void *p) {
        const uint64_t a = (uint64_t)reinterpret_cast<uintptr_t>(p);
        lo[k] = (uint32_t)a;
        hi[k / 2] = k & 1 ? hi[k / 2] | (uint32_t)(a >> 32) << 16 : (uint32_t)(a >> 32);
    }
};

struct StepList {
    StepTensor t[kListMax];
    uint32_t start[kListMax + 1];
    int32_t count, chunk;
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

// ---- kRun consecutive values: 16 bytes of fp32, 8 of bf16, 4 of E4M3 ---------------------------------
constexpr int kRun = 4;

typedef float vec4f_t __attribute__((ext_vector_type(4)));
typedef uint32_t vec2u_t __attribute__((ext_vector_type(2)));

// STREAM: past the caches, for what is not used again before the next step
template <bool STREAM, typename V>
__device__ __forceinline__ V load_vec(const V *p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool STREAM, typename V>
__device__ __forceinline__ void store_vec(V *p, V v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool STREAM = true>
__device__ __forceinline__ void load_run(const float *p, float (&v)[kRun]) {
    const vec4f_t a = load_vec<STREAM>(reinterpret_cast<const vec4f_t *>(p));
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
}
template <bool STREAM = true>
__device__ __forceinline__ void load_run(const bf16_t *p, float (&v)[kRun]) {
    const vec2u_t a = load_vec<STREAM>(reinterpret_cast<const vec2u_t *>(p));
    v[0] = __uint_as_float(a.x << 16), v[1] = __uint_as_float(a.x & 0xffff0000u);
    v[2] = __uint_as_float(a.y << 16), v[3] = __uint_as_float(a.y & 0xffff0000u);
}
template <bool STREAM = true>
__device__ __forceinline__ void store_run(float *p, const float (&v)[kRun]) {
    store_vec<STREAM>(reinterpret_cast<vec4f_t *>(p), vec4f_t{v[0], v[1], v[2], v[3]});
}
template <bool STREAM = true>
__device__ __forceinline__ void store_run(bf16_t *p, const float (&v)[kRun]) {
    store_vec<STREAM>(reinterpret_cast<vec2u_t *>(p), vec2u_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])});
}

// ---- moments in 8 bits ------------------------------------------------------------------------------
__device__ __forceinline__ float scale_value(uint32_t scale) { return __uint_as_float(scale << 23); }

// four E4M3 bytes times their block's scale
__device__ __forceinline__ void load_e4m3(uint32_t q, uint32_t scale, float (&v)[kRun]) {
    const float s = scale_value(scale);
    const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
    v[0] = a.x * s, v[1] = a.y * s, v[2] = b.x * s, v[3] = b.y * s;
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
    return o > v ? o : v;
}

// The largest finite magnitude of a lane's N values, as its bits (the maximum passes NaN over).
template <int N>
__device__ __forceinline__ uint32_t largest(const float (&x)[N]) {
    float a = fabsf(x[0]);
#pragma unroll
    for (int j = 1; j < N; ++j) a = fmaxf(a, fabsf(x[j]));
    uint32_t e = __float_as_uint(a);
    if (__ballot(e >= 0x7f800000u)) {       // an infinity among the wave's values, or a lane of NaN: they do not count
        e = 0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const uint32_t b = __float_as_uint(x[j]) & 0x7fffffffu;
            e = b < 0x7f800000u && b > e ? b : e;
        }
    }
    return e;
}
// The scale of a block from the bits of its largest value.
__device__ __forceinline__ uint32_t scale_of(uint32_t e) {
    e >>= 23;
    return (e < 23u ? 23u : e) - 7u;
}
// The same over the eight neighbouring lanes that hold a block in runs of four: pairs, quads, the two quads.
__device__ __forceinline__ uint32_t block_scale(const float (&x)[kRun]) {
    return scale_of(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(largest(x)))));
}

// What is stored of x: the value over its scale, as the hardware's conversion with random bits takes it: it adds the
// upper 20 of them below E4M3's mantissa and cuts off, which with a 16-bit draw on top is floor(magnitude / spacing
// + d / 65536), also below E4M3's normal range; infinities and NaN become NaN.  (Three instructions a value where
// shifts and masks of fp32's bits take eight: 58M bf16 weights and gradients 119 us with those, 113 so.)
// ROOT: not negative, and 2^-9 of the scale at least where x is above zero.
template <bool ROOT>
__device__ __forceinline__ float scaled(float x, uint32_t scale) {
    const float y = x * __uint_as_float((254u - scale) << 23);
    if constexpr (ROOT) return x > 0.0f ? fmaxf(y, 0x1p-9f) : y;
    return y;
}
// four values under the draws z, 16 bits each
template <bool ROOT>
__device__ __forceinline__ uint32_t store_e4m3(const float (&x)[kRun], uint32_t scale, uint64_t z) {
    const uint32_t lo = (uint32_t)z, hi = (uint32_t)(z >> 32);
    int q = 0;
    q = __builtin_amdgcn_cvt_sr_fp8_f32(scaled<ROOT>(x[0], scale), (int)(lo << 16), q, 0);
    q = __builtin_amdgcn_cvt_sr_fp8_f32(scaled<ROOT>(x[1], scale), (int)(lo & 0xffff0000u), q, 1);
    q = __builtin_amdgcn_cvt_sr_fp8_f32(scaled<ROOT>(x[2], scale), (int)(hi << 16), q, 2);
    q = __builtin_amdgcn_cvt_sr_fp8_f32(scaled<ROOT>(x[3], scale), (int)(hi & 0xffff0000u), q, 3);
    return (uint32_t)q;
}
// one value under the draw in the upper half of d
template <bool ROOT>
__device__ __forceinline__ uint8_t store_e4m3(float x, uint32_t scale, uint32_t d) {
    return (uint8_t)__builtin_amdgcn_cvt_sr_fp8_f32(scaled<ROOT>(x, scale), (int)(d & 0xffff0000u), 0, 0);
}

// ---- the step of N values a lane --------------------------------------------------------------------
// r = sqrt(v), correctly rounded (the 8-bit moments are rounded from it, and two implementations have to meet
// the same value).  s = v y with y = 1 / sqrt(v) to one unit is off by a few units; one step of Newton's method with
// the residual of a fused multiply-add, s + (v - s^2) y / 2, rounds to the right one.  Powers of four scale every step
// exactly within the range below, so two binades stand for all: equal to sqrtf for every value of them (and of four
// more).  Half of the instructions that sqrtf takes (58M bf16 weights and gradients with 8-bit moments, where the
// vector ALUs are the bound: 132 us with it, 115 so).
template <int N>
__device__ __forceinline__ void roots(const float (&v)[N], float (&r)[N]) {
    uint32_t lo = __float_as_uint(v[0]), hi = lo;
#pragma unroll
    for (int j = 1; j < N; ++j) {
        const uint32_t b = __float_as_uint(v[j]);
        lo = b < lo ? b : lo;
        hi = b > hi ? b : hi;
    }
    if (__ballot(lo < 0x12800000u || hi >= 0x7f800000u)) {    // below 2^-90, zeros among them, or not finite
#pragma unroll
        for (int j = 0; j < N; ++j) r[j] = sqrtf(v[j]);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float y = __builtin_amdgcn_rsqf(v[j]), s = v[j] * y;
        r[j] = __fmaf_rn(__fmaf_rn(-s, s, v[j]), 0.5f * y, s);
    }
}

// w, m, v: weights and moments, updated; r: the root of v.
template <int N>
__device__ __forceinline__ void step_values(float (&w)[N], const float (&g)[N], float (&m)[N], float (&v)[N], float (&r)[N],
                                            const StepList &l, const Scalars &c, float lr, float wd) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float x = __fmul_rn(g[j], c.gs);
        m[j] = __fmaf_rn(l.b1, m[j], __fmul_rn(l.c1, x));
        v[j] = __fmaf_rn(l.b2, v[j], __fmul_rn(__fmul_rn(l.c2, x), x));
    }
    roots(v, r);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float u = m[j] * c.rbc1 * __builtin_amdgcn_rcpf(__fmaf_rn(r[j], c.rbc2, l.eps));
        w[j] = __fmaf_rn(-lr, __fmaf_rn(wd, w[j], u), w[j]);
    }
}

// Values i0 .. i0 + n of tensor t (number k of the list), a chunk.  The tensor's whole blocks of 32 go in runs of four
// a lane; its last, partial block one value a lane, on the workgroup's last wave.
template <int KIND, bool KEEP>
__device__ __forceinline__ void step_chunk(const StepTensor &t, const StepList &l, const Scalars &c, uint32_t k, int64_t i0,
                                           uint32_t n) {
    typedef std::conditional_t<(KIND & kBf16) != 0, bf16_t, float> TW;
    typedef std::conditional_t<(KIND & kGradBf16) != 0, bf16_t, float> TG;
    constexpr bool B8 = (KIND & kBits8) != 0, MASTER = (KIND & kMaster) != 0;
    const float lr = c.lr * t.lr_scale, wd = t.weight_decay;
    TW *W = t.at<TW>(0) + i0;
    float *W32 = t.at<float>(1) + i0;
    const TG *G = t.at<TG>(2) + i0;
    float *M = t.at<float>(3) + i0, *V = t.at<float>(4) + i0;
    uint32_t *QM = t.at<uint32_t>(3) + i0 / 4, *QV = t.at<uint32_t>(4) + i0 / 4;
    uint16_t *S = t.at<uint16_t>(5) + i0 / kBlock;
    const uint32_t whole = n / kBlock * kBlock;
    // eight neighbouring lanes, a whole block, go through together
    for (uint32_t i = kRun * threadIdx.x; i < whole; i += kRun * kStepThreads) {
        float w[kRun], g[kRun], m[kRun], v[kRun], r[kRun];
        load_run(G + i, g);
        if constexpr (MASTER) load_run(W32 + i, w);
        else load_run<!KEEP>(W + i, w);
        if constexpr (B8) {
            const uint32_t sc = S[i / kBlock], qm = __builtin_nontemporal_load(QM + i / 4),
                           qv = __builtin_nontemporal_load(QV + i / 4);
            load_e4m3(qm, sc & 0xffu, m);
            load_e4m3(qv, sc >> 8, v);
        } else {
            load_run(M + i, m);
            load_run(V + i, v);
        }
        if constexpr (B8) {
#pragma unroll
            for (int j = 0; j < kRun; ++j) v[j] = __fmul_rn(v[j], v[j]);
        }
        step_values(w, g, m, v, r, l, c, lr, wd);
        if constexpr (MASTER) store_run(W32 + i, w);
        store_run<!KEEP>(W + i, w);
        if constexpr (B8) {
            const uint32_t sm = block_scale(m), sv = block_scale(r);
            const uint64_t z = splitmix64_at(c.key, ((uint64_t)k << 40) + ((uint64_t)i0 + i) / 4);
            __builtin_nontemporal_store(store_e4m3<false>(m, sm, z), QM + i / 4);
            __builtin_nontemporal_store(store_e4m3<true>(r, sv, ~z), QV + i / 4);
            if ((threadIdx.x & 7) == 0) S[i / kBlock] = (uint16_t)(sm | sv << 8);
        } else {
            store_run(M + i, m);
            store_run(V + i, v);
        }
    }
    const int lane = (int)threadIdx.x - (kStepThreads - kWave);
    const uint32_t i = whole + (uint32_t)lane;
    if (n == whole || lane < 0) return;         // wave-uniform
    const bool in = i < n;                      // lanes 0 .. 30 at most
    float w[1] = {0.0f}, g[1] = {0.0f}, m[1] = {0.0f}, v[1] = {0.0f}, r[1];
    if (in) {
        g[0] = load_f32(G, i);
        if constexpr (B8) {
            const uint32_t sc = S[i / kBlock];
            m[0] = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)QM)[i], 0) * scale_value(sc & 0xffu);
            v[0] = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)QV)[i], 0) * scale_value(sc >> 8);
            v[0] = __fmul_rn(v[0], v[0]);
        } else {
            m[0] = M[i];
            v[0] = V[i];
        }
        if constexpr (MASTER) w[0] = W32[i];
        else w[0] = load_f32(W, i);
    }
    step_values(w, g, m, v, r, l, c, lr, wd);
    uint32_t sm = 0, sv = 0;
    if constexpr (B8) {
        sm = largest(m), sv = largest(r);
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) {
            const uint32_t x = (uint32_t)__shfl_xor((int)sm, o), y = (uint32_t)__shfl_xor((int)sv, o);
            sm = x > sm ? x : sm;
            sv = y > sv ? y : sv;
        }
        sm = scale_of(sm), sv = scale_of(sv);
    }
    if (!in) return;
    if constexpr (MASTER) W32[i] = w[0];
    store_out(W, i, w[0]);
    if constexpr (B8) {
        const uint32_t d = (uint32_t)(splitmix64_at(c.key, ((uint64_t)k << 40) + ((uint64_t)i0 + i) / 4) >> (16 * (i & 3))) << 16;
        ((uint8_t *)QM)[i] = store_e4m3<false>(m[0], sm, d);
        ((uint8_t *)QV)[i] = store_e4m3<true>(r[0], sv, ~d);
        if (lane == 0) S[i / kBlock] = (uint16_t)(sm | sv << 8);
    } else {
        M[i] = m[0];
        V[i] = v[0];
    }
}

// KEEP: the weights go through the caches.
template <bool KEEP>
__global__ __launch_bounds__(kStepThreads) void k_adamw(StepList l) {
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
    const int k = tensor_of<kListMax>(l.start, l.count, blockIdx.x);
    const StepTensor &t = l.t[k];
    const int64_t i0 = (int64_t)(blockIdx.x - l.start[k]) * l.chunk;
    const uint32_t no = l.first + (uint32_t)k, n = blockIdx.x + 1 < l.start[k + 1] ? (uint32_t)l.chunk : t.last & 0xffffu;
    switch (t.last >> 16) {
    case 0: step_chunk<0, KEEP>(t, l, c, no, i0, n); break;
    case kBf16: step_chunk<kBf16, KEEP>(t, l, c, no, i0, n); break;
    case kBf16 | kMaster: step_chunk<kBf16 | kMaster, KEEP>(t, l, c, no, i0, n); break;
    case kGradBf16: step_chunk<kGradBf16, KEEP>(t, l, c, no, i0, n); break;
    case kGradBf16 | kBf16: step_chunk<kGradBf16 | kBf16, KEEP>(t, l, c, no, i0, n); break;
    case kGradBf16 | kBf16 | kMaster: step_chunk<kGradBf16 | kBf16 | kMaster, KEEP>(t, l, c, no, i0, n); break;
    case kBits8: step_chunk<kBits8, KEEP>(t, l, c, no, i0, n); break;
    case kBits8 | kBf16: step_chunk<kBits8 | kBf16, KEEP>(t, l, c, no, i0, n); break;
    case kBits8 | kBf16 | kMaster: step_chunk<kBits8 | kBf16 | kMaster, KEEP>(t, l, c, no, i0, n); break;
    case kBits8 | kGradBf16: step_chunk<kBits8 | kGradBf16, KEEP>(t, l, c, no, i0, n); break;
    case kBits8 | kGradBf16 | kBf16: step_chunk<kBits8 | kGradBf16 | kBf16, KEEP>(t, l, c, no, i0, n); break;
    case kBits8 | kGradBf16 | kBf16 | kMaster:
        step_chunk<kBits8 | kGradBf16 | kBf16 | kMaster, KEEP>(t, l, c, no, i0, n);
        break;
    }
}

// workgroups of a launch (which has fewer than 2^32 threads); the largest tensor fits one
constexpr int64_t kMaxGrid = ((int64_t)1 << 31) / kThreads;
static_assert(haste::kParamValuesMax / kChunk <= kMaxGrid, "one launch");

}  // namespace

namespace haste {

size_t grad_norm_ws(const haste_param_t *p, int64_t n) {
    const int64_t chunk = norm_chunk(p, n);
    int64_t parts = 0;
    for (int64_t k = 0; k < n; ++k) parts += cdiv(p[k].n, chunk);
    return (size_t)(parts > 0 ? parts : 1) * 8;
}

hipError_t grad_norm(const haste_param_t *p, int64_t n, float max_norm, float *out, void *ws, hipStream_t s) {
    double *part = (double *)ws;
    int64_t parts = 0;
    const int64_t chunk = norm_chunk(p, n);
    NormList l;
    l.chunk = (int32_t)chunk;
    l.count = 0;
    l.bf16[0] = l.bf16[1] = l.bf16[2] = 0;
    int64_t grid = 0;
    for (int64_t k = 0; k <= n; ++k) {
        if (k < n && p[k].n == 0) continue;
        const int64_t c = k < n ? cdiv(p[k].n, chunk) : 0;
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

// The updated arrays' addresses in an open hash table: on the stack for up to 512 tensors, for more in host memory, so
// that every address is looked up once (65536 tensors in 2.1 ms; 31 where a table of 512 was filled again and again).
int64_t adamw_repeated(const haste_param_t *p, int64_t n) {
    constexpr int kOnStack = 512;
    const void *stack[8 * kOnStack];                 // 5 addresses a tensor at most
    int bits = 6;
    while (((int64_t)1 << bits) < 8 * n) ++bits;
    const void **slot = stack;
    if (n > kOnStack) {
        slot = static_cast<const void **>(calloc((size_t)1 << bits, sizeof(void *)));
        if (!slot) return -2;
    } else {
        for (int i = 0; i < 1 << bits; ++i) slot[i] = nullptr;
    }
    int64_t found = -1;
    for (int64_t k = 0; k < n && found < 0; ++k) {
        if (p[k].n == 0) continue;
        const void *a[5] = {p[k].W, p[k].W32, p[k].m, p[k].v, p[k].state_bits == 8 ? p[k].scale : nullptr};
        for (const void *x : a) {
            if (!x) continue;
            uint32_t h = (uint32_t)(((uint64_t)(uintptr_t)x * 0x9E3779B97F4A7C15ull) >> (64 - bits));
            while (slot[h] && slot[h] != x) h = (h + 1) & ((1u << bits) - 1);
            if (slot[h]) found = k;
            slot[h] = x;
        }
    }
    if (slot != stack) free(slot);
    return found;
}

// Gradients and moments are not used again before the next step and go past the caches.  So do weights, but for
// lists that half of the memory-side cache holds: those go through it, and the next forward pass finds them there (58M
// bf16 weights, the step and a read of the weights behind it, past the caches and through them: 257 and 241 us with fp32
// moments, 350 and 319 with fp32 copies too, 155 and 147 with 8-bit moments.  The step alone, where three models take
// turns and none finds its weights: 238 either way, 299 and 314, 127 and 128.  233 MB of fp32 weights: 365 either way).
constexpr int64_t kKeepBytes = (int64_t)128 << 20;

hipError_t adamw(const haste_param_t *p, int64_t n, const haste_adamw_opts_t &o, hipStream_t s) {
    StepList l;
    int64_t bytes = 0, total = 0;
    for (int64_t k = 0; k < n; ++k) {
        bytes += p[k].n * (p[k].dtype == HASTE_DTYPE_BF16 ? 2 : 4);
        total += p[k].n;
    }
    // launches that leave most of the chip's wave slots empty take half of a chunk a workgroup, one run a lane: 211
    // tensors of 3M values in three launches 22.0 us and 20.4 so, but 4M in one launch 18.2 and 19.6
    const int64_t chunk = total <= cdiv(n, kListMax) * ((int64_t)1 << 21) ? kChunk / 2 : kChunk;
    const auto kernel = bytes <= kKeepBytes ? k_adamw<true> : k_adamw<false>;
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
    l.chunk = (int32_t)chunk;
    l.count = 0;
    l.start[0] = 0;
    int64_t grid = 0;
    for (int64_t k = 0; k <= n; ++k) {
        // a run's tensors have consecutive numbers, so one of no values keeps its slot in it
        const int64_t c = k < n ? cdiv(p[k].n, chunk) : 0;
        if (l.count > 0 && (k == n || l.count == kListMax || grid + c > kMaxGrid)) {
            if (grid > 0) hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(kStepThreads), 0, s, l);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            grid = 0;
            l.count = 0;
        }
        if (k == n) break;
        if (l.count == 0) l.first = (uint32_t)k;
        StepTensor &t = l.t[l.count];
        t.put(0, p[k].W);
        t.put(1, p[k].W32);
        t.put(2, p[k].grad);
        t.put(3, p[k].m);
        t.put(4, p[k].v);
        t.put(5, p[k].state_bits == 8 ? p[k].scale : nullptr);
        t.lr_scale = p[k].lr_scale;
        t.weight_decay = p[k].weight_decay;
        const int kind = (p[k].dtype == HASTE_DTYPE_BF16 ? kBf16 : 0) | (p[k].W32 ? kMaster : 0) |
                         (p[k].grad_dtype == HASTE_DTYPE_BF16 ? kGradBf16 : 0) | (p[k].state_bits == 8 ? kBits8 : 0);
        t.last = (uint32_t)(p[k].n - (c - 1) * chunk) | (uint32_t)kind << 16;
        grid += c;
        l.start[++l.count] = (uint32_t)grid;
    }
    return hipSuccess;
}

}  // namespace haste
