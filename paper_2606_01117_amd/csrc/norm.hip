// Layer norm of rows, forward and backward, with the reduction of the gradients of weight and bias.
//
// A row belongs to a team of 16, 64, 256, 512 or 1024 threads, which hold it in registers: every value is read
// once and every sum is taken from the registers, the squares around the row's mean.  A thread holds NC runs of
// four consecutive values, TEAM runs apart.  Rows wider than kWideF, or of fewer than four values, go through a
// loop that reads them again.
//
// No load hangs on a branch (a load behind one is waited for at its end, and so one after the other): a run that
// would reach past its row starts at the row's last four values instead, and what the run before it holds too is
// masked in the sums and not stored; a row past the last is read as the last one.
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

// STREAM: past the caches, not read again
template <bool STREAM, typename V>
__device__ __forceinline__ V load_vec(const V *p) {
    if constexpr (STREAM) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool STREAM = false>
__device__ __forceinline__ Raw4<float> load4(const float *p) {
    const u32x4_t v = load_vec<STREAM>(reinterpret_cast<const u32x4_el_t *>(p));
    return {{v.x, v.y, v.z, v.w}};
}
template <bool STREAM = false>
__device__ __forceinline__ Raw4<bf16_t> load4(const bf16_t *p) {
    const u32x2_t v = load_vec<STREAM>(reinterpret_cast<const u32x2_el_t *>(p));
    return {{v.x, v.y}};
}
__device__ __forceinline__ void unpack4(const Raw4<float> &r, float (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(r.w[j]);
}
__device__ __forceinline__ void unpack4(const Raw4<bf16_t> &r, float (&v)[4]) {
    v[0] = __uint_as_float(r.w[0] << 16), v[1] = __uint_as_float(r.w[0] & 0xffff0000u);
    v[2] = __uint_as_float(r.w[1] << 16), v[3] = __uint_as_float(r.w[1] & 0xffff0000u);
}
__device__ __forceinline__ void store4(float *p, const float (&v)[4]) {
    const u32x4_t w = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    *reinterpret_cast<u32x4_el_t *>(p) = w;
}
__device__ __forceinline__ void store4(bf16_t *p, const float (&v)[4]) {
    const u32x2_t w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    *reinterpret_cast<u32x2_el_t *>(p) = w;
}

// A run of a row of F values: it starts at the value `at`, and its own values are those from `skip` on.
struct Run {
    int at, skip;
    __device__ __forceinline__ Run(int run, int F) {
        const int f = 4 * run;
        at = f < F - 4 ? f : F - 4;
        skip = f - at;                          // 0, of a last one 1 .. 3, of one past the row 4 or more
    }
    __device__ __forceinline__ bool any() const { return skip < 4; }
};
// stores the run; its neighbour's values, which it holds too, are the same
template <typename T>
__device__ __forceinline__ void store4(T *row, const Run &r, const float (&v)[4]) {
    if (r.any()) store4(row + r.at, v);
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
// X is stored through the caches: whoever reads it next finds it there (65536 x 768 bf16: 33 us past them instead
// of 38, but with the product X W of 768 columns behind it 123 us instead of 119).
template <typename TH, typename TX, int TEAM, int NC>
__global__ __launch_bounds__(TEAM > 256 ? TEAM : 256) void k_ln_fwd(int64_t B, int F, const TH *H, int64_t ldh,
                                                                    const float *__restrict__ weight,
                                                                    const float *__restrict__ bias, float eps, TX *X,
                                                                    int64_t ldx, float *__restrict__ mean,
                                                                    float *__restrict__ rstd) {
    __shared__ float red[2 * 16];
    int turn = 0;
    const int t = threadIdx.x % TEAM;
    const int64_t teams = blockDim.x / TEAM, next = gridDim.x * teams;
    Raw4<TH> raw[NC];
    auto ask = [&](int64_t b) {
        const TH *h = H + (b < B ? b : B - 1) * ldh;
#pragma unroll
        for (int i = 0; i < NC; ++i) raw[i] = load4(h + Run(i * TEAM + t, F).at);
    };
    ask(blockIdx.x * teams + threadIdx.x / TEAM);
    float w[NC][4], c[NC][4];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const Run r(i * TEAM + t, F);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[i][j] = 1.0f, c[i][j] = 0.0f;
        if (weight) unpack4(load4(weight + r.at), w[i]);
        if (bias) unpack4(load4(bias + r.at), c[i]);
    }
    // every team of a workgroup goes round as often as the first one, for the barriers; a row's values are asked
    // for before the row before it is summed
    for (int64_t b0 = blockIdx.x * teams; b0 < B; b0 += next) {
        const int64_t b = b0 + threadIdx.x / TEAM;
        float v[NC][4], s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NC; ++i) unpack4(raw[i], v[i]);
        ask(b + next);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int skip = i == NC - 1 ? Run(i * TEAM + t, F).skip : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) s[0] += j < skip ? 0.0f : v[i][j];
        }
        team_sum<TEAM>(s, red, turn);
        const float mu = s[0] / (float)F;
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int skip = i == NC - 1 ? Run(i * TEAM + t, F).skip : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[i][j] -= mu;
                const float d = j < skip ? 0.0f : v[i][j];
                s[0] = __fmaf_rn(d, d, s[0]);
            }
        }
        team_sum<TEAM>(s, red, turn);
        const float rs = 1.0f / sqrtf(s[0] / (float)F + eps);
        if (b < B) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                float o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = __fmaf_rn(v[i][j] * rs, w[i][j], c[i][j]);
                store4(X + b * ldx, Run(i * TEAM + t, F), o);
            }
            if (mean && t == 0) {
                mean[b] = mu;
                rstd[b] = rs;
            }
        }
    }
}

// ---- backward ---------------------------------------------------------------------------------------
// The arrays of a backward call.
template <typename TH, typename TD>
struct Bwd {
    int64_t B;
    int F;
    const TH *H;
    int64_t ldh;
    const float *weight, *mean, *rstd;
    const TD *dX;
    int64_t lddx;
    TH *dH;
    int64_t lddh;
};

// Rows first, first + next, ... of a team: both sums of a row and its gradient from one read of H and dX; where
// WG, every thread adds its values' terms of dweight and dbias over the rows in aw and ab.  H and dX are read for
// the last time here, so rows of whole 16-byte accesses go past the caches (STREAM: 65536 x 768 bf16 55 us, 63
// through them); others share their accesses' lines with their neighbours and stay (4099 x 1003 fp32: 21.3 us
// past them, 20.3).
template <typename TH, typename TD, int TEAM, int NC, bool WG, bool STREAM>
__device__ __forceinline__ void bwd_rows(const Bwd<TH, TD> &a, int64_t b0, int64_t next, float (&aw)[NC][4],
                                         float (&ab)[NC][4]) {
    __shared__ float red[2 * 16 * 2];
    int turn = 0;
    const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM, F = a.F;
    Raw4<TH> rh[NC];
    Raw4<TD> rd[NC];
    float mu_next, rs_next;
    auto ask = [&](int64_t b) {
        const int64_t k = b < a.B ? b : a.B - 1;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const Run r(i * TEAM + t, F);
            rh[i] = load4<STREAM>(a.H + k * a.ldh + r.at);
            rd[i] = load4<STREAM>(a.dX + k * a.lddx + r.at);
        }
        mu_next = a.mean[k];
        rs_next = a.rstd[k];
    };
    // a row's values are asked for before the row before it is summed, where the registers of 1024 threads, or of 512
    // (bwd_threads), hold both.  (Where neighbouring rows share lines and there are many rows, some lines are then fetched
    // twice: 65536 x 513 bf16 54.5 us so and 49.8 without; but 3000 x 513 9.3 and 10.1, 17081 x 2049 59.9 and 65.8.)
    constexpr bool EARLY = TEAM == 1024 ? NC < 3 : !WG || NC != 4;
    if (EARLY) ask(b0 + team);
    float w[NC][4];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[i][j] = 1.0f;
            aw[i][j] = ab[i][j] = 0.0f;
        }
        if (a.weight) unpack4(load4(a.weight + Run(i * TEAM + t, F).at), w[i]);
    }
    for (; b0 < a.B; b0 += next) {
        const int64_t b = b0 + team;
        const bool in = b < a.B;
        if (!EARLY) ask(b);
        float x[NC][4], g[NC][4];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            unpack4(rh[i], x[i]);
            unpack4(rd[i], g[i]);
        }
        const float mu = mu_next, rs = rs_next;
        if (EARLY) ask(b + next);
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i][j] = (x[i][j] - mu) * rs;
        if (WG && in) {
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    aw[i][j] = __fmaf_rn(g[i][j], x[i][j], aw[i][j]);
                    ab[i][j] += g[i][j];
                }
        }
        if (!a.dH) continue;
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int skip = i == NC - 1 ? Run(i * TEAM + t, F).skip : 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[i][j] *= w[i][j];
                const float q = j < skip ? 0.0f : g[i][j], p = j < skip ? 0.0f : x[i][j];
                s[0] += q;
                s[1] = __fmaf_rn(q, p, s[1]);
            }
        }
        team_sum<TEAM>(s, red, turn);
        const float m0 = s[0] / (float)F, m1 = s[1] / (float)F;
        if (in) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                float o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = (g[i][j] - m0 - x[i][j] * m1) * rs;
                store4(a.dH + b * a.lddh, Run(i * TEAM + t, F), o);
            }
        }
    }
}

// stores a run's own values alone
__device__ __forceinline__ void store_own(float *out, const Run &r, const float (&v)[4]) {
    if (r.skip == 0) {
        store4(out + r.at, v);
        return;
    }
#pragma unroll
    for (int j = 1; j < 4; ++j)
        if (j >= r.skip) out[r.at + j] = v[j];
}

// threads of a workgroup whose threads hold so many runs in registers.  Four runs of 1024 threads, rows beyond 12288 values,
// do not quite fit their 128: 13 to 30 registers go to scratch.  (2000 x 16384 bf16 55 us, 87 with an fp32 dX; 64 and 85
// where weight is read again for each row instead, 113 and 131 in the loops for rows of any width.)
constexpr int bwd_threads(int runs) { return runs > 4 ? 512 : 1024; }

// Rows, and (part not NULL) part[workgroup][0][f] and part[workgroup][1][f], the workgroup's sums for dweight and
// dbias: its teams' terms, added in LDS run by run.
template <typename TH, typename TD, int TEAM, int NC, bool STREAM>
__global__ __launch_bounds__(bwd_threads(NC)) void k_ln_bwd(Bwd<TH, TD> a, float *__restrict__ part) {
    extern __shared__ float4 lds[];             // [teams][runs]
    const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM, teams = blockDim.x / TEAM, F = a.F;
    float aw[NC][4], ab[NC][4];
    bwd_rows<TH, TD, TEAM, NC, true, STREAM>(a, (int64_t)blockIdx.x * teams, (int64_t)gridDim.x * teams, aw, ab);
    if (!part) return;
    const int runs = (F + 3) / 4;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float *out = part + (2 * (int64_t)blockIdx.x + k) * F;
        if (teams == 1) {
#pragma unroll
            for (int i = 0; i < NC; ++i) store_own(out, Run(i * TEAM + t, F), k ? ab[i] : aw[i]);
            continue;
        }
        if (k) __syncthreads();
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int q = i * TEAM + t;
            const float *v = k ? ab[i] : aw[i];
            if (q < runs) lds[team * runs + q] = make_float4(v[0], v[1], v[2], v[3]);
        }
        __syncthreads();
        for (int q = threadIdx.x; q < runs; q += blockDim.x) {
            float4 s = lds[q];
            for (int r = 1; r < teams; ++r) {
                const float4 v = lds[r * runs + q];
                s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
            const float v[4] = {s.x, s.y, s.z, s.w};
            store_own(out, Run(q, F), v);
        }
    }
}

// Few rows, dH not in dX's place: one launch.  The workgroups from row_blocks on take eight columns each, straight
// to dweight and dbias, every thread of a column blockDim / 8 rows apart.
template <typename TH, typename TD, int TEAM, int NC>
__global__ __launch_bounds__(TEAM > 256 ? TEAM : 256) void k_ln_bwd_few(Bwd<TH, TD> a, unsigned row_blocks, float *__restrict__ dweight,
                                                     float *__restrict__ dbias, int beta) {
    constexpr int T = TEAM > 256 ? TEAM : 256;
    __shared__ float sw[T], sb[T];
    if (blockIdx.x < row_blocks) {
        const int teams = blockDim.x / TEAM;
        float aw[NC][4], ab[NC][4];
        bwd_rows<TH, TD, TEAM, NC, false, false>(a, (int64_t)blockIdx.x * teams, (int64_t)row_blocks * teams, aw, ab);
        return;
    }
    const int64_t f = (int64_t)(blockIdx.x - row_blocks) * 8 + (threadIdx.x & 7);
    float w = 0.0f, c = 0.0f;
    if (f < a.F) {
#pragma unroll 8
        for (int64_t b = threadIdx.x >> 3; b < a.B; b += blockDim.x >> 3) {
            const float d = load_f32(a.dX + b * a.lddx, f);
            w = __fmaf_rn(d, (load_f32(a.H + b * a.ldh, f) - a.mean[b]) * a.rstd[b], w);
            c += d;
        }
    }
    sw[threadIdx.x] = w;
    sb[threadIdx.x] = c;
    for (unsigned n = blockDim.x / 2; n >= 8; n /= 2) {
        __syncthreads();
        if (threadIdx.x < n) {
            sw[threadIdx.x] = w += sw[threadIdx.x + n];
            sb[threadIdx.x] = c += sb[threadIdx.x + n];
        }
    }
    if (threadIdx.x >= 8 || f >= a.F) return;
    if (dweight) dweight[f] = beta ? dweight[f] + w : w;
    if (dbias) dbias[f] = beta ? dbias[f] + c : c;
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
// One value a load: right for every width, and far from the memory's rate (2000 x 20000 bf16: forward 104 us, backward
// 139; 30 and 45 at a copy's rate).  The layer's rows have hundreds of values.
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
constexpr int64_t kWideF = 16384;      // rows beyond it are not held in registers
bool held(int64_t F) { return F >= 4 && F <= kWideF; }
constexpr int kMaxRowBlocks = 65536;   // workgroups of the kernels for them; more rows go round

// The team that holds a row in few registers a thread, forward and backward (which adds up terms in registers too).
constexpr int fwd_team(int64_t F) { return F <= 256 ? 16 : F <= 1024 ? 64 : F <= 4096 ? 256 : 1024; }
constexpr int bwd_team(int64_t F) { return F <= 256 ? 16 : F <= 1024 ? 64 : F <= 2048 ? 256 : F <= 4096 ? 512 : 1024; }
constexpr int64_t runs_of(int64_t F, int team) { return (F + 4 * team - 1) / (4 * team); }

// Where no more than three quarters of its runs were filled, a smaller team of up to six runs a thread takes bf16 rows
// (39024 x 1025 bf16: forward 56 us and 37, backward 90 and 58; 8000 x 5000: 44 and 34, 69 and 50).  Rows of fp32 alone
// are bound by memory with the runs half empty too, and slower in more registers (31250 x 1280: forward 58 and 61,
// backward, where H's type decides, 91 and 100).
constexpr int pick_team(int64_t F, int team, bool bf16) {
    const int small = team == 1024 || team == 512 ? 256 : team == 256 ? 64 : 16;
    return bf16 && team > 16 && 4 * F <= 3 * (4 * team * runs_of(F, team)) && runs_of(F, small) <= 6 ? small : team;
}

// The teams of both passes: bf16 as pick_team takes it.
template <bool BF16>
struct Forward {
    static constexpr int team(int64_t F) { return pick_team(F, fwd_team(F), BF16); }
};
template <bool BF16>
struct Backward {
    static constexpr int team(int64_t F) { return pick_team(F, bwd_team(F), BF16); }
};

// a width that a pass gives to this team in this many runs: kernels are built for these alone
template <typename PASS>
constexpr bool taken(int team, int runs) {
    for (int64_t F = 4 * team * (runs - 1) + 1; F <= 4 * team * runs && F <= kWideF; ++F)
        if (F >= 4 && PASS::team(F) == team) return true;
    return false;
}

// f(team, runs of four values a thread), both as constants
template <typename PASS, int TEAM, int RUNS, typename F>
void with_runs(int64_t n, F &&f) {
    if constexpr (RUNS <= 6) {
        if (n != RUNS) return with_runs<PASS, TEAM, RUNS + 1>(n, f);
        if constexpr (taken<PASS>(TEAM, RUNS)) f(std::integral_constant<int, TEAM>{}, std::integral_constant<int, RUNS>{});
    }
}
template <typename PASS, typename F>
void with_team(int64_t width, F &&f) {
    const int team = PASS::team(width);
    const int64_t n = runs_of(width, team);
    switch (team) {
    case 16: return with_runs<PASS, 16, 1>(n, f);
    case 64: return with_runs<PASS, 64, 1>(n, f);
    case 256: return with_runs<PASS, 256, 1>(n, f);
    case 512: return with_runs<PASS, 512, 1>(n, f);
    default: return with_runs<PASS, 1024, 1>(n, f);
    }
}

// The backward kernel's workgroups.  Each leaves one row of sums, so there are no more than CUs, and a CU's rows
// share its workgroup's teams, up to bwd_threads of its registers, about four rows a team at least (one, two or four
// rows a team are alike, 4099 x 1003 fp32 16.9 to 16.3 us; in up to 1024 workgroups of a row a team 20.3).
struct BwdShape {
    int team, threads;
    int64_t blocks;
};
BwdShape bwd_shape(int64_t B, int64_t F, int32_t dtype_h) {
    const int team = dtype_h == HASTE_DTYPE_BF16 ? Backward<true>::team(F) : Backward<false>::team(F);
    const int most = bwd_threads((int)runs_of(F, team));
    int threads = team > 256 ? team : 256;
    while (threads < most && B > (int64_t)256 * 4 * (threads / team)) threads *= 2;
    const int64_t want = haste::cdiv(B, threads / team);
    return {team, threads, want < 256 ? want : 256};
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
            if (!held(F)) {
                hipLaunchKernelGGL((k_ln_fwd_wide<TH, TX>), dim3((unsigned)(B < kMaxRowBlocks ? B : kMaxRowBlocks)),
                                   dim3(kThreads), 0, s, B, F, (const TH *)H, ldh, weight, bias, eps, (TX *)X, ldx, mean, rstd);
                return;
            }
            with_team<Forward<sizeof(TH) == 2 || sizeof(TX) == 2>>(F, [&](auto team, auto nc) {
                // 16 waves a CU, which are all there at once, and 32 of teams that wait for each other (65536 x 768
                // bf16 38.9 us with 16, 40.2 with 32; 8192 x 8192 63.7 and 51.8)
                const int threads = team > 256 ? (int)team : 256;
                const int64_t want = cdiv(B, threads / team), most = team > 256 ? 512 : 1024;
                hipLaunchKernelGGL((k_ln_fwd<TH, TX, team, nc>), dim3((unsigned)(want < most ? want : most)), dim3(threads), 0,
                                   s, B, (int)F, (const TH *)H, ldh, weight, bias, eps, (TX *)X, ldx, mean, rstd);
            });
        });
    });
    return hipGetLastError();
}

// Rows whose column sums a second pass over them forms, in the same launch, as fast as a second launch would add partial
// sums.  A workgroup of that pass takes eight columns, so it fetches lines that its neighbours fetch too, and of wide
// rows' teams it leaves threads without a row: it is as good up to 1.3M to 2.1M values, by the team's threads.  (us in one
// launch and in two, bf16 rows unless noted: 512 x 768 5.3 and 6.4; 512 x 2048 8.1 and 9.0, x 4096 15.7 and 12.2, x 8192
// 30.1 and 18.8; 300 x 5000 11.1 and 14.2, 400 x 5000 14.1 and 14.3, 512 x 6144 20.1 and 16.0; fp32 200 x 5000 12.4 and
// 13.5, 400 x 5000 17.4 and 15.5.  Below that the second launch costs the host 2.6: 64 x 8192 10.3 and 12.0 with it.)
bool ln_bwd_few(int64_t B, int64_t F, int32_t dtype_h) {
    if (B > 512 || !held(F)) return false;
    const int threads = bwd_shape(B, F, dtype_h).threads;
    return B * F <= (int64_t)(threads == 256 ? 8 : threads == 512 ? 6 : 5) << 18;
}

size_t ln_bwd_ws(int64_t B, int64_t F) {
    int64_t parts = wide_parts(B);
    if (held(F)) {
        const int64_t a = bwd_shape(B, F, HASTE_DTYPE_F32).blocks, b = bwd_shape(B, F, HASTE_DTYPE_BF16).blocks;
        parts = a > b ? a : b;
    }
    return (size_t)(parts * 2 * F * 4);
}

hipError_t ln_bwd(int64_t B, int64_t F, int32_t dtype_h, const void *H, int64_t ldh, const float *weight,
                  const float *mean, const float *rstd, int32_t dtype_dx, const void *dX, int64_t lddx, void *dH,
                  int64_t lddh, float *dweight, float *dbias, int beta, void *ws, hipStream_t s) {
    float *part = (float *)ws;
    const bool wg = dweight || dbias;
    const BwdShape n = held(F) ? bwd_shape(B, F, dtype_h) : BwdShape{};
    const int64_t parts = !held(F) ? wide_parts(B) : n.blocks;
    const bool few = wg && dH != dX && ln_bwd_few(B, F, dtype_h);
    with_type(dtype_h, [&](auto th) {
        with_type(dtype_dx, [&](auto td) {
            typedef decltype(th) TH;
            typedef decltype(td) TD;
            if (!held(F)) {
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
            const auto whole = [](const void *p, int64_t ld, int64_t size) {
                return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) % 16 == 0;
            };
            const bool stream = whole(H, ldh, sizeof(TH)) && whole(dX, lddx, sizeof(TD));
            const Bwd<TH, TD> a = {B, (int)F, (const TH *)H, ldh, weight, mean, rstd, (const TD *)dX, lddx, (TH *)dH, lddh};
            with_team<Backward<sizeof(TH) == 2>>(F, [&](auto team, auto nc) {
                const int teams = n.threads / team;
                const size_t lds = wg && teams > 1 ? (size_t)teams * cdiv(F, 4) * 16 : 0;
                if (few) {
                    const unsigned rows = dH ? (unsigned)n.blocks : 0;
                    hipLaunchKernelGGL((k_ln_bwd_few<TH, TD, team, nc>), dim3(rows + (unsigned)cdiv(F, 8)), dim3(n.threads), 0, s,
                                       a, rows, dweight, dbias, beta);
                } else if (stream) {
                    hipLaunchKernelGGL((k_ln_bwd<TH, TD, team, nc, true>), dim3((unsigned)n.blocks), dim3(n.threads), lds, s, a,
                                       wg ? part : nullptr);
                } else {
                    hipLaunchKernelGGL((k_ln_bwd<TH, TD, team, nc, false>), dim3((unsigned)n.blocks), dim3(n.threads), lds, s, a,
                                       wg ? part : nullptr);
                }
            });
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (wg && !few)
        hipLaunchKernelGGL(k_ln_wsum, dim3((unsigned)cdiv(2 * F, kWave)), dim3(1024), 0, s, part, parts, F, dweight, dbias, beta);
    return hipGetLastError();
}

}  // namespace haste
