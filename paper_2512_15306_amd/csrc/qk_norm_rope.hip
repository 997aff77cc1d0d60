// Queries and keys of a QKV projection: RMSNorm of every head and the rotation by position in one pass, and the gradient of both.
//
//   n[i] = x[i] rstd w[i],  rstd = 1 / sqrt(mean x^2 + eps)  over the D values of a head (without weights: n = x)
//   pairs (a, b) of the first `rot` values: i and i + rot/2, or neighbours;   y_a = n_a cos t - n_b sin t,  y_b = n_b cos t + n_a sin t
//   backward: g = the same rotation by -t of dy;  dw += g x rstd;  dx = rstd (g w - x rstd mean(g w x rstd))
//
// HBM-bound: 2 bytes read and 2 written per value (backward 4 and 2).  What there is to compute is arranged around the angles: t = position f mod one turn is
// a product of 64-bit whole numbers, with the frequency as a 64-bit fraction of a turn (off by 2^-52 of itself and 2^-64 of a turn at most): the product is exact, so far positions lose no more than that times the position, and no
// table is read; a sine and a cosine by their series then cost about 25 instructions, which a lane pays once per token for its four pairs and uses
// for all heads.  For that a wave takes a token and walks over its heads, as many at a time as fit (four of 128 values), eight
// values a lane in two pieces of 8 bytes that hold both halves of its pairs: no exchange between lanes but the sums of a head.
// The sums of dw stay in a lane's registers over all tokens and heads of its wave; each workgroup leaves one row of them, which a second kernel adds
// in the order of the workgroups (no atomics).
//
// Heads of 128 values, buffers changing from call to call.  Forward: 8192 tokens of 28 + 4 heads (135 MB) 25.4 us, 5.3 TB/s; 32 tokens 4 us, one trip to memory and back behind the angles.  Backward: 8192 tokens of
// 40 + 8 (337 MB) 75 us, 4.5 TB/s, of which the second kernel's 4; 1777 tokens of 9 + 3 heads of 80 (12 MB) 11.5 us: two launches, each a chain of waits.
#include "api_checks.h"
#include "llmq_device.h"

namespace llmq {

typedef uint16_t u16;

struct QkArgs {
    int64_t M;
    int Hq, Hkv, D, rot, interleaved;
    const u16* x;                               // [M, Hq + 2 Hkv, D]
    const u16 *wq, *wk;                         // NULL: no norm
    const int64_t* positions;
    const double* inv_freq;
    float eps;
    float* rstd;                                // [M, Hq + Hkv]; written by the forward pass if not NULL, read by the backward pass
    u16 *q, *k;                                 // forward: outputs; backward: gradients of the outputs (not written)
    const u16* dv;                              // backward: NULL: V's gradient is in its place already
    u16* dx;                                    // backward: [M, Hq + 2 Hkv, D]
    int64_t x_stride, q_stride, k_stride, dv_stride, dx_stride;        // elements from row to row
    float* dw_partial;                          // backward: a row of 2 D sums for each workgroup, or NULL
    unsigned* amax_partial;                     // backward: a word for each workgroup, or NULL
    int split;                                  // waves that share a token
};

// A frequency in radians as a 64-bit fraction of a turn per position (whole turns do not matter)
__device__ inline uint64_t turns_of(double inv_freq) {
    double t = inv_freq * 0.15915494309189533577;            // 1 / (2 pi)
    t -= __builtin_floor(t);
    t = t < 1.0 ? t * 4294967296.0 : 0.0;                    // (the difference may round to a whole turn)
    const unsigned hi = (unsigned)t, lo = (unsigned)((t - (double)hi) * 4294967296.0);
    return ((uint64_t)hi << 32) | lo;
}

// Cosine and sine of a fraction of a turn: to the nearest quarter, the rest (at most pi/4) by the Taylor series, whose first missing terms are
// x^11/11! < 2e-9 and x^10/10! < 3e-8.
__device__ inline void cos_sin(uint64_t turns, float& c, float& s) {
    const unsigned top = (unsigned)(turns >> 32);
    const unsigned quarter = (top + 0x20000000u) >> 30;
    const float x = (float)(int)(top - (quarter << 30)) * 1.46291807926715968e-9f;         // 2 pi / 2^32
    const float z = x * x;
    const float sine = x * __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), 1.0f);
    const float cosine = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.0f / 40320, -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    const bool odd = quarter & 1;
    const float a = odd ? sine : cosine, b = odd ? cosine : sine;
    c = ((quarter + 1) & 2) ? -a : a;
    s = (quarter & 2) ? -b : b;
}

// Sum over groups of G neighbouring lanes, in all of them
template <int G>
__device__ inline float group_sum(float v) {
    auto dpp = [&](auto ctrl) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xF, 0xF, false)); };
    v += dpp(std::integral_constant<int, 0xB1>{});           // quad_perm [1,0,3,2]
    v += dpp(std::integral_constant<int, 0x4E>{});           // quad_perm [2,3,0,1]
    v += dpp(std::integral_constant<int, 0x141>{});          // row_half_mirror
    if constexpr (G >= 16) v += dpp(std::integral_constant<int, 0x140>{});      // row_mirror
    if constexpr (G >= 32) { const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false); v = __uint_as_float(r[0]) + __uint_as_float(r[1]); }
    if constexpr (G >= 64) { const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false); v = __uint_as_float(r[0]) + __uint_as_float(r[1]); }
    return v;
}

// 1 / sqrt(x): the hardware's, to within a unit in the last place, and a Newton step.  The instruction takes subnormals for zeros, so those are brought up first (heads of values below 2^-63 without eps).
__device__ inline float inverse_root(float x) {
    const bool subnormal = x < 0x1p-126f;
    const float y = __builtin_amdgcn_rsqf(subnormal ? x * 0x1p24f : x) * (subnormal ? 0x1p12f : 1.0f);
    const float e = __builtin_fmaf(-x * y, y, 1.0f);
    return e == e ? __builtin_fmaf(0.5f * y, e, y) : y;      // (0 and infinity: y is infinity and 0)
}

// Eight values of a head: two pieces of four
struct Eight { v2u lo, hi; };
__device__ inline void unpack(const Eight& e, float (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        f[2 * j] = __uint_as_float(e.lo[j] << 16);
        f[2 * j + 1] = __uint_as_float(e.lo[j] & 0xFFFF0000u);
        f[4 + 2 * j] = __uint_as_float(e.hi[j] << 16);
        f[5 + 2 * j] = __uint_as_float(e.hi[j] & 0xFFFF0000u);
    }
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
__device__ inline unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector(v2f{a, b}, bf16x2)); }
__device__ inline Eight pack(const float (&f)[8]) {
    return Eight{v2u{pack2(f[0], f[1]), pack2(f[2], f[3])}, v2u{pack2(f[4], f[5]), pack2(f[6], f[7])}};
}

// The lane's place among the G lanes of a head: its two pieces' columns and its angles' frequencies
template <int G, bool NEIGHBOURS>
struct Place {
    int l, sub;                                  // lane of the head; head among those of a pass
    bool there, turned;
    int lo, hi;                                  // first columns of the pieces
    unsigned off_lo, off_hi;                     // their places behind the first head of a pass
    uint64_t f[4];
    __device__ Place(const QkArgs& a) {
        const int lane = threadIdx.x & (kWave - 1);
        l = lane % G, sub = lane / G;
        there = 8 * l < a.D;
        turned = 8 * l < a.rot;
        lo = turned && !NEIGHBOURS ? 4 * l : 8 * l;       // (the values behind the turned ones start at a multiple of 8 as well)
        hi = turned && !NEIGHBOURS ? 4 * l + a.rot / 2 : 8 * l + 4;
        off_lo = (unsigned)(sub * a.D + lo), off_hi = (unsigned)(sub * a.D + hi);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = turned ? turns_of(a.inv_freq[4 * l + j]) : 0;
    }
    __device__ Eight weights(const u16* p) const { return Eight{*reinterpret_cast<const v2u*>(p + lo), *reinterpret_cast<const v2u*>(p + hi)}; }
    // p: the first head of the pass (the same for the whole wave)
    __device__ Eight load(const u16* p) const {
        return Eight{__builtin_nontemporal_load(reinterpret_cast<const v2u*>(p + off_lo)), __builtin_nontemporal_load(reinterpret_cast<const v2u*>(p + off_hi))};
    }
    template <bool STREAM>
    __device__ void store(u16* p, const Eight& e) const {
        store_hinted<STREAM>(e.lo, reinterpret_cast<v2u*>(p + off_lo));
        store_hinted<STREAM>(e.hi, reinterpret_cast<v2u*>(p + off_hi));
    }
    // SIGN 1: by the angles, -1: back
    template <int SIGN>
    __device__ void turn(const float (&c)[4], const float (&s)[4], float (&v)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            constexpr int kStep = NEIGHBOURS ? 1 : 4;
            const int i = NEIGHBOURS ? 2 * j : j;
            const float x = v[i], y = v[i + kStep];
            v[i] = __builtin_fmaf(x, c[j], SIGN > 0 ? -y * s[j] : y * s[j]);
            v[i + kStep] = __builtin_fmaf(y, c[j], SIGN > 0 ? x * s[j] : -x * s[j]);
        }
    }
    __device__ void angles(int64_t position, float (&c)[4], float (&s)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) cos_sin((uint64_t)position * f[j], c[j], s[j]);
    }
};

constexpr int kQkThreads = 256, kQkWaves = kQkThreads / kWave;
constexpr int kQkBwdThreads = 256, kQkBwdWaves = kQkBwdThreads / kWave;

// The passes of a wave over the heads of a token: first all of the queries, then all of the keys, so that a pass has one weight and one base address.
// each(f): f(tag, first, last, head0) for the wave's share of the queries' passes, then of the keys'; tag::value: whether they are queries.
template <int G>
struct Passes {
    static constexpr int kHeads = kWave / G;
    int queries, first, last;
    __device__ Passes(const QkArgs& a, int part) {
        queries = (a.Hq + kHeads - 1) / kHeads;
        const int all = queries + (a.Hkv + kHeads - 1) / kHeads, per_part = (all + a.split - 1) / a.split;
        first = part * per_part;
        last = first + per_part < all ? first + per_part : all;
    }
    template <class F>
    __device__ __attribute__((always_inline)) void each(F&& f) const {
        if (first < queries) f(std::true_type{}, first, last < queries ? last : queries);
        if (last > queries) f(std::false_type{}, (first > queries ? first : queries) - queries, last - queries);
    }
};
// Batches of N passes [first, last): while one is computed the next is on its way.
template <class Batch, int N, class Request, class Compute>
__device__ __attribute__((always_inline)) inline void pipelined(int first, int last, Request&& request, Compute&& compute) {
    Batch in[2][N];
    request(first, in[0]);
    for (int p = first; p < last; p += 2 * N) {
        request(p + N, in[1]);
        compute(p, in[0]);
        request(p + 2 * N, in[0]);
        compute(p + N, in[1]);
    }
}

template <int G, bool NORM, bool NEIGHBOURS>
__global__ __launch_bounds__(kQkThreads) void qk_fwd_kernel(const QkArgs a) {
    const int wave = blockIdx.x * kQkWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = gridDim.x * kQkWaves;
    const Place<G, NEIGHBOURS> at(a);
    const Passes<G> ps(a, wave % a.split);
    const int heads = a.Hq + a.Hkv;
    const float per_d = 1.0f / (float)a.D;
    float wq[8], wk[8];
    if constexpr (NORM) {
        if (at.there) { unpack(at.weights(a.wq), wq); unpack(at.weights(a.wk), wk); }
    }
    // (one / two / four passes in a batch, with six, six and five workgroups to a CU, back to back on the same buffers: 8192 tokens of 28 + 4 heads of 128 28.0 / 27.4 / 29.0 us, 512 of them 4.9 / 5.2 / 6.0, 2048 12.3 / 11.7 / 11.9)
    constexpr int kAtOnce = 2;
    for (int64_t m = wave / a.split; m < a.M; m += waves / a.split) {
        float c[4], s[4];
        at.angles(a.rot ? a.positions[m] : 0, c, s);
        ps.each([&](auto tag, int first, int last) __attribute__((always_inline)) {
            constexpr bool query = decltype(tag)::value;
            const int count = query ? a.Hq : a.Hkv, head0 = query ? 0 : a.Hq;
            const u16* x = a.x + m * a.x_stride + (int64_t)head0 * a.D;
            u16* y = query ? a.q + m * a.q_stride : a.k + m * a.k_stride;
            auto request = [&](int p0, Eight (&in)[kAtOnce]) __attribute__((always_inline)) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int head = (p0 + u) * ps.kHeads;
                    if (p0 + u < last && at.there && head + at.sub < count) in[u] = at.load(x + (int64_t)head * a.D);
                }
            };
            auto compute = [&](int p0, const Eight (&in)[kAtOnce]) __attribute__((always_inline)) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int head = (p0 + u) * ps.kHeads;
                    if (p0 + u < last) {
                        const bool mine = at.there && head + at.sub < count;
                        float v[8];
                        unpack(in[u], v);
                        if constexpr (NORM) {
                            float sum = 0.0f;
#pragma unroll
                            for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(v[j], v[j], sum);
                            const float rstd = inverse_root(__builtin_fmaf(group_sum<G>(mine ? sum : 0.0f), per_d, a.eps));
#pragma unroll
                            for (int j = 0; j < 8; ++j) v[j] = v[j] * rstd * (query ? wq[j] : wk[j]);
                            if (a.rstd && at.l == 0 && mine) a.rstd[m * heads + head0 + head + at.sub] = rstd;
                        }
                        at.template turn<1>(c, s, v);
                        if (mine) at.template store<false>(y + (int64_t)head * a.D, pack(v));
                    }
                }
            };
            pipelined<Eight, kAtOnce>(first, last, request, compute);
        });
    }
}

__device__ inline void track(unsigned& mag, const Eight& e) { mag = pk_max_mag(pk_max_mag(pk_max_mag(pk_max_mag(mag, e.lo[0]), e.lo[1]), e.hi[0]), e.hi[1]); }

// The gradient of V on its way to its place, V values a lane at once, `step` lanes side by side
template <int V>
__device__ inline void move_v(const QkArgs& a, int64_t m, int first, int step, unsigned& mag) {
    const int64_t n = (int64_t)a.Hkv * a.D;
    u16* to = a.dx + m * a.dx_stride + (int64_t)(a.Hq + a.Hkv) * a.D;
    const u16* from = a.dv ? a.dv + m * a.dv_stride : to;
    if (!a.dv && !a.amax_partial) return;
    for (int64_t i = (int64_t)first * V; i < n; i += (int64_t)step * V) {
        if constexpr (V == 4) {
            const v2u v = *reinterpret_cast<const v2u*>(from + i);
            mag = pk_max_mag(pk_max_mag(mag, v[0]), v[1]);
            if (a.dv) *reinterpret_cast<v2u*>(to + i) = v;
        } else {
            const u16 v = from[i];
            mag = pk_max_mag(mag, v);
            if (a.dv) to[i] = v;
        }
    }
}

template <int THREADS>
__device__ inline void leave_absmax(const QkArgs& a, unsigned mag, unsigned* s_part) {
    if (!a.amax_partial) return;
    mag = (mag & 0xFFFFu) > (mag >> 16) ? mag & 0xFFFFu : mag >> 16;
    mag = block_max_u32<THREADS>(mag, s_part);
    if (threadIdx.x == 0) a.amax_partial[blockIdx.x] = mag;
}

template <int G, bool NORM, bool NEIGHBOURS, bool STREAM>
__global__ __launch_bounds__(kQkBwdThreads) void qk_bwd_kernel(const QkArgs a) {
    __shared__ float s_dw[NORM ? kQkBwdWaves : 1][NORM ? 2 * 8 * G : 1];
    __shared__ unsigned s_part[kQkBwdWaves];
    const int wave = blockIdx.x * kQkBwdWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = gridDim.x * kQkBwdWaves, part = wave % a.split;
    const Place<G, NEIGHBOURS> at(a);
    const Passes<G> ps(a, part);
    const int heads = a.Hq + a.Hkv;
    const float per_d = 1.0f / (float)a.D;
    float wq[8], wk[8], dwq[8] = {}, dwk[8] = {};
    unsigned mag = 0;
    if constexpr (NORM) {
        if (at.there) { unpack(at.weights(a.wq), wq); unpack(at.weights(a.wk), wk); }
    }
    struct In { Eight x, dy; float rstd; };
    constexpr int kAtOnce = 2;
    for (int64_t m = wave / a.split; m < a.M; m += waves / a.split) {
        float c[4], s[4];
        at.angles(a.rot ? a.positions[m] : 0, c, s);
        ps.each([&](auto tag, int first, int last) __attribute__((always_inline)) {
            constexpr bool query = decltype(tag)::value;
            const int count = query ? a.Hq : a.Hkv, head0 = query ? 0 : a.Hq;
            const u16* dy = query ? a.q + m * a.q_stride : a.k + m * a.k_stride;
            const u16* x = NORM ? a.x + m * a.x_stride + (int64_t)head0 * a.D : nullptr;
            const float* rstd = NORM ? a.rstd + m * heads + head0 : nullptr;
            u16* dx = a.dx + m * a.dx_stride + (int64_t)head0 * a.D;
            auto request = [&](int p0, In (&in)[kAtOnce]) __attribute__((always_inline)) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int head = (p0 + u) * ps.kHeads;
                    if (p0 + u < last) {
                        in[u] = In{};                        // (what is not there adds nothing to the sums)
                        if (at.there && head + at.sub < count) {
                            in[u].dy = at.load(dy + (int64_t)head * a.D);
                            if constexpr (NORM) {
                                in[u].x = at.load(x + (int64_t)head * a.D);
                                in[u].rstd = rstd[head + at.sub];
                            }
                        }
                    }
                }
            };
            auto compute = [&](int p0, const In (&in)[kAtOnce]) __attribute__((always_inline)) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int head = (p0 + u) * ps.kHeads;
                    if (p0 + u < last) {
                        float g[8];
                        unpack(in[u].dy, g);
                        at.template turn<-1>(c, s, g);
                        if constexpr (NORM) {
                            float n[8], sum = 0.0f;
                            unpack(in[u].x, n);
                            const float r = in[u].rstd;
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                n[j] *= r;
                                if constexpr (query) dwq[j] = __builtin_fmaf(g[j], n[j], dwq[j]);
                                else dwk[j] = __builtin_fmaf(g[j], n[j], dwk[j]);
                                g[j] *= query ? wq[j] : wk[j];
                                sum = __builtin_fmaf(g[j], n[j], sum);
                            }
                            const float mean = group_sum<G>(at.there ? sum : 0.0f) * per_d;
#pragma unroll
                            for (int j = 0; j < 8; ++j) g[j] = r * __builtin_fmaf(-n[j], mean, g[j]);
                        }
                        if (at.there && head + at.sub < count) {
                            const Eight out = pack(g);
                            track(mag, out);
                            at.template store<STREAM>(dx + (int64_t)head * a.D, out);
                        }
                    }
                }
            };
            pipelined<In, kAtOnce>(first, last, request, compute);
        });
        move_v<4>(a, m, (threadIdx.x & (kWave - 1)) + part * kWave, a.split * kWave, mag);
    }
    if constexpr (NORM) {
        if (a.dw_partial) {
            // the heads of a pass first, then the waves
#pragma unroll
            for (int j = 0; j < 8; ++j) {
#pragma unroll
                for (int step = G; step < kWave; step *= 2) {
                    dwq[j] += __shfl_xor(dwq[j], step);
                    dwk[j] += __shfl_xor(dwk[j], step);
                }
                const int col = j < 4 ? at.lo + j : at.hi + j - 4;
                if (at.sub == 0 && at.there) {
                    s_dw[threadIdx.x / kWave][col] = dwq[j];
                    s_dw[threadIdx.x / kWave][a.D + col] = dwk[j];
                }
            }
            __syncthreads();
            for (int i = threadIdx.x; i < 2 * a.D; i += kQkBwdThreads) {
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kQkBwdWaves; ++w) sum += s_dw[w][i];
                a.dw_partial[(int64_t)blockIdx.x * 2 * a.D + i] = sum;
            }
        }
    }
    leave_absmax<kQkBwdThreads>(a, mag, s_part);
}

// ---- Any head size, stride and alignment: a wave for each head of a token, value by value, twice over the head.  Pair p of the turned values, or the single value
// behind them.
struct PairCols { int a, b; };
__device__ inline PairCols pair_cols(const QkArgs& a, int p) { return a.interleaved ? PairCols{2 * p, 2 * p + 1} : PairCols{p, p + a.rot / 2}; }
__device__ inline float value(const u16* p, int i) { return __uint_as_float((unsigned)p[i] << 16); }
__device__ inline u16 rounded(float f) { return __builtin_bit_cast(u16, (__bf16)f); }

template <bool NORM>
__global__ __launch_bounds__(kQkThreads) void qk_fwd_any_kernel(const QkArgs a) {
    const int lane = threadIdx.x & (kWave - 1), heads = a.Hq + a.Hkv;
    const int64_t waves = (int64_t)gridDim.x * kQkWaves;
    for (int64_t at = (int64_t)blockIdx.x * kQkWaves + threadIdx.x / kWave; at < a.M * heads; at += waves) {
        const int64_t m = at / heads;
        const int head = (int)(at - m * heads);
        const u16* x = a.x + m * a.x_stride + (int64_t)head * a.D;
        u16* y = head < a.Hq ? a.q + m * a.q_stride + (int64_t)head * a.D : a.k + m * a.k_stride + (int64_t)(head - a.Hq) * a.D;
        const u16* w = head < a.Hq ? a.wq : a.wk;
        float rstd = 1.0f;
        if constexpr (NORM) {
            float sum = 0.0f;
            for (int i = lane; i < a.D; i += kWave) { const float v = value(x, i); sum = __builtin_fmaf(v, v, sum); }
            rstd = inverse_root(group_sum<kWave>(sum) / (float)a.D + a.eps);
            if (a.rstd && lane == 0) a.rstd[at] = rstd;
        }
        auto normed = [&](int i) { return NORM ? value(x, i) * rstd * value(w, i) : value(x, i); };
        for (int p = lane; p < a.rot / 2; p += kWave) {
            const PairCols col = pair_cols(a, p);
            const float u = normed(col.a), v = normed(col.b);
            float c, s;
            cos_sin((uint64_t)a.positions[m] * turns_of(a.inv_freq[p]), c, s);
            y[col.a] = rounded(__builtin_fmaf(u, c, -v * s));
            y[col.b] = rounded(__builtin_fmaf(v, c, u * s));
        }
        for (int i = a.rot + lane; i < a.D; i += kWave) y[i] = rounded(normed(i));
    }
}

// A workgroup's sums of dw lie in LDS, a row for each wave, room for the widest heads there are
constexpr int kQkAnyWidth = 1024;
template <bool NORM>
__global__ __launch_bounds__(kQkThreads) void qk_bwd_any_kernel(const QkArgs a) {
    __shared__ float s_dw[NORM ? kQkWaves : 1][NORM ? 2 * kQkAnyWidth : 1];
    __shared__ unsigned s_part[kQkWaves];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, heads = a.Hq + a.Hkv;
    const int64_t waves = (int64_t)gridDim.x * kQkWaves;
    unsigned mag = 0;
    if constexpr (NORM) {
        for (int i = lane; i < 2 * a.D; i += kWave) s_dw[wave][i] = 0.0f;      // (a lane's own columns: pairs and single values have one lane each)
        __syncthreads();
    }
    for (int64_t at = (int64_t)blockIdx.x * kQkWaves + wave; at < a.M * heads; at += waves) {
        const int64_t m = at / heads;
        const int head = (int)(at - m * heads);
        const u16* dy = head < a.Hq ? a.q + m * a.q_stride + (int64_t)head * a.D : a.k + m * a.k_stride + (int64_t)(head - a.Hq) * a.D;
        const u16* x = a.x + m * a.x_stride + (int64_t)head * a.D;
        const u16* w = head < a.Hq ? a.wq : a.wk;
        u16* dx = a.dx + m * a.dx_stride + (int64_t)head * a.D;
        const float rstd = NORM ? a.rstd[at] : 1.0f;
        // f(column, gradient of the normed value) for the columns of this lane
        auto each = [&](auto f) {
            for (int p = lane; p < a.rot / 2; p += kWave) {
                const PairCols col = pair_cols(a, p);
                const float u = value(dy, col.a), v = value(dy, col.b);
                float c, s;
                cos_sin((uint64_t)a.positions[m] * turns_of(a.inv_freq[p]), c, s);
                f(col.a, __builtin_fmaf(u, c, v * s));
                f(col.b, __builtin_fmaf(v, c, -u * s));
            }
            for (int i = a.rot + lane; i < a.D; i += kWave) f(i, value(dy, i));
        };
        float mean = 0.0f;
        if constexpr (NORM) {
            float sum = 0.0f;
            float* dw = s_dw[wave] + (head < a.Hq ? 0 : a.D);
            each([&](int i, float g) {
                const float n = value(x, i) * rstd;
                dw[i] += g * n;
                sum = __builtin_fmaf(g * value(w, i), n, sum);
            });
            mean = group_sum<kWave>(sum) / (float)a.D;
        }
        // (a pair's two gradients are read before either place is written, so dx may be dy)
        auto out = [&](int i, float g) {
            if constexpr (NORM) g = rstd * __builtin_fmaf(-value(x, i) * rstd, mean, g * value(w, i));
            const u16 o = rounded(g);
            mag = pk_max_mag(mag, o);
            dx[i] = o;
        };
        each(out);
        if (head == 0) move_v<1>(a, m, lane, kWave, mag);
    }
    if constexpr (NORM) {
        __syncthreads();
        if (a.dw_partial)
            for (int i = threadIdx.x; i < 2 * a.D; i += kQkThreads) {
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kQkWaves; ++w) sum += s_dw[w][i];
                a.dw_partial[(int64_t)blockIdx.x * 2 * a.D + i] = sum;
            }
    }
    leave_absmax<kQkThreads>(a, mag, s_part);
}

constexpr int kQkMaxBlocks = 1024;              // workgroups of the backward pass: rows of its workspace

// The workgroups' sums: a workgroup has 16 columns and 64 lanes to each, which take every 64th row in turn and are
// then added pairwise: an order that the number of rows alone decides.  The last workgroup finds the absmax.  A short
// kernel of waits: with 16 lanes to a column instead, the whole backward pass takes 0.1 us longer for 1777 tokens and
// 0.4 us for 8192.
constexpr int kFinalCols = 16, kFinalRows = 64, kFinalThreads = kFinalCols * kFinalRows;
__global__ __launch_bounds__(kFinalThreads) void qk_bwd_final_kernel(const float* dw_partial, const unsigned* amax_partial, int n, int D, float* dwq, float* dwk, int accumulate,
                                                                    float fmax, float* d_amax, float* d_scale) {
    __shared__ float s_sum[kFinalRows][kFinalCols + 1];
    __shared__ unsigned s_part[kFinalThreads / kWave];
    if (blockIdx.x == gridDim.x - 1) {
        if (!amax_partial) return;
        unsigned m = 0;
        for (int i = threadIdx.x; i < n; i += kFinalThreads) m = m > amax_partial[i] ? m : amax_partial[i];
        m = block_max_u32<kFinalThreads>(m, s_part);
        if (threadIdx.x == 0) {
            const float amax = __uint_as_float(amax_bits_from_bf16_mag(m));
            *d_amax = amax;
            if (d_scale) *d_scale = scale_of_amax(amax, fmax);
        }
        return;
    }
    const int c = threadIdx.x % kFinalCols, r = threadIdx.x / kFinalCols, col = blockIdx.x * kFinalCols + c;
    float sum = 0.0f;
    if (col < 2 * D) {
        constexpr int kAtOnce = kQkMaxBlocks / kFinalRows;   // all of a lane's loads are on their way together
        float v[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) v[k] = r + kFinalRows * k < n ? dw_partial[(int64_t)(r + kFinalRows * k) * 2 * D + col] : 0.0f;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) sum += v[k];
    }
    s_sum[r][c] = sum;
#pragma unroll
    for (int step = kFinalRows / 2; step >= 1; step /= 2) {
        __syncthreads();
        if (r < step) s_sum[r][c] += s_sum[r + step][c];
    }
    if (r == 0 && col < 2 * D) {
        float* out = col < D ? dwq : dwk;
        if (out) {
            const int i = col < D ? col : col - D;
            out[i] = accumulate ? out[i] + s_sum[0][c] : s_sum[0][c];
        }
    }
}

// ---- host side
static bool aligned8(const void* p, int64_t stride) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0 && stride % 4 == 0; }

// Lanes to a head of the vector kernels, or 0: pieces of four values have to be whole and to start at multiples of 8 bytes.
static int lanes_of_head(int D, int rot) {
    if (D % 8 != 0 || rot % 8 != 0 || D > 8 * kWave) return 0;
    return D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : 64;
}

struct QkGrid { int blocks, split; };
// A wave takes a token; where there are fewer than `wanted` waves that way, the heads of a token are shared out among 2, 4, ... of them, each of which finds the angles for itself.
// most: workgroups
static QkGrid qk_grid(int64_t M, int passes, int64_t wanted, int wg_waves, int most) {
    int split = 1;
    while (split < passes && M * split < wanted) split *= 2;
    const int64_t blocks = (M * split + wg_waves - 1) / wg_waves;
    int n = (int)(blocks < most ? blocks : most);
    if (split > wg_waves) { const int per = split / wg_waves; n = (n + per - 1) / per * per; }      // (a multiple of `split` waves)
    return {n, split};
}

static int launch_qk_fwd(QkArgs a, hipStream_t stream, int cus) {
    const int G = lanes_of_head(a.D, a.rot);
    const bool vec = G && aligned8(a.x, a.x_stride) && aligned8(a.q, a.q_stride) && aligned8(a.k, a.k_stride) && aligned8(a.wq, 0) && aligned8(a.wk, 0);
    if (!vec) {
        const int64_t blocks = (a.M * (a.Hq + a.Hkv) + kQkWaves - 1) / kQkWaves, most = (int64_t)cus * 32;
        const dim3 grid((unsigned)(blocks < most ? blocks : most));
        if (a.wq) hipLaunchKernelGGL(qk_fwd_any_kernel<true>, grid, dim3(kQkThreads), 0, stream, a);
        else hipLaunchKernelGGL(qk_fwd_any_kernel<false>, grid, dim3(kQkThreads), 0, stream, a);
    } else {
        const QkGrid g = qk_grid(a.M, (a.Hq + kWave / G - 1) / (kWave / G) + (a.Hkv + kWave / G - 1) / (kWave / G), 8 * cus, kQkWaves, cus * 6);
        a.split = g.split;
        auto launch = [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            auto with = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(g.blocks), dim3(kQkThreads), 0, stream, a); };
            if (a.wq) a.interleaved ? with(qk_fwd_kernel<L, true, true>) : with(qk_fwd_kernel<L, true, false>);
            else a.interleaved ? with(qk_fwd_kernel<L, false, true>) : with(qk_fwd_kernel<L, false, false>);
        };
        if (G == 8) launch(std::integral_constant<int, 8>{});
        else if (G == 16) launch(std::integral_constant<int, 16>{});
        else if (G == 32) launch(std::integral_constant<int, 32>{});
        else launch(std::integral_constant<int, 64>{});
    }
    return hipGetLastError() == hipSuccess ? LLMQ_OK : LLMQ_ERR_DEVICE;
}

struct QkFinal { float *dwq, *dwk; int accumulate, fmt; float *d_amax, *d_scale; };

static int launch_qk_bwd(QkArgs a, const QkFinal& f, hipStream_t stream, int cus) {
    const int G = lanes_of_head(a.D, a.rot);
    const bool vec = G && aligned8(a.q, a.q_stride) && aligned8(a.k, a.k_stride) && aligned8(a.dx, a.dx_stride) && aligned8(a.dv, a.dv_stride) &&
                     (!a.wq || (aligned8(a.x, a.x_stride) && aligned8(a.wq, 0) && aligned8(a.wk, 0)));
    int blocks;
    if (!vec) {
        const int64_t wanted = (a.M * (a.Hq + a.Hkv) + kQkWaves - 1) / kQkWaves;
        blocks = (int)(wanted < kQkMaxBlocks ? wanted : kQkMaxBlocks);
        if (a.wq) hipLaunchKernelGGL(qk_bwd_any_kernel<true>, dim3(blocks), dim3(kQkThreads), 0, stream, a);
        else hipLaunchKernelGGL(qk_bwd_any_kernel<false>, dim3(blocks), dim3(kQkThreads), 0, stream, a);
    } else {
        const QkGrid g = qk_grid(a.M, (a.Hq + kWave / G - 1) / (kWave / G) + (a.Hkv + kWave / G - 1) / (kWave / G), 4 * cus, kQkBwdWaves, 3 * cus < kQkMaxBlocks ? 3 * cus : kQkMaxBlocks);
        a.split = g.split;
        blocks = g.blocks;
        auto launch = [&](auto lanes) {
            constexpr int L = decltype(lanes)::value;
            auto with = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(g.blocks), dim3(kQkBwdThreads), 0, stream, a); };
            auto of = [&](auto stream) {
                constexpr bool ST = decltype(stream)::value;
                if (a.wq) a.interleaved ? with(qk_bwd_kernel<L, true, true, ST>) : with(qk_bwd_kernel<L, true, false, ST>);
                else a.interleaved ? with(qk_bwd_kernel<L, false, true, ST>) : with(qk_bwd_kernel<L, false, false, ST>);
            };
            // (of the pass and the quantizer of its result behind it, 112 MiB of query and key gradients take 105 us with plain stores and 110 streamed, 140 129 and 132,
            // 192 224 and 210; alone, with nothing to read them, 77 and 69, 92 and 83, 138 and 124)
            if (streams_out(a.M * (a.Hq + a.Hkv) * (int64_t)a.D * 2, a.D, 64)) of(std::true_type{});
            else of(std::false_type{});
        };
        if (G == 8) launch(std::integral_constant<int, 8>{});
        else if (G == 16) launch(std::integral_constant<int, 16>{});
        else if (G == 32) launch(std::integral_constant<int, 32>{});
        else launch(std::integral_constant<int, 64>{});
    }
    if (a.dw_partial || a.amax_partial) {
        const int cols = a.dw_partial ? (2 * a.D + kFinalCols - 1) / kFinalCols : 0;
        hipLaunchKernelGGL(qk_bwd_final_kernel, dim3(cols + 1), dim3(kFinalThreads), 0, stream, a.dw_partial, a.amax_partial, blocks, a.D, f.dwq, f.dwk, f.accumulate, fp8_max(f.fmt), f.d_amax, f.d_scale);
    }
    return hipGetLastError() == hipSuccess ? LLMQ_OK : LLMQ_ERR_DEVICE;
}

}  // namespace llmq

namespace {

constexpr int64_t kMaxHeads = 1 << 16, kMaxHead = llmq::kQkAnyWidth;

int check_qk(int64_t M, int64_t Hq, int64_t Hkv, int64_t D, int rot, int interleaved) {
    if (!dim_ok(M) || Hq < 1 || Hq > kMaxHeads || Hkv < 1 || Hkv > kMaxHeads || D < 1 || D > kMaxHead || M * (Hq + 2 * Hkv) * D >= kMaxElems) return LLMQ_ERR_SHAPE;
    if (rot < 0 || rot > D || rot % 2 != 0) return LLMQ_ERR_SHAPE;
    if (interleaved != 0 && interleaved != 1) return LLMQ_ERR_FLAGS;
    return LLMQ_OK;
}
// Rows of `width` elements, `stride` apart
bool stride_ok(int64_t M, int64_t width, int64_t stride) { return (M == 1 || stride >= width) && stride >= 0 && stride < kMaxDim && M * stride < kMaxElems; }

size_t qk_workspace(int64_t D) { return round256((size_t)llmq::kQkMaxBlocks * 2 * (size_t)D * sizeof(float)) + (size_t)llmq::kQkMaxBlocks * sizeof(unsigned); }

}  // namespace

extern "C" {

int llmq_qk_norm_rope_fwd(const void* qkv_bf16, int64_t qkv_stride, int64_t M, int Hq, int Hkv, int D, const void* wq_bf16, const void* wk_bf16, float eps,
                          const int64_t* d_positions, const double* d_inv_freq, int rot, int interleaved, void* q_bf16, int64_t q_stride, void* k_bf16,
                          int64_t k_stride, float* rstd, void* stream) {
    if (!qkv_bf16 || !q_bf16 || !k_bf16 || !wq_bf16 != !wk_bf16 || (rot > 0 && (!d_positions || !d_inv_freq))) return LLMQ_ERR_NULL;
    const int st = check_qk(M, Hq, Hkv, D, rot, interleaved);
    if (st != LLMQ_OK) return st;
    if (!stride_ok(M, (int64_t)(Hq + 2 * Hkv) * D, qkv_stride) || !stride_ok(M, (int64_t)Hq * D, q_stride) || !stride_ok(M, (int64_t)Hkv * D, k_stride)) return LLMQ_ERR_SHAPE;
    if (wq_bf16 && !(eps >= 0.0f && eps <= 3.402823466e+38f)) return LLMQ_ERR_VALUE;
    if (!aligned(qkv_bf16, 2) || !aligned(q_bf16, 2) || !aligned(k_bf16, 2) || !aligned(wq_bf16, 2) || !aligned(wk_bf16, 2) || !aligned(d_positions, 8) ||
        !aligned(d_inv_freq, 8) || !aligned(rstd, 4))
        return LLMQ_ERR_ALIGN;
    typedef llmq::u16 u16;
    llmq::QkArgs a{};
    a.M = M, a.Hq = Hq, a.Hkv = Hkv, a.D = D, a.rot = rot, a.interleaved = interleaved;
    a.x = static_cast<const u16*>(qkv_bf16), a.x_stride = qkv_stride;
    a.wq = static_cast<const u16*>(wq_bf16), a.wk = static_cast<const u16*>(wk_bf16), a.eps = eps;
    a.positions = d_positions, a.inv_freq = d_inv_freq, a.rstd = rstd;
    a.q = static_cast<u16*>(q_bf16), a.q_stride = q_stride, a.k = static_cast<u16*>(k_bf16), a.k_stride = k_stride;
    return llmq::launch_qk_fwd(a, static_cast<hipStream_t>(stream), num_cus());
}

size_t llmq_qk_norm_rope_workspace_bytes(int64_t M, int Hq, int Hkv, int D) {
    return check_qk(M, Hq, Hkv, D, 0, 0) == LLMQ_OK ? qk_workspace(D) : 0;
}

int llmq_qk_norm_rope_bwd(const void* dq_bf16, int64_t dq_stride, const void* dk_bf16, int64_t dk_stride, const void* dv_bf16, int64_t dv_stride,
                          const void* qkv_bf16, int64_t qkv_stride, int64_t M, int Hq, int Hkv, int D, const void* wq_bf16, const void* wk_bf16,
                          const float* rstd, const int64_t* d_positions, const double* d_inv_freq, int rot, int interleaved, void* dqkv_bf16,
                          int64_t dqkv_stride, float* dwq, float* dwk, int accumulate, int fmt, float* d_amax, float* d_scale, void* ws, size_t ws_bytes,
                          void* stream) {
    if (!dq_bf16 || !dk_bf16 || !dqkv_bf16 || !wq_bf16 != !wk_bf16 || (rot > 0 && (!d_positions || !d_inv_freq)) || (d_scale && !d_amax)) return LLMQ_ERR_NULL;
    const bool norm = wq_bf16 != nullptr, sums = dwq || dwk;
    if (norm ? !qkv_bf16 || !rstd : sums) return LLMQ_ERR_NULL;
    if ((sums || d_amax) && !ws) return LLMQ_ERR_NULL;
    const int st = check_qk(M, Hq, Hkv, D, rot, interleaved);
    if (st != LLMQ_OK) return st;
    if (!stride_ok(M, (int64_t)(Hq + 2 * Hkv) * D, dqkv_stride) || !stride_ok(M, (int64_t)Hq * D, dq_stride) || !stride_ok(M, (int64_t)Hkv * D, dk_stride) ||
        (dv_bf16 && !stride_ok(M, (int64_t)Hkv * D, dv_stride)) || (norm && !stride_ok(M, (int64_t)(Hq + 2 * Hkv) * D, qkv_stride)))
        return LLMQ_ERR_SHAPE;
    if (d_amax && !fmt_ok(fmt)) return LLMQ_ERR_FORMAT;
    if (!aligned(dq_bf16, 2) || !aligned(dk_bf16, 2) || !aligned(dv_bf16, 2) || !aligned(qkv_bf16, 2) || !aligned(wq_bf16, 2) || !aligned(wk_bf16, 2) || !aligned(rstd, 4) ||
        !aligned(d_positions, 8) || !aligned(d_inv_freq, 8) || !aligned(dqkv_bf16, 2) || !aligned(dwq, 4) || !aligned(dwk, 4) || !aligned(d_amax, 4) || !aligned(d_scale, 4) || !aligned(ws, 16))
        return LLMQ_ERR_ALIGN;
    if ((sums || d_amax) && ws_bytes < qk_workspace(D)) return LLMQ_ERR_WORKSPACE;
    // (two workgroups would write the same sums)
    if (dwq && dwk && dwq < dwk + D && dwk < dwq + D) return LLMQ_ERR_VALUE;
    typedef llmq::u16 u16;
    llmq::QkArgs a{};
    a.M = M, a.Hq = Hq, a.Hkv = Hkv, a.D = D, a.rot = rot, a.interleaved = interleaved;
    a.x = static_cast<const u16*>(qkv_bf16), a.x_stride = qkv_stride;
    a.wq = static_cast<const u16*>(wq_bf16), a.wk = static_cast<const u16*>(wk_bf16);
    a.positions = d_positions, a.inv_freq = d_inv_freq, a.rstd = const_cast<float*>(rstd);
    a.q = static_cast<u16*>(const_cast<void*>(dq_bf16)), a.q_stride = dq_stride, a.k = static_cast<u16*>(const_cast<void*>(dk_bf16)), a.k_stride = dk_stride;
    a.dv = static_cast<const u16*>(dv_bf16), a.dv_stride = dv_stride;
    a.dx = static_cast<u16*>(dqkv_bf16), a.dx_stride = dqkv_stride;
    a.dw_partial = sums ? static_cast<float*>(ws) : nullptr;
    a.amax_partial = d_amax ? reinterpret_cast<unsigned*>(static_cast<uint8_t*>(ws) + round256((size_t)llmq::kQkMaxBlocks * 2 * (size_t)D * sizeof(float))) : nullptr;
    return llmq::launch_qk_bwd(a, llmq::QkFinal{dwq, dwk, accumulate != 0, d_amax ? fmt : 0, d_amax, d_scale}, static_cast<hipStream_t>(stream), num_cus());
}

}  // extern "C"
