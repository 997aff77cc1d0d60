// One AdamW step over many tensors in one launch, moments in binary32 or in 8 bits with a power-of-two scale for each block of 128.
//
//   g' = g s;  m' = m b1 + g' (1 - b1);  v' = v b2 + g'^2 (1 - b2)
//   w' = (w - w lr decay) - (m' / (sqrt(v') / sqrt(1 - b2^t) + eps)) (lr / (1 - b1^t))
//
// HBM-bound: with a master copy 28 bytes per element and 16 with moments in 8 bits, each read or written once.  A model's tensors range from a norm's weights to
// hundreds of millions of values; a table in device memory says for every workgroup which piece of which tensor is its own, so the launch is one
// and its workgroups are alike.
//
// 8-bit moments: m, and the root of v, in E4M3 codes.  The root halves the exponents v would need.  With b2 near one a step changes v by less than half a step of
// its code, and rounded to the nearest it would never move; so codes are rounded up or down with the probability that keeps their mean, by
// 16 random bits from a hash of element and step: the same bits on every run.  For the root there are two means to keep.  Its own: then its square comes out larger by the
// variance, 0.13 % a step on average over the codes (a sixth of the square of the spacing, 1/8 to 1/16), which the average over 1 / (1 - b2) steps multiplies: 2.5 % of v
// for b2 = 0.95, and without bound from 0.9987 on.  Its square's, by the probability f (2 n + f) / (2 n + 1) for n + f units: v is right for any b2.  The first is what roots
// get for b2 up to 31/32, the second above.  Below 2^-6 (2^-15 of the block's largest value) codes are rounded to the nearest,
// and a root above zero is kept above zero: a moment that came up beside a root that went to zero would make a step without bound.
// Weights in BF16 without a master copy can be rounded the same way, for the same reason.
#include <math.h>
#include <string.h>

#include "api_checks.h"
#include "blocks.h"

namespace llmq {

struct AdamWTensor {
    uint16_t* w;
    float* master;
    const void* g;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    unsigned* amax;
    int64_t n, counter;
    int flags, pad;
};
struct AdamWPiece { int tensor, piece; };
struct AdamWHyper { float b1, b2, c1, c2, lr_decay, lr_m, root_scale, eps; unsigned key, pad; };
static_assert(sizeof(AdamWHyper) == 4 * LLMQ_ADAMW_HYPER_WORDS, "");

constexpr float kRootMeanBeta = 0.96875f;
constexpr int kAdamThreads = 256, kAdamLane = 8, kAdamTrips = 2, kAdamPiece = kAdamThreads * kAdamLane * kAdamTrips;

// 32 well mixed bits for a counter under a key.  The multipliers are odd numbers from the golden ratio and the square roots of 2 and 3.
__host__ __device__ inline unsigned mixed_bits(uint64_t counter, unsigned key) {
    unsigned x = (unsigned)counter * 0x9E3779B1u + key + (unsigned)(counter >> 32) * 0xBB67AE85u;
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

// 2^(code - 127); NaN for 255
__device__ inline float power_of(unsigned code) { return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7FC00000u : code << 23); }

// Largest of 16 lanes (a block of 128 values, eight a lane), in all of them
__device__ inline unsigned max_of_16(unsigned v) {
    auto with = [&](unsigned t) { v = v > t ? v : t; };
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));
    return v;
}

// E4M3 code of a magnitude of at most 448, by 16 random bits; square: the mean of the code's square is kept instead of its own
__device__ inline unsigned code_of(float a, unsigned rnd, bool square) {
    const unsigned bits = __float_as_uint(a);
    unsigned normal = ((bits + (rnd << 4)) >> 20) - 960u;
    if (square) {
        const float f = (float)(bits & 0xFFFFFu) * 0x1p-20f, n2 = (float)(16u + 2u * ((bits >> 20) & 7u));
        normal = (bits >> 20) - 960u + (((float)rnd + 0.5f) * (n2 + 1.0f) < f * (n2 + f) * 65536.0f ? 1u : 0u);
    }
    const unsigned small = (unsigned)(int)__builtin_rintf(a * 512.0f);
    const unsigned c = a >= 0.015625f ? normal : small;
    return c < 127u ? c : 127u;                              // (a NaN's)
}

// Eight values of a lane, of which `valid` exist; zeros behind them
template <class T>
__device__ inline void load8(const T* p, int valid, T (&v)[8]) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T) < 8 ? 16 / sizeof(T) : 8)));
    constexpr int kVec = sizeof(vec) / sizeof(T);
    if (valid >= 8) {
#pragma unroll
        for (int i = 0; i < 8; i += kVec) {
            const vec x = __builtin_nontemporal_load(reinterpret_cast<const vec*>(p + i));
#pragma unroll
            for (int j = 0; j < kVec; ++j) v[i + j] = x[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? p[i] : T(0);
    }
}
template <class T>
__device__ inline void store8(T* p, int valid, const T (&v)[8]) {
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T) < 8 ? 16 / sizeof(T) : 8)));
    constexpr int kVec = sizeof(vec) / sizeof(T);
    if (valid >= 8) {
#pragma unroll
        for (int i = 0; i < 8; i += kVec) {
            vec x;
#pragma unroll
            for (int j = 0; j < kVec; ++j) x[j] = v[i + j];
            __builtin_nontemporal_store(x, reinterpret_cast<vec*>(p + i));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = v[i];
    }
}
__device__ inline void bf16_values(const uint16_t (&b)[8], float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float((unsigned)b[i] << 16);
}

// The step for eight elements of a lane.  Every operation is rounded by itself (no fused multiply-add), so that the values, and the codes with them, are
// the same wherever the formulas are evaluated in binary32.
template <bool CODES>
__device__ inline unsigned adamw_eight(const AdamWTensor& t, const AdamWHyper& h, float grad_scale, int64_t at) {
#pragma clang fp contract(off)
    const int64_t left = t.n - at;
    const int valid = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    float g[8], w[8], m[8], v[8];
    uint16_t half[8];
    if (t.flags & LLMQ_ADAMW_GRAD_F32) {
        load8(static_cast<const float*>(t.g) + at, valid, g);
    } else {
        load8(static_cast<const uint16_t*>(t.g) + at, valid, half);
        bf16_values(half, g);
    }
    if (t.master) {
        load8(t.master + at, valid, w);
    } else {
        load8(t.w + at, valid, half);
        bf16_values(half, w);
    }
    if constexpr (CODES) {
        uint8_t mc[8], vc[8];
        load8(static_cast<const uint8_t*>(t.m) + at, valid, mc);
        load8(static_cast<const uint8_t*>(t.v) + at, valid, vc);
        const float ms = valid ? power_of(t.m_scale[at / kBlock]) : 1.0f, vs = valid ? power_of(t.v_scale[at / kBlock]) : 1.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = __builtin_amdgcn_cvt_f32_fp8(mc[i], 0) * ms;
            v[i] = __builtin_amdgcn_cvt_f32_fp8(vc[i], 0) * vs;
            v[i] = v[i] * v[i];
        }
    } else {
        load8(static_cast<const float*>(t.m) + at, valid, m);
        load8(static_cast<const float*>(t.v) + at, valid, v);
    }
    const float lr_decay = t.flags & LLMQ_ADAMW_NO_DECAY ? 0.0f : h.lr_decay;
    float root[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        g[i] = g[i] * grad_scale;
        m[i] = m[i] * h.b1 + g[i] * h.c1;
        v[i] = v[i] * h.b2 + (g[i] * g[i]) * h.c2;
        root[i] = __builtin_sqrtf(v[i]);
        const float decayed = w[i] - w[i] * lr_decay;
        w[i] = decayed - (m[i] / (root[i] * h.root_scale + h.eps)) * h.lr_m;
    }
    const uint64_t counter = (uint64_t)(t.counter + at);
    if constexpr (CODES) {
        unsigned m_mag = 0, v_mag = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned a = __float_as_uint(m[i]) & 0x7FFFFFFFu, b = __float_as_uint(root[i]) & 0x7FFFFFFFu;
            m_mag = m_mag > a ? m_mag : a;
            v_mag = v_mag > b ? v_mag : b;
        }
        const unsigned ms = scale_code<0>(max_of_16(m_mag)), vs = scale_code<0>(max_of_16(v_mag));
        const float m_up = power_of(254u - ms), v_up = power_of(254u - vs);
        uint8_t mc[8], vc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned rnd = mixed_bits(counter + i, h.key);
            mc[i] = (uint8_t)(code_of(__builtin_fabsf(m[i]) * m_up, rnd & 0xFFFFu, false) | (m[i] < 0.0f ? 0x80u : 0u));
            const unsigned c = code_of(root[i] * v_up, rnd >> 16, h.b2 > kRootMeanBeta);
            vc[i] = (uint8_t)(c == 0 && root[i] > 0.0f ? 1u : c);
        }
        store8(static_cast<uint8_t*>(t.m) + at, valid, mc);
        store8(static_cast<uint8_t*>(t.v) + at, valid, vc);
        if (valid && at % kBlock == 0) {
            t.m_scale[at / kBlock] = (uint8_t)ms;
            t.v_scale[at / kBlock] = (uint8_t)vs;
        }
    } else {
        store8(static_cast<float*>(t.m) + at, valid, m);
        store8(static_cast<float*>(t.v) + at, valid, v);
    }
    if (t.master) store8(t.master + at, valid, w);
    unsigned mag = 0;
    if (t.w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            half[i] = __builtin_bit_cast(uint16_t, (__bf16)w[i]);
            if (!t.master && (t.flags & LLMQ_ADAMW_STOCHASTIC)) {
                const unsigned bits = __float_as_uint(w[i]);
                if ((bits & 0x7F800000u) != 0x7F800000u) half[i] = (uint16_t)((bits + (mixed_bits(counter + i, ~h.key) & 0xFFFFu)) >> 16);
            }
            const unsigned a = half[i] & 0x7FFFu;
            if (i < valid) mag = mag > a ? mag : a;
        }
        store8(t.w + at, valid, half);
    }
    return mag;
}

__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamWTensor* tensors, const AdamWPiece* pieces, unsigned first, const AdamWHyper by_value, const AdamWHyper* d_hyper,
                                                             const float* d_grad_scale) {
    __shared__ unsigned s_part[kAdamThreads / kWave];
    const float grad_scale = d_grad_scale ? *d_grad_scale : 1.0f;
    if (!__builtin_isfinite(grad_scale)) return;             // the step is skipped
    const AdamWHyper h = d_hyper ? *d_hyper : by_value;
    const AdamWPiece p = pieces[blockIdx.x + first];
    const AdamWTensor t = tensors[p.tensor];
    int64_t at = (int64_t)p.piece * kAdamPiece + threadIdx.x * kAdamLane;
    unsigned mag = 0;
#pragma unroll 1
    for (int k = 0; k < kAdamTrips; ++k, at += kAdamThreads * kAdamLane) {
        const unsigned a = t.flags & LLMQ_ADAMW_STATES_8BIT ? adamw_eight<true>(t, h, grad_scale, at) : adamw_eight<false>(t, h, grad_scale, at);
        mag = mag > a ? mag : a;
    }
    if (t.amax) {
        mag = block_max_u32<kAdamThreads>(mag, s_part);
        if (threadIdx.x == 0) {
            const unsigned bits = amax_bits_from_bf16_mag(mag);
            if (bits > __hip_atomic_load(t.amax, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(t.amax, bits);
        }
    }
}

__global__ void adamw_clear_kernel(const AdamWTensor* tensors, int count, const float* d_grad_scale) {
    if (d_grad_scale && !__builtin_isfinite(*d_grad_scale)) return;
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < count && tensors[i].amax) *tensors[i].amax = 0u;
}

}  // namespace llmq

namespace {

constexpr int kAdamWFlags = LLMQ_ADAMW_GRAD_F32 | LLMQ_ADAMW_STATES_8BIT | LLMQ_ADAMW_NO_DECAY | LLMQ_ADAMW_STOCHASTIC;
constexpr int64_t kMaxTensors = 1 << 24, kMaxPieces = (int64_t)1 << 31;

int check_adamw(const llmq_adamw_tensor* t, int64_t count, int64_t& pieces) {
    if (!t) return LLMQ_ERR_NULL;
    if (count < 1 || count > kMaxTensors) return LLMQ_ERR_SHAPE;
    pieces = 0;
    for (int64_t i = 0; i < count; ++i) {
        const llmq_adamw_tensor& x = t[i];
        if (x.flags & ~kAdamWFlags) return LLMQ_ERR_FLAGS;
        const bool codes = (x.flags & LLMQ_ADAMW_STATES_8BIT) != 0;
        if ((!x.w_bf16 && !x.w_f32) || !x.grad || !x.m || !x.v || (codes && (!x.m_scale || !x.v_scale)) || (x.d_amax && !x.w_bf16)) return LLMQ_ERR_NULL;
        if ((x.flags & LLMQ_ADAMW_STOCHASTIC) && x.w_f32) return LLMQ_ERR_FLAGS;            // binary32 weights are not rounded
        if (x.n < 1 || x.n >= kMaxElems || x.first_counter < 0) return LLMQ_ERR_SHAPE;
        if (!aligned(x.w_bf16, 16) || !aligned(x.w_f32, 16) || !aligned(x.grad, 16) || !aligned(x.m, 16) || !aligned(x.v, 16) || !aligned(x.d_amax, 4)) return LLMQ_ERR_ALIGN;
        pieces += (x.n + llmq::kAdamPiece - 1) / llmq::kAdamPiece;
        if (pieces >= kMaxPieces) return LLMQ_ERR_SHAPE;
    }
    return LLMQ_OK;
}

size_t adamw_table(int64_t count) { return round256((size_t)count * sizeof(llmq::AdamWTensor)); }

}  // namespace

extern "C" {

size_t llmq_adamw_plan_bytes(const llmq_adamw_tensor* tensors, int64_t count) {
    int64_t pieces = 0;
    return check_adamw(tensors, count, pieces) == LLMQ_OK ? adamw_table(count) + (size_t)pieces * sizeof(llmq::AdamWPiece) : 0;
}

int llmq_adamw_plan(const llmq_adamw_tensor* tensors, int64_t count, void* plan, size_t plan_bytes, int64_t info[4]) {
    if (!plan || !info) return LLMQ_ERR_NULL;
    int64_t pieces = 0;
    const int st = check_adamw(tensors, count, pieces);
    if (st != LLMQ_OK) return st;
    if (plan_bytes < adamw_table(count) + (size_t)pieces * sizeof(llmq::AdamWPiece)) return LLMQ_ERR_WORKSPACE;
    memset(plan, 0, adamw_table(count));
    int64_t with_amax = 0, at = 0;
    for (int64_t i = 0; i < count; ++i) {
        const llmq_adamw_tensor& x = tensors[i];
        llmq::AdamWTensor t{};
        t.w = static_cast<uint16_t*>(x.w_bf16), t.master = x.w_f32, t.g = x.grad, t.m = x.m, t.v = x.v, t.m_scale = x.m_scale, t.v_scale = x.v_scale;
        t.amax = reinterpret_cast<unsigned*>(x.d_amax), t.n = x.n, t.counter = x.first_counter, t.flags = x.flags;
        memcpy(static_cast<uint8_t*>(plan) + (size_t)i * sizeof(t), &t, sizeof(t));
        with_amax |= x.d_amax != nullptr;
        for (int64_t p = 0; p * llmq::kAdamPiece < x.n; ++p, ++at) {
            const llmq::AdamWPiece piece{(int)i, (int)p};
            memcpy(static_cast<uint8_t*>(plan) + adamw_table(count) + (size_t)at * sizeof(piece), &piece, sizeof(piece));
        }
    }
    info[0] = count, info[1] = pieces, info[2] = with_amax, info[3] = 0;
    return LLMQ_OK;
}

int llmq_adamw_hyper(int64_t step, double lr, double beta1, double beta2, double eps, double weight_decay, uint64_t seed, uint32_t hyper[LLMQ_ADAMW_HYPER_WORDS]) {
    if (!hyper) return LLMQ_ERR_NULL;
    const bool fine = step >= 1 && isfinite(lr) && lr >= 0 && beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1 && isfinite(eps) && (float)eps > 0.0f && isfinite(weight_decay) &&
                      weight_decay >= 0;
    if (!fine) return LLMQ_ERR_VALUE;
    llmq::AdamWHyper h{};
    h.b1 = (float)beta1, h.b2 = (float)beta2, h.c1 = (float)(1 - beta1), h.c2 = (float)(1 - beta2);
    h.lr_decay = (float)(lr * weight_decay), h.lr_m = (float)(lr / (1 - pow(beta1, (double)step))), h.root_scale = (float)(1 / sqrt(1 - pow(beta2, (double)step))), h.eps = (float)eps;
    h.key = llmq::mixed_bits((uint64_t)step, llmq::mixed_bits(seed, 0));
    memcpy(hyper, &h, sizeof(h));
    return LLMQ_OK;
}

int llmq_adamw_step(const void* d_plan, const int64_t info[4], const uint32_t* hyper, const void* d_hyper, const float* d_grad_scale, void* stream) {
    if (!d_plan || !info || !hyper == !d_hyper) return LLMQ_ERR_NULL;
    if (info[0] < 1 || info[0] > kMaxTensors || info[1] < 1 || info[1] >= kMaxPieces) return LLMQ_ERR_SHAPE;
    if (!aligned(d_plan, 16) || !aligned(d_hyper, 4) || !aligned(d_grad_scale, 4)) return LLMQ_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const llmq::AdamWTensor* tensors = static_cast<const llmq::AdamWTensor*>(d_plan);
    const llmq::AdamWPiece* pieces = reinterpret_cast<const llmq::AdamWPiece*>(static_cast<const uint8_t*>(d_plan) + adamw_table(info[0]));
    llmq::AdamWHyper h{};
    if (hyper) memcpy(&h, hyper, sizeof(h));
    if (info[2]) hipLaunchKernelGGL(llmq::adamw_clear_kernel, dim3((unsigned)((info[0] + 255) / 256)), dim3(256), 0, s, tensors, (int)info[0], d_grad_scale);
    const int64_t most = llmq::max_workgroups();
    for (int64_t first = 0; first < info[1]; first += most)
        hipLaunchKernelGGL(llmq::adamw_kernel, dim3((unsigned)(info[1] - first < most ? info[1] - first : most)), dim3(llmq::kAdamThreads), 0, s, tensors, pieces, (unsigned)first, h,
                           static_cast<const llmq::AdamWHyper*>(d_hyper), d_grad_scale);
    return hipGetLastError() == hipSuccess ? LLMQ_OK : LLMQ_ERR_DEVICE;
}

}  // extern "C"
