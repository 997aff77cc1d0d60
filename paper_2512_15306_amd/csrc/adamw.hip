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
// get for b2 up to 31/32, the second above: it would be right everywhere, but a step of the 233 million elements below takes 667 us with it and 622 with the first (back to back), more
// than 4 % of v, 2 % of a weight's step, are worth.
// Below 2^-6 (2^-15 of the block's largest value) the codes are as far apart as at 2^-6 and are rounded up or down too: to the nearest, 4 would stay 4 under b1 = 0.9, and a weight whose
// gradient has stopped would go on by a share of lr a step without end (79 lr in 1000 steps on average, where it is 2.2 rounded so and in exact moments).  There roots keep their square's mean for any b2: by their own,
// v would come out 10 to 70 % too large (roots of 1 to 4 times the smallest code).  Only a root above zero is kept above zero: a moment that came up beside a root that went to zero would make a step
// without bound.
// Weights in BF16 without a master copy can be rounded the same way, for the same reason.
//
// 233 million elements in 8 tensors, moments in 8 bits and a master copy (3.74 GB): 634 us, 5.9 TB/s; 12.5 million in 96 tensors of 128 to 520662 elements, moments in binary32
// (351 MB): 59 us, 6.0 TB/s: a large copy has 5.85.  With an absmax word for every tensor 30 us more for the first, 44 for the second (back to back): each workgroup finds the largest of its piece and looks at the word.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

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
// A lane has four elements, a wave 256 that follow each other, so that every load and store of a wave is one piece of memory.  A workgroup's piece of a tensor is no more than that
// for its four waves: many short workgroups keep more loads on their way than fewer that go through several such groups, also with the next group's loads ahead of the step for
// the last.  Pieces of 1024 / 4096, microseconds: 255816 elements 4.9 / 9.8, 1.6 million 8.8 / 11.9, 12.5 million in binary32 59.6 / 68.7, 233 million in 8 bits 652 / 676 (before codes_of left small
// codes to the waves that hold some).
constexpr int kAdamThreads = 256, kAdamLane = 4, kAdamPiece = kAdamThreads * kAdamLane;

// 32 well mixed bits for a counter under a key.  The multipliers are odd numbers from the golden ratio and the square roots of 2 and 3.
__host__ __device__ inline unsigned mixed_bits(uint64_t counter, unsigned key) {
    unsigned x = (unsigned)counter * 0x9E3779B1u + key + (unsigned)(counter >> 32) * 0xBB67AE85u;
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

// 2^(code - 127); NaN for 255
__device__ inline float power_of(unsigned code) { return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7FC00000u : code << 23); }

// Largest of 32 lanes (a block of 128 values, four a lane), in all of them
__device__ inline unsigned max_of_32(unsigned v) {
    auto with = [&](unsigned t) { v = v > t ? v : t; };
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false));
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false));
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false));
    with((unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false));
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return r[0] > r[1] ? r[0] : r[1];
}

// E4M3 code of a magnitude below 2^-6, brought to 2^8 times that: the last bits of a + 4 are whole steps of 2^-9 and 20 bits behind them, by which it is rounded up or down.  ROOT: so that the
// mean of the code's square is kept.
template <bool ROOT>
__device__ inline unsigned small_code(float a, unsigned rnd) {
    const unsigned at = __float_as_uint(a + 4.0f) - 0x40800000u;
    if constexpr (!ROOT) return (at + (rnd << 4)) >> 20;
    const float f = (float)(at & 0xFFFFFu) * 0x1p-20f, n2 = (float)(2u * (at >> 20));
    const unsigned code = (at >> 20) + (((float)rnd + 0.5f) * (n2 + 1.0f) < f * (n2 + f) * 65536.0f ? 1u : 0u);
    return code == 0 && a > 0.0f ? 1u : code;
}
// E4M3 codes (their low 7 bits) of the magnitudes of x with |x| 2^(127 - scale) <= 448, by 16 random bits each.  They are brought to 2^8 times that: the low byte of the exponent
// and the first three bits of the mantissa is then the code of a normal value, with 20 bits behind it.  Few waves hold values below 2^-6 (one in 40 where the gradients of a block are alike), and the others do not
// pay for them: the step is near what the vector units do while it waits for memory (233 million elements 622 us, 725 with both computed for every value).
// SQUARE: the mean of the codes' squares is kept instead of their own.
template <bool ROOT, bool SQUARE>
__device__ inline void codes_of(const v4f& x, int scale, const unsigned (&rnd)[4], unsigned (&codes)[4]) {
    float a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = __builtin_amdgcn_ldexpf(__builtin_fabsf(x[i]), 135 - scale);
        const unsigned bits = __float_as_uint(a[i]);
        if constexpr (SQUARE) {
            const float f = (float)(bits & 0xFFFFFu) * 0x1p-20f, n2 = (float)(16u + 2u * ((bits >> 20) & 7u));
            codes[i] = (bits >> 20) + (((float)rnd[i] + 0.5f) * (n2 + 1.0f) < f * (n2 + f) * 65536.0f ? 1u : 0u);
        } else {
            codes[i] = (bits + (rnd[i] << 4)) >> 20;
        }
    }
    const float least = __builtin_fminf(__builtin_fminf(a[0], a[1]), __builtin_fminf(a[2], a[3]));
    if (__builtin_amdgcn_ballot_w64(least < 4.0f)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (a[i] < 4.0f) codes[i] = small_code<ROOT>(a[i], rnd[i]);
    }
}
__device__ inline unsigned pack_bytes(unsigned a, unsigned b, unsigned c, unsigned d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}

// What a tensor holds, fixed for its workgroups: moments in codes; gradients in binary32; a master copy (or binary32 weights); BF16 weights.  GUARD: the piece reaches over the
// tensor's end.
template <bool CODES_, bool G32_, bool MASTER_, bool HALF_, bool GUARD_>
struct Kind { static constexpr bool CODES = CODES_, G32 = G32_, MASTER = MASTER_, HALF = HALF_, GUARD = GUARD_; };

// Four elements at p, of which `valid` exist; zeros behind them
template <bool GUARD, class V, class T>
__device__ inline V load4(const T* p, int valid) {
    static_assert(sizeof(V) == 4 * sizeof(T), "");
    if constexpr (!GUARD) {
        return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    } else {
        T e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = i < valid ? p[i] : T(0);
        return __builtin_bit_cast(V, e);
    }
}
template <bool GUARD, class V, class T>
__device__ inline void store4(T* p, int valid, const V& v) {
    static_assert(sizeof(V) == 4 * sizeof(T), "");
    if constexpr (!GUARD) {
        __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
    } else {
        T e[4];
        __builtin_memcpy(e, &v, sizeof(v));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < valid) p[i] = e[i];
    }
}

// A lane's four elements as they lie in memory
template <class K>
struct Group {
    std::conditional_t<K::G32, v4f, v2u> g;
    std::conditional_t<K::MASTER, v4f, v2u> w;
    std::conditional_t<K::CODES, unsigned, v4f> m, v;
    unsigned ms, vs;
};
__device__ inline v4f bf16_values(const v2u& b) {
    return v4f{__uint_as_float(b[0] << 16), __uint_as_float(b[0] & 0xFFFF0000u), __uint_as_float(b[1] << 16), __uint_as_float(b[1] & 0xFFFF0000u)};
}
template <class K>
__device__ inline int valid_of(const AdamWTensor& t, int64_t at) {
    const int64_t left = t.n - at;
    return !K::GUARD || left >= 4 ? 4 : left > 0 ? (int)left : 0;
}
template <class K>
__device__ inline void request(const AdamWTensor& t, int64_t at, Group<K>& r) {
    const int valid = valid_of<K>(t, at);
    if constexpr (K::G32) r.g = load4<K::GUARD, v4f>(static_cast<const float*>(t.g) + at, valid);
    else r.g = load4<K::GUARD, v2u>(static_cast<const uint16_t*>(t.g) + at, valid);
    if constexpr (K::MASTER) r.w = load4<K::GUARD, v4f>(t.master + at, valid);
    else r.w = load4<K::GUARD, v2u>(t.w + at, valid);
    if constexpr (K::CODES) {
        r.m = load4<K::GUARD, unsigned>(static_cast<const uint8_t*>(t.m) + at, valid);
        r.v = load4<K::GUARD, unsigned>(static_cast<const uint8_t*>(t.v) + at, valid);
        r.ms = valid ? t.m_scale[at / kBlock] : 127u;
        r.vs = valid ? t.v_scale[at / kBlock] : 127u;
    } else {
        r.m = load4<K::GUARD, v4f>(static_cast<const float*>(t.m) + at, valid);
        r.v = load4<K::GUARD, v4f>(static_cast<const float*>(t.v) + at, valid);
    }
}
__device__ inline v4f decoded(unsigned codes) {
    return v4f{__builtin_amdgcn_cvt_f32_fp8((int)codes, 0), __builtin_amdgcn_cvt_f32_fp8((int)codes, 1), __builtin_amdgcn_cvt_f32_fp8((int)codes, 2), __builtin_amdgcn_cvt_f32_fp8((int)codes, 3)};
}

// The step for a lane's four elements; returns the largest magnitude of its new BF16 weights.  Every operation is rounded by itself (no fused multiply-add), so that
// the values, and the codes with them, are the same wherever the formulas are evaluated in binary32.
template <class K>
__device__ inline unsigned step_of(const AdamWTensor& t, const AdamWHyper& h, float grad_scale, int64_t at, const Group<K>& r) {
#pragma clang fp contract(off)
    const int valid = valid_of<K>(t, at);
    v4f g, w, m, v, root;
    if constexpr (K::G32) g = r.g; else g = bf16_values(r.g);
    if constexpr (K::MASTER) w = r.w; else w = bf16_values(r.w);
    if constexpr (K::CODES) {
        const float ms = power_of(r.ms), vs = power_of(r.vs);
        m = decoded(r.m);
        v = decoded(r.v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m[i] * ms;
            v[i] = v[i] * vs;
            v[i] = v[i] * v[i];
        }
    } else {
        m = r.m;
        v = r.v;
    }
    const float lr_decay = t.flags & LLMQ_ADAMW_NO_DECAY ? 0.0f : h.lr_decay;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] = g[i] * grad_scale;
        m[i] = m[i] * h.b1 + g[i] * h.c1;
        v[i] = v[i] * h.b2 + (g[i] * g[i]) * h.c2;
        root[i] = __builtin_sqrtf(v[i]);
        const float decayed = w[i] - w[i] * lr_decay;
        w[i] = decayed - (m[i] / (root[i] * h.root_scale + h.eps)) * h.lr_m;
    }
    const uint64_t counter = (uint64_t)(t.counter + at);
    if constexpr (K::CODES) {
        unsigned m_mag = 0, v_mag = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned a = __float_as_uint(m[i]) & 0x7FFFFFFFu, b = __float_as_uint(root[i]) & 0x7FFFFFFFu;
            m_mag = m_mag > a ? m_mag : a;
            v_mag = v_mag > b ? v_mag : b;
        }
        const unsigned ms = scale_code<0>(max_of_32(m_mag)), vs = scale_code<0>(max_of_32(v_mag));
        auto codes = [&](auto square) __attribute__((always_inline)) {
            unsigned mc[4], vc[4], m_rnd[4], v_rnd[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned rnd = mixed_bits(counter + i, h.key);
                m_rnd[i] = rnd & 0xFFFFu, v_rnd[i] = rnd >> 16;
            }
            codes_of<false, false>(m, (int)ms, m_rnd, mc);
            codes_of<true, decltype(square)::value>(root, (int)vs, v_rnd, vc);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                mc[i] = (mc[i] & 0x7Fu) | (__float_as_uint(m[i]) >> 24 & 0x80u);
                vc[i] &= 0x7Fu;
            }
            store4<K::GUARD>(static_cast<uint8_t*>(t.m) + at, valid, pack_bytes(mc[0], mc[1], mc[2], mc[3]));
            store4<K::GUARD>(static_cast<uint8_t*>(t.v) + at, valid, pack_bytes(vc[0], vc[1], vc[2], vc[3]));
        };
        if (h.b2 > kRootMeanBeta) codes(std::true_type{});
        else codes(std::false_type{});
        if (valid && at % kBlock == 0) {
            t.m_scale[at / kBlock] = (uint8_t)ms;
            t.v_scale[at / kBlock] = (uint8_t)vs;
        }
    } else {
        store4<K::GUARD>(static_cast<float*>(t.m) + at, valid, m);
        store4<K::GUARD>(static_cast<float*>(t.v) + at, valid, v);
    }
    if constexpr (K::MASTER) store4<K::GUARD>(t.master + at, valid, w);
    unsigned mag = 0;
    if constexpr (K::HALF) {
        unsigned half[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            half[i] = __builtin_bit_cast(uint16_t, (__bf16)w[i]);
            if constexpr (!K::MASTER) {
                const unsigned bits = __float_as_uint(w[i]);
                if ((t.flags & LLMQ_ADAMW_STOCHASTIC) && (bits & 0x7F800000u) != 0x7F800000u) half[i] = (bits + (mixed_bits(counter + i, ~h.key) & 0xFFFFu)) >> 16;
            }
        }
        const v2u packed = {half[0] | half[1] << 16, half[2] | half[3] << 16};
        store4<K::GUARD>(t.w + at, valid, packed);
        if (t.amax) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < valid) mag = mag > (half[i] & 0x7FFFu) ? mag : half[i] & 0x7FFFu;
        }
    }
    return mag;
}

template <class K>
__device__ inline unsigned step_of_piece(const AdamWTensor& t, const AdamWHyper& h, float grad_scale, int64_t at) {
    Group<K> r;
    request(t, at, r);
    return step_of(t, h, grad_scale, at, r);
}

__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamWTensor* tensors, const AdamWPiece* pieces, unsigned first, const AdamWHyper by_value, const AdamWHyper* d_hyper,
                                                             const float* d_grad_scale) {
    __shared__ unsigned s_part[kAdamThreads / kWave];
    const float grad_scale = d_grad_scale ? *d_grad_scale : 1.0f;
    if (!__builtin_isfinite(grad_scale)) return;             // the step is skipped
    const AdamWHyper h = d_hyper ? *d_hyper : by_value;
    const AdamWPiece p = pieces[blockIdx.x + first];
    const AdamWTensor t = tensors[p.tensor];
    const int64_t at = (int64_t)p.piece * kAdamPiece + threadIdx.x * kAdamLane;
    unsigned mag = 0;
    auto with = [&](auto codes, auto g32, auto master, auto half) __attribute__((always_inline)) {
        constexpr bool C = decltype(codes)::value, G = decltype(g32)::value, M = decltype(master)::value, H = decltype(half)::value;
        if (t.n - (int64_t)p.piece * kAdamPiece >= kAdamPiece) mag = step_of_piece<Kind<C, G, M, H, false>>(t, h, grad_scale, at);
        else mag = step_of_piece<Kind<C, G, M, H, true>>(t, h, grad_scale, at);
    };
    auto with_weights = [&](auto codes, auto g32) __attribute__((always_inline)) {
        if (t.master && t.w) with(codes, g32, std::true_type{}, std::true_type{});
        else if (t.master) with(codes, g32, std::true_type{}, std::false_type{});
        else with(codes, g32, std::false_type{}, std::true_type{});
    };
    const bool g32 = t.flags & LLMQ_ADAMW_GRAD_F32;
    if (t.flags & LLMQ_ADAMW_STATES_8BIT) g32 ? with_weights(std::true_type{}, std::true_type{}) : with_weights(std::true_type{}, std::false_type{});
    else g32 ? with_weights(std::false_type{}, std::true_type{}) : with_weights(std::false_type{}, std::false_type{});
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

// Whether an array that a step writes shares memory with another one of the plan: its workgroups run in any order.  (Gradients are only read, and may be shared.  Absmax words are left to the caller.)
int check_apart(const llmq_adamw_tensor* t, int64_t count) {
    struct Range { uintptr_t first, end; bool written; };
    Range* const r = new (std::nothrow) Range[(size_t)count * 7];
    if (!r) return LLMQ_ERR_WORKSPACE;
    Range* last = r;
    auto add = [&](const void* p, int64_t bytes, bool written) {
        if (p) *last++ = Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes, written};
    };
    for (int64_t i = 0; i < count; ++i) {
        const llmq_adamw_tensor& x = t[i];
        const bool codes = (x.flags & LLMQ_ADAMW_STATES_8BIT) != 0;
        const int64_t moment = codes ? x.n : 4 * x.n, scales = (x.n + 127) / 128;
        add(x.w_bf16, 2 * x.n, true);
        add(x.w_f32, 4 * x.n, true);
        add(x.grad, x.flags & LLMQ_ADAMW_GRAD_F32 ? 4 * x.n : 2 * x.n, false);
        add(x.m, moment, true);
        add(x.v, moment, true);
        add(codes ? x.m_scale : nullptr, scales, true);
        add(codes ? x.v_scale : nullptr, scales, true);
    }
    std::sort(r, last, [](const Range& a, const Range& b) { return a.first < b.first; });
    uintptr_t end = 0, written_end = 0;                      // of all ranges so far, of the written ones
    int st = LLMQ_OK;
    for (const Range* p = r; p < last; ++p) {
        if (p->first < (p->written ? end : written_end)) st = LLMQ_ERR_VALUE;
        end = std::max(end, p->end);
        if (p->written) written_end = std::max(written_end, p->end);
    }
    delete[] r;
    return st;
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
    int st = check_adamw(tensors, count, pieces);
    if (st == LLMQ_OK) st = check_apart(tensors, count);
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
    if (!isfinite(h.lr_decay) || !isfinite(h.lr_m) || !isfinite(h.root_scale) || !isfinite(h.eps)) return LLMQ_ERR_VALUE;
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
