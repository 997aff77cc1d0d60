// Contractions of FP8 operands with block scales, joined with the SwiGLU behind them (llmq_fp8_gemm_blocks_swiglu_fwd) or in front of them (_bwd).
//
//   forward   g = A Wg^T, u = A Wu^T;   h = bf16( silu(g) u ),  silu(g) = g sg,  sg = 1 / (1 + e^-g);   GU = bf16(g), bf16(u) if wanted
//   backward  dh = A B^T;   dG = bf16( dh u sg (1 + g (1 - sg)) ),  dU = bf16( dh g sg ) from the kept GU;   h = bf16( g sg u ) if wanted
//
// The contraction is the tile kernel's (gemm_tile.h) and that for few rows; what is joined to it works on the sums where they are, so that GU (forward) and dh (backward) need not be
// written and read again, and dh is not rounded in between.  In the forward pass a tile's columns are pairs: half of them of gate rows, half of the up rows that belong to them, dealt out so that a lane has both sums of
// a pair.  e^-g and the reciprocal are the hardware's (v_exp_f32, v_rcp_f32: errors of 2^-23 and, from the product in front of the exponential, |g| 2^-24 of the result), which BF16 does not see and which
// take 5 instructions; every one of them is time in which the matrix cores of its CU wait.
//
// Bound by the matrix cores at the board's power cap (2.9 PFLOP/s inside the K loop) and, at the end of a tile, by what a CU can write.  8192 x 18944 x 3584: forward 950 us, 2.34 PFLOP/s (contraction and SwiGLU one
// after the other 870 + 160, and GU written and read), backward with h 622 (450 + 268).
#pragma once
#include "gemm_small.h"

namespace llmq {

struct GluPlan {
    int n_whole;                                // tiles
    const uint16_t* gu;                         // backward: the kept GU [M, 2 I]
    uint16_t *gu_out, *h_out;                   // forward: GU, backward: h; or NULL
};

// Backward, dGU may be GU: every element of GU is read, by the lane that stores its gradient, before that store, and the pointers are not declared apart, so that stores keep their place behind the loads.
template <int DIR>
using GluOut = std::conditional_t<DIR == kGluBackward, uint16_t*, uint16_t* __restrict__>;

__device__ inline float glu_sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * g)); }
__device__ inline float glu_value(float g, float u) { return g * glu_sigmoid(g) * u; }
// dG and dU, and h
__device__ inline void glu_gradient(float dh, float g, float u, float& dg, float& du, float& h) {
    const float sg = glu_sigmoid(g), s = g * sg, d = dh * sg;
    du = dh * s;
    dg = d * u * __builtin_fmaf(g, 1.0f - sg, 1.0f);
    h = s * u;
}
__device__ inline float bf16_lo(unsigned w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(unsigned w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ inline v2u bf16_of(const v4f& v) { return __builtin_bit_cast(v2u, __builtin_convertvector(v, bf16x4)); }

// A wave's part of a BF16 matrix, 32 rows of it (i) in pieces of eight columns: the lane's piece k, of SLOTS pieces in a row, is one of a row 64 / SLOTS further down for every k.  It is
// addressed by an offset of the lane through a buffer that ends with the part's last element.  EDGE kinds: pieces beside the matrix get an offset outside the buffer, and rows behind it are outside by
// themselves.  Only the lane's offset is documented to be compared with the buffer's end, so the row is part of it; where every row exists, loads have the row in the uniform offset.  Widths that are no multiples of 8: whole pieces at any address where the part lies inside the matrix (1000 x 4001 x 1040 backward 17.6 us, element by element 42.8), elsewhere element by element.
template <int EDGE, int SLOTS>
struct GluRows {
    static constexpr int kOut = 0x7FFFFF00, kRowStep = kWave / SLOTS;
    enum Mode { kPieces, kAnyAddress, kElements };
    uint16_t* base;                             // of the lane's piece 0
    __amdgpu_buffer_rsrc_t rs;
    int pitch, voff, rows_left, cols_left;      // bytes from row to row; of the lane's piece 0
    Mode mode;
    // part_rows x 8 SLOTS elements from p on, of which rows x cols exist (may be <= 0); rows are `ld` elements apart
    __device__ __attribute__((always_inline)) GluRows(const uint16_t* p, int ld, int part_rows, int rows, int cols, bool vector, int lane) {
        const int here = EDGE == kNoEdge || rows > part_rows ? part_rows : rows, r = lane / SLOTS, c = 8 * (lane % SLOTS);
        mode = EDGE == kNoEdge || vector ? kPieces : cols >= 8 * SLOTS ? kAnyAddress : kElements;
        if (EDGE == kNoEdge) cols = 8 * SLOTS;
        rs = make_rsrc(p, here > 0 && cols > 0 ? (unsigned)(((size_t)(here - 1) * ld + cols) * 2) : 0u);
        pitch = 2 * ld, rows_left = here - r, cols_left = cols - c;
        voff = EDGE == kNoEdge || c < cols ? r * pitch + 2 * c : kOut;
        base = const_cast<uint16_t*>(p) + (int64_t)r * ld + c;
    }
    __device__ bool vector() const { return EDGE == kNoEdge || mode == kPieces; }
    __device__ int row(int i, int k) const { return (32 * i + k * kRowStep) * pitch; }              // (below 2^30: kOut and a row are below 2^32)
    __device__ bool exists(int i, int k) const { return 32 * i + k * kRowStep < rows_left && cols_left > 0; }
    __device__ int piece(int i, int k) const { return (int)((unsigned)voff + (unsigned)row(i, k)); }
    __device__ int element(int i, int k, int e) const { return (int)((unsigned)(e < cols_left ? voff + 2 * e : kOut) + (unsigned)row(i, k)); }
    __device__ v4u_at2* address(int i, int k) const { return reinterpret_cast<v4u_at2*>(reinterpret_cast<uint8_t*>(base) + (int64_t)(32 * i + k * kRowStep) * pitch); }
    // STREAMED: past what the caches hold
    template <bool STREAMED = false>
    __device__ __attribute__((always_inline)) v4u load(int i, int k) const {
        if (EDGE == kNoEdge) return __builtin_amdgcn_raw_buffer_load_b128(rs, voff, row(i, k), STREAMED ? 2 : 0);
        if (vector()) return __builtin_amdgcn_raw_buffer_load_b128(rs, piece(i, k), 0, STREAMED ? 2 : 0);
        v4u v = {0, 0, 0, 0};
        if (mode == kAnyAddress) {
            if (exists(i, k)) v = *address(i, k);
            return v;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 1] |= (unsigned)(unsigned short)__builtin_amdgcn_raw_buffer_load_b16(rs, element(i, k, e), 0, 0) << (16 * (e & 1));
        return v;
    }
    // and, of the EDGE kinds, the magnitudes of what is stored
    __device__ __attribute__((always_inline)) void store(int i, int k, const v4u& v, unsigned& mag) const {
        if (vector() || mode == kAnyAddress) {
            const bool there = EDGE != kNoEdge && exists(i, k);
            // (The row in the lane's offset of whole tiles too: behind a wide buffer store the compiler keeps the next instruction off the stored registers only if the store has no scalar
            // offset.  With one, a third of the runs of 1777 x 2720 x 1024 had last words of pieces that were the next piece's.)
            if (vector()) __builtin_amdgcn_raw_buffer_store_b128(v, rs, piece(i, k), 0, 0);
            else if (there) *address(i, k) = v;
            if (there) {
#pragma unroll
                for (int e = 0; e < 4; ++e) mag = pk_max_mag(mag, v[e]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned short bits = (unsigned short)(e & 1 ? v[e >> 1] >> 16 : v[e >> 1]);
                __builtin_amdgcn_raw_buffer_store_b16(bits, rs, element(i, k, e), 0, 0);
                if (32 * i + k * kRowStep < rows_left && e < cols_left) mag = pk_max_mag(mag, (unsigned)bits);
            }
        }
    }
};

// Epilogue of the forward tile.  A lane holds, of block (i, j), four consecutive pairs of a row: their gates in columns j of the wave tile and their ups in columns MJ / 2 + j.  The wave's
// results go through its part of LDS 32 rows at a time and leave in rows (gemm_tile.h, the epilogue of the plain contraction, has the layout and its reasons).
template <int NI, int MI, int MJ, int EDGE>
struct GluForward {
    template <class Acc>
    static __device__ __attribute__((always_inline)) unsigned write_out(const Acc& acc, uint8_t* stage, uint16_t* h, const GluPlan& plan, int row0, int M, int col0, int I, int lane) {
        constexpr int HJ = MJ / 2, kSlots = 2 * HJ, kPitch = 16 * kSlots, kPlane = 32 * kPitch, kPieces = 32 * kSlots / kWave;
        static_assert(kPieces >= 1 && kWave % kSlots == 0, "every lane moves whole pieces");
        const int fr_row = lane & 15, fr_q = lane >> 4, slot0 = fr_q >> 1, half_off = (fr_q & 1) << 3;
        const bool vector = EDGE == kNoEdge || I % 8 == 0;
        typedef GluRows<EDGE, kSlots> Rows;
        const Rows out(h + (size_t)row0 * I + col0, I, 32 * NI, M - row0, I - col0, vector, lane);
        unsigned mag = 0;
        float maxabs = 0.0f;
        auto body = [&](auto keep) __attribute__((always_inline)) {
            constexpr bool KEEP = decltype(keep)::value;
            const uint16_t* gu = KEEP ? plan.gu_out + (size_t)row0 * 2 * I + col0 : h;
            const Rows gate(gu, 2 * I, 32 * NI, M - row0, I - col0, vector, lane), up(gu + (KEEP ? I : 0), 2 * I, 32 * NI, M - row0, I - col0, vector, lane);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int ii = 0; ii < 2; ++ii) {
                    const int row = 16 * ii + fr_row;
#pragma unroll
                    for (int j = 0; j < HJ; ++j) {
                        const v4f g = acc.get(2 * i + ii, j), u = acc.get(2 * i + ii, HJ + j);
                        v4f y;
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = glu_value(g[e], u[e]);
                        maxabs = __builtin_elementwise_maximum(__builtin_elementwise_maximum(maxabs, __builtin_fabsf(y[0])), __builtin_fabsf(y[1]));
                        maxabs = __builtin_elementwise_maximum(__builtin_elementwise_maximum(maxabs, __builtin_fabsf(y[2])), __builtin_fabsf(y[3]));
                        uint8_t* dst = stage + row * kPitch + ((((2 * j + slot0 + row) % kSlots) << 4) | half_off);
                        *reinterpret_cast<v2u*>(dst) = bf16_of(y);
                        if constexpr (KEEP) {
                            *reinterpret_cast<v2u*>(dst + kPlane) = bf16_of(g);
                            *reinterpret_cast<v2u*>(dst + 2 * kPlane) = bf16_of(u);
                        }
                    }
                }
                v4u piece[KEEP ? 3 : 1][kPieces];
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    const int p = lane + k * kWave, r = p / kSlots, sl = p % kSlots;
#pragma unroll
                    for (int n = 0; n < (KEEP ? 3 : 1); ++n) piece[n][k] = *reinterpret_cast<const v4u*>(stage + n * kPlane + r * kPitch + (((sl + r) % kSlots) << 4));
                }
                __builtin_amdgcn_sched_barrier(0);
                unsigned ignored = 0;
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    out.store(i, k, piece[0][k], mag);
                    if constexpr (KEEP) {
                        gate.store(i, k, piece[1][k], ignored);
                        up.store(i, k, piece[2][k], ignored);
                    }
                }
            }
        };
        if (plan.gu_out) body(BoolTag<true>{});
        else body(BoolTag<false>{});
        return EDGE == kNoEdge ? (unsigned)__builtin_bit_cast(uint16_t, (__bf16)maxabs) : mag;
    }
};

// Eight columns of a row: dG, dU and h as BF16, and the largest magnitude of the first two before rounding (rounding is monotonic, NaN stays)
__device__ inline void glu_gradient8(const v4f (&dh)[2], const v4u& g, const v4u& u, v4u& dg, v4u& du, v4u& h, float& maxabs) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        v4f a, b, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned gw = g[2 * half + e / 2], uw = u[2 * half + e / 2];
            float x, z, w;
            glu_gradient(dh[half][e], e & 1 ? bf16_hi(gw) : bf16_lo(gw), e & 1 ? bf16_hi(uw) : bf16_lo(uw), x, z, w);
            a[e] = x, b[e] = z, y[e] = w;
            maxabs = __builtin_elementwise_maximum(__builtin_elementwise_maximum(maxabs, __builtin_fabsf(x)), __builtin_fabsf(z));
        }
        const v2u wa = bf16_of(a), wb = bf16_of(b), wy = bf16_of(y);
        dg[2 * half] = wa[0], dg[2 * half + 1] = wa[1];
        du[2 * half] = wb[0], du[2 * half + 1] = wb[1];
        h[2 * half] = wy[0], h[2 * half + 1] = wy[1];
    }
}

// Epilogue of the backward tile: dh through LDS in binary32, 32 rows at a time, so that a lane has eight consecutive columns of a row, as GU is loaded and dGU stored.  GU is requested in parts of four such
// pieces, ahead parts in advance in whole tiles (8192 x 18944 x 3584 with h: 648 us without, 631 with two, 621 with three, 622 with four), for 32 rows at a time in guarded ones, and in 128 x 128, where that
// is half of all, if h is not wanted (both halves in advance / one at a time: 512 x 8192 x 1024 14.4 / 13.6, x 2048 17.5 / 17.0, 1024 x 4096 x 4096 24.5 / 23.7; with h 512 x 8192 x 2048 18.07 / 18.2).
// STREAMED: GU past what the caches hold.
template <int NI, int MI, int MJ, int EDGE, bool STREAMED>
struct GluBackward {
    static constexpr int kSlots = 2 * MJ, kPitch = 32 * kSlots, kPieces = 32 * kSlots / kWave, kAtOnce = kPieces < 4 ? kPieces : 4, kParts = kPieces / kAtOnce, kAll = NI * kParts;
    static constexpr int ahead(bool with_h) { return EDGE != kNoEdge || (kAll <= 2 && !with_h) ? 0 : 3 < kAll ? 3 : kAll; }
    static_assert(kPieces >= 1 && kWave % kSlots == 0 && kPieces % kAtOnce == 0, "every lane moves whole pieces");
    struct Kept { v4u g[kAtOnce], u[kAtOnce]; };
    typedef GluRows<EDGE, kSlots> Rows;
    static __device__ __attribute__((always_inline)) void request(Kept& into, const Rows& gate, const Rows& up, int part) {
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            into.g[k] = gate.template load<STREAMED>(part / kParts, part % kParts * kAtOnce + k);
            into.u[k] = up.template load<STREAMED>(part / kParts, part % kParts * kAtOnce + k);
        }
    }
    template <class Acc>
    static __device__ __attribute__((always_inline)) unsigned write_out(const Acc& acc, uint8_t* stage, uint16_t* dgu, const GluPlan& plan, int row0, int M, int col0, int I, int lane) {
        const int fr_row = lane & 15, fr_q = lane >> 4, piece0 = fr_q >> 1, unit_off = (fr_q & 1) * (16 * kSlots);
        const bool by_eight = EDGE == kNoEdge || I % 8 == 0;
        auto rows_of = [&](const uint16_t* p, int ld) __attribute__((always_inline)) { return Rows(p + (size_t)row0 * ld + col0, ld, 32 * NI, M - row0, I - col0, by_eight, lane); };
        const Rows gate = rows_of(plan.gu, 2 * I), up = rows_of(plan.gu + I, 2 * I), dgate = rows_of(dgu, 2 * I), dup = rows_of(dgu + I, 2 * I), h = rows_of(plan.h_out ? plan.h_out : dgu, I);
        unsigned mag = 0, ignored = 0;
        float maxabs = 0.0f;
        auto body = [&](auto with_h) __attribute__((always_inline)) {
            constexpr int AHEAD = ahead(decltype(with_h)::value), kKept = AHEAD ? AHEAD + 1 : kParts;
            auto staged = [&](int k, v4f (&dh)[2]) __attribute__((always_inline)) {
                const int p = lane + k * kWave, r = p / kSlots, sl = p % kSlots;
                const uint8_t* src = stage + r * kPitch + (((sl + r) % kSlots) << 4);
                dh[0] = *reinterpret_cast<const v4f*>(src);
                dh[1] = *reinterpret_cast<const v4f*>(src + 16 * kSlots);
            };
            auto finish = [&](int i, int k, const v4f (&dh)[2], const v4u& g, const v4u& u) __attribute__((always_inline)) {
                v4u dg, du, y;
                glu_gradient8(dh, g, u, dg, du, y, maxabs);
                dgate.store(i, k, dg, mag);
                dup.store(i, k, du, mag);
                if constexpr (decltype(with_h)::value) h.store(i, k, y, ignored);
            };
            Kept kept[kKept];
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) request(kept[n], gate, up, n);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (AHEAD == 0) {
                    if (gate.vector()) {
#pragma unroll
                        for (int part = 0; part < kParts; ++part) request(kept[part], gate, up, i * kParts + part);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int ii = 0; ii < 2; ++ii) {
                    const int row = 16 * ii + fr_row;
#pragma unroll
                    for (int j = 0; j < MJ; ++j) *reinterpret_cast<v4f*>(stage + row * kPitch + unit_off + (((2 * j + piece0 + row) % kSlots) << 4)) = acc.get(2 * i + ii, j);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (gate.vector()) {
#pragma unroll
                    for (int part = 0; part < kParts; ++part) {
                        const int n = i * kParts + part, k0 = part * kAtOnce;
                        if constexpr (AHEAD > 0) {
                            if (n + AHEAD < kAll) request(kept[(n + AHEAD) % kKept], gate, up, n + AHEAD);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                        v4f dh[kAtOnce][2];
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) staged(k0 + k, dh[k]);
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
                            finish(i, k0 + k, dh[k], kept[n % kKept].g[k], kept[n % kKept].u[k]);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                } else {
                    if constexpr (EDGE != kNoEdge) {
                        // two pieces at a time, whose GU is on its way together
#pragma unroll 1
                        for (int k = 0; k < kPieces; k += 2) {
                            v4u g[2], u[2];
#pragma unroll
                            for (int n = 0; n < 2; ++n) g[n] = gate.load(i, k + n), u[n] = up.load(i, k + n);
#pragma unroll
                            for (int n = 0; n < 2; ++n) {
                                v4f dh[2];
                                staged(k + n, dh);
                                finish(i, k + n, dh, g[n], u[n]);
                            }
                        }
                    }
                }
            }
        };
        if (plan.h_out) body(BoolTag<true>{});
        else body(BoolTag<false>{});
        return EDGE == kNoEdge ? (unsigned)__builtin_bit_cast(uint16_t, (__bf16)maxabs) : mag;
    }
};

template <int DIR, class Base, int PAIR_BLOCKS = 1, bool STREAMED = false>
struct GluTuning : Base {
    static constexpr bool kBlockScales = true;
    static constexpr int kGlu = DIR;
    static constexpr int kPairBlocks = PAIR_BLOCKS;
    typedef GluPlan Plan;
    typedef GluOut<DIR> Out;
    template <int NI, int MI, int MJ, int EDGE>
    using Epilogue = std::conditional_t<DIR == kGluForward, GluForward<NI, MI, MJ, EDGE>, GluBackward<NI, MI, MJ, EDGE, STREAMED>>;
};

// M x I x T: rows, pairs (forward) or columns (backward), contraction
struct GluOperands {
    const uint8_t *A, *sA, *B, *sB;
    int64_t M, I, T;
    uint16_t* c;                                // forward: h, backward: dGU
    GluPlan plan;
    unsigned* amax;
};

// What a contraction takes: the kernel for few rows, else the tile.  loose: the up rows do not start at a multiple of 32.
struct GluChoice {
    bool few;
    TilePlan tile;
    bool loose;
};

template <int FA, int FB, int DIR, int NI, int NJ, int EDGE>
static void launch_glu_tile(const GluOperands& p, bool loose, hipStream_t stream, int num_cus) {
    constexpr int kCols = DIR == kGluForward ? 32 * NJ : 64 * NJ;             // of h
    const int tiles_r = (int)((p.M + 64 * NI - 1) / (64 * NI)), tiles_c = (int)((p.I + kCols - 1) / kCols);
    GluPlan plan = p.plan;
    plan.n_whole = tiles_r * tiles_c;
    const int grid = (plan.n_whole + kXcds - 1) / kXcds * kXcds, slots = resident_slots(num_cus, NI, NJ);
    const int touch = NI == 2 && NJ == 2 ? touch_ahead_pair() : touch_ahead(), band = band_rows();
    const int share_b = band < tiles_r ? band : tiles_r, share_a = 4 < tiles_c ? 4 : tiles_c;
    const int next_stride = EDGE == kNoEdge ? successor_stride(NI, NJ, plan.n_whole, slots) : 0;
    auto launch = [&](auto tuning, int threads = kGemmThreads) {
        hipLaunchKernelGGL((gemm_tile_kernel<FA, FB, NI, NJ, EDGE != kNoEdge, decltype(tuning), false, false, kWholeTiles, EDGE>), dim3(grid), dim3(threads), 0, stream, p.A, p.B, p.c, (int)p.I, (int)p.T,
                           reinterpret_cast<const float*>(p.sA), reinterpret_cast<const float*>(p.sB), p.amax, tiles_r, tiles_c, touch, band, next_stride, (int)p.T, (int)p.T, BK, BK, share_a, share_b,
                           plan, (int)p.M, 0);
    };
    // blocks of B whose codes share a register (forward): whole tiles of 256 columns start at multiples of 128 pairs, of which an up row is one of 64 too; the wave of eight has one block of either kind
    constexpr int kShared = EDGE == kNoEdge && NJ == 4 ? 4 : 2;
    const bool forward_loose = DIR == kGluForward && loose;
    if constexpr (NI == 2 && NJ == 2 && EDGE != kEdgeUnaligned) {
        if (deep_stages(plan.n_whole, slots)) {
            if (deep_takes_eight_waves((p.T + BK - 1) / BK, false)) launch(GluTuning<DIR, GemmDeepWideTuning>{}, 2 * kGemmThreads);
            else if (forward_loose) launch(GluTuning<DIR, GemmDeepTuning, 1>{});
            else launch(GluTuning<DIR, GemmDeepTuning, DIR == kGluForward ? kShared : 1>{});
            return;
        }
    }
    if constexpr (DIR == kGluForward && NI == 2 && NJ == 2) {
        if (loose) { launch(GluTuning<DIR, GemmTuning, 1>{}); return; }
    }
    // (GU of more than the memory-side cache holds beside the operands is read past it: 8192 x 18944 x 3584 648 -> 627 us, of what it does hold 1777 x 2720 x 1024 17.9 -> 19.9)
    if constexpr (DIR == kGluBackward && NI == 4 && NJ == 4 && EDGE == kNoEdge) {
        if (4 * p.M * p.I > ((int64_t)128 << 20)) { launch(GluTuning<DIR, GemmTuning, 1, true>{}); return; }
    }
    launch(GluTuning<DIR, GemmTuning, DIR == kGluForward ? kShared : 1>{});
}

// ---- Few rows: see gemm_blocks_few_kernel, whose waves, slots and sums these are.  Forward: a workgroup has 16 pairs, block 0 of its columns their gate rows and block 1 their up rows.
// WAVES share the K steps, SLOTS of which each keeps on their way.  ALIGNED: rows of whole dwords go straight to LDS; others through registers, from offsets cut to the last 16 bytes of the operand.  What a row's
// last chunk brings along of the next row is cleared before it is multiplied.
template <int FA, int FB, int DIR, int RB, int CB, int WAVES, int SLOTS, bool ALIGNED>
__global__ __launch_bounds__(WAVES * kWave) void gemm_glu_few_kernel(const uint8_t* __restrict__ A, const uint8_t* __restrict__ sA, const uint8_t* __restrict__ B, const uint8_t* __restrict__ sB,
                                                                       GluOut<DIR> C, const GluPlan plan, int M, int I, int T, unsigned* __restrict__ amax_bits) {
    static_assert(DIR == kGluBackward || CB == 2, "gates and ups");
    constexpr bool PAIRS = DIR == kGluForward;
    constexpr int kRows = 16 * (RB + CB), kSlot = kRows * BK, kLoads = kRows / 8, kOutOfRange = 0x7FFFFF00, kGroups = PAIRS ? 2 : 1, kOfGroup = CB / kGroups;
    // one LDS object per slot, which the compiler tells apart (see the tile kernel)
    __shared__ __attribute__((aligned(1024))) uint8_t s_0[WAVES * kSlot];
    __shared__ __attribute__((aligned(1024))) uint8_t s_1[WAVES * kSlot];
    __shared__ __attribute__((aligned(1024))) uint8_t s_2[SLOTS > 2 ? WAVES * kSlot : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t s_3[SLOTS > 3 ? WAVES * kSlot : 16];
    const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r0 = (int)blockIdx.y * (16 * RB), c0 = (int)blockIdx.x * (16 * kOfGroup), steps = (T + BK - 1) / BK, mine = (steps - wave + WAVES - 1) / WAVES;      // steps wave, wave + 4, ...
    const int rows_a = M - r0 < 16 * RB ? M - r0 : 16 * RB, rows_b = I - c0 < 16 * kOfGroup ? I - c0 : 16 * kOfGroup;      // of a group
    const uint8_t *const a0 = A + (int64_t)r0 * T, *const b0 = B + (int64_t)c0 * T;
    const int64_t group_bytes = (int64_t)I * T;
    const __amdgpu_buffer_rsrc_t rsA = make_rsrc(a0, (unsigned)((int64_t)rows_a * T)), rsG = make_rsrc(b0, (unsigned)((int64_t)rows_b * T)),
                                 rsU = PAIRS ? make_rsrc(b0 + group_bytes, (unsigned)((int64_t)rows_b * T)) : rsG;
    const int rows_of_b = PAIRS ? 2 * I : I, pitchA = (M + 127) & ~127, pitchB = (rows_of_b + 127) & ~127;
    const __amdgpu_buffer_rsrc_t rsSA = make_rsrc(sA, (unsigned)(steps * pitchA)), rsSB = make_rsrc(sB, (unsigned)(steps * pitchB));
    int code_a[RB], code_b[CB];
#pragma unroll
    for (int i = 0; i < RB; ++i) code_a[i] = (int)block_scale_offset(r0 + 16 * i + (lane & 15), 0, M);
#pragma unroll
    for (int j = 0; j < CB; ++j) code_b[j] = (int)block_scale_offset((PAIRS && j >= kOfGroup ? I : 0) + c0 + 16 * (j % kOfGroup) + (lane & 15), 0, rows_of_b);
    const unsigned end_a = (unsigned)(rows_a * T - 16), end_g = (unsigned)(rows_b * T - 16), end_u = end_g;      // the last 16 bytes of a group's rows
    struct Codes { int a[RB], b[CB]; };
    struct Chunks { v4u c[ALIGNED ? 1 : kLoads]; };
    Codes codes[SLOTS];
    Chunks chunks[SLOTS];
    const int ld_row = lane >> 3;
    auto request = [&](uint8_t* slot, int n, Codes& e, Chunks& held) __attribute__((always_inline)) {
        const int step = wave + n * WAVES;
        const bool there = n < mine;
#pragma unroll
        for (int i = 0; i < RB; ++i) e.a[i] = (int)(unsigned char)__builtin_amdgcn_raw_buffer_load_b8(rsSA, code_a[i], there ? step * pitchA : kOutOfRange, 0);
#pragma unroll
        for (int j = 0; j < CB; ++j) e.b[j] = (int)(unsigned char)__builtin_amdgcn_raw_buffer_load_b8(rsSB, code_b[j], there ? step * pitchB : kOutOfRange, 0);
        __builtin_amdgcn_sched_barrier(0);
        static_for<kLoads>([&](auto piece) {
            constexpr int p = decltype(piece)::value;
            constexpr bool of_a = p < 2 * RB, of_up = PAIRS && p >= 2 * RB + 2 * kOfGroup;
            constexpr int row0 = 8 * (of_a ? p : (p - 2 * RB) % (2 * kOfGroup));
            const int row = row0 + ld_row, k = step * BK + (((lane & 7) ^ row_swizzle(row & 15)) << 4);
            if constexpr (ALIGNED) {
                // (rows behind the operand lie outside the buffer)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(of_a ? rsA : of_up ? rsU : rsG, (lds_void*)(slot + wave * kSlot + p * 8 * BK), 16, there && k < T ? row * T + k : kOutOfRange, 0, 0, 0);
            } else {
                // (all lanes, whatever their chunk is: a branch around each load takes twice the time)
                const unsigned at = (unsigned)(row * T + k), end = of_a ? end_a : of_up ? end_u : end_g;
                if (there) held.c[p] = *reinterpret_cast<const v4u_any*>((of_a ? a0 : of_up ? b0 + group_bytes : b0) + (at < end ? at : end));
            }
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    const int fr_row = lane & 15, fr_q = lane >> 4, swz = row_swizzle(fr_row);
    const int ch0 = ((fr_q * 2) ^ swz) << 4, ch1 = ((fr_q * 2 + 1) ^ swz) << 4;
    v4f acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // LDS runs a wave's accesses in order, and the direct loads that follow are requested behind the wait for the reads
    // behind: steps requested after this one.  The last steps request none, whose codes would be no use to anybody and dropped by the compiler, but counted here.
    auto multiply = [&](uint8_t* slot, int n, Codes& e, Chunks& held, auto behind, auto more) __attribute__((always_inline)) {
        uint8_t* const slab = slot + wave * kSlot;
        // the last K step: a row's chunk that ends in it, or (through registers) lies behind it
        const int left = T - (wave + n * WAVES) * BK;
        if constexpr (ALIGNED) {
            wait_vmcnt<decltype(behind)::value * (kLoads + RB + CB)>();
            if (left < BK && T % 16 != 0) {
                static_for<kLoads>([&](auto piece) {
                    const int valid = left - (((lane & 7) ^ row_swizzle((8 * decltype(piece)::value + ld_row) & 15)) << 4);
                    if (valid > 0 && valid < 16) {
                        v4u* const at = reinterpret_cast<v4u*>(slab + decltype(piece)::value * 8 * BK + lane * 16);
                        *at = first_bytes(*at, valid);
                    }
                });
            }
        } else {
            if (left < BK) {
                static_for<kLoads>([&](auto piece) {
                    constexpr int p = decltype(piece)::value;
                    constexpr bool of_a = p < 2 * RB, of_up = PAIRS && p >= 2 * RB + 2 * kOfGroup;
                    const int row = 8 * (of_a ? p : (p - 2 * RB) % (2 * kOfGroup)) + ld_row, kin = ((lane & 7) ^ row_swizzle(row & 15)) << 4, valid = left - kin;
                    if (valid < 16) {
                        // (a group's last row was loaded from another place)
                        if (valid > 0 && row == (of_a ? rows_a : rows_b) - 1) held.c[p] = load16_upto((of_a ? a0 : of_up ? b0 + group_bytes : b0) + (int64_t)(row + 1) * T - valid, valid);
                        held.c[p] = first_bytes(held.c[p], valid);
                    }
                });
            }
            static_for<kLoads>([&](auto piece) { *reinterpret_cast<v4u*>(slab + decltype(piece)::value * 8 * BK + lane * 16) = held.c[decltype(piece)::value]; });
        }
        auto fragment = [&](int first_row) -> v8i {
            const uint8_t* p = slab + (first_row + fr_row) * BK;
            const v4i lo = *reinterpret_cast<const v4i*>(p + ch0), hi = *reinterpret_cast<const v4i*>(p + ch1);
            return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        };
        v8i a[RB], b[CB];
#pragma unroll
        for (int i = 0; i < RB; ++i) a[i] = fragment(16 * i);
#pragma unroll
        for (int j = 0; j < CB; ++j) b[j] = fragment(16 * (RB + j));
        const Codes now = e;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < CB; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i], acc[i][j], FB, FA, 0, now.b[j], 0, now.a[i]);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (decltype(more)::value) request(slot, n + SLOTS, e, held);
    };
    auto slot_of = [&](auto k) -> uint8_t* { constexpr int K = decltype(k)::value; return K == 0 ? s_0 : K == 1 ? s_1 : K == 2 ? s_2 : s_3; };
    static_for<SLOTS>([&](auto k) { request(slot_of(k), decltype(k)::value, codes[decltype(k)::value], chunks[decltype(k)::value]); });
    int n = 0;
    for (; n + SLOTS <= mine; n += SLOTS)
        static_for<SLOTS>([&](auto k) { multiply(slot_of(k), n + decltype(k)::value, codes[decltype(k)::value], chunks[decltype(k)::value], IntTag<SLOTS - 1>{}, BoolTag<true>{}); });
    static_for<SLOTS - 1>([&](auto k) {
        if (n + decltype(k)::value < mine) multiply(slot_of(k), n + decltype(k)::value, codes[decltype(k)::value], chunks[decltype(k)::value], IntTag<SLOTS - 1 - decltype(k)::value>{}, BoolTag<false>{});
    });
    wait_vmcnt<0>();                             // nothing lands in LDS any more
    __syncthreads();
    v4f* const s_sum = reinterpret_cast<v4f*>(s_0);                          // [wave][block][lane]
    static_assert(RB * CB * kWave * sizeof(v4f) <= (size_t)kSlot, "the sums of a wave fit its slot");
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) s_sum[(wave * (RB * CB) + i * CB + j) * kWave + lane] = acc[i][j];
    __syncthreads();
    auto sum_of = [&](int block) -> v4f {
        v4f y = s_sum[block * kWave + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) y += s_sum[(w * (RB * CB) + block) * kWave + lane];
        return y;
    };
    unsigned mag = 0;
    // a lane's four columns of a row: whole where widths are multiples of 4, else element by element
    auto store = [&](uint16_t* dst, const v4f& y, int left, bool counts) __attribute__((always_inline)) {
        const v2u out = bf16_of(y);
        if (I % 4 == 0) {
            if (counts) mag = pk_max_mag(pk_max_mag(mag, out[0]), out[1]);
            *reinterpret_cast<v2u*>(dst) = out;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) {
                    const unsigned bits = e & 1 ? out[e >> 1] >> 16 : out[e >> 1] & 0xFFFFu;
                    if (counts) mag = pk_max_mag(mag, bits);
                    dst[e] = (uint16_t)bits;
                }
        }
    };
    // a wave finishes every fourth block (of pairs)
    for (int block = wave; block < RB * kOfGroup; block += WAVES) {
        const int i = block / kOfGroup, j = block % kOfGroup, r = r0 + 16 * i + (lane & 15), c = c0 + 16 * j + (lane >> 4) * 4, left = I - c;
        const v4f sum = sum_of(i * CB + j);
        v4f other = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (PAIRS) other = sum_of(i * CB + kOfGroup + j);
        if (r >= M || left <= 0) continue;
        const int64_t at = (int64_t)r * I + c, at2 = (int64_t)r * 2 * I + c;
        if constexpr (PAIRS) {
            v4f y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = glu_value(sum[e], other[e]);
            store(C + at, y, left, true);
            if (plan.gu_out) {
                store(plan.gu_out + at2, sum, left, false);
                store(plan.gu_out + at2 + I, other, left, false);
            }
        } else {
            float g[4], u[4];
            if (I % 4 == 0) {
                const v2u gw = *reinterpret_cast<const v2u*>(plan.gu + at2), uw = *reinterpret_cast<const v2u*>(plan.gu + at2 + I);
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] = e & 1 ? bf16_hi(gw[e >> 1]) : bf16_lo(gw[e >> 1]), u[e] = e & 1 ? bf16_hi(uw[e >> 1]) : bf16_lo(uw[e >> 1]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] = e < left ? bf16_lo(plan.gu[at2 + e]) : 0.0f, u[e] = e < left ? bf16_lo(plan.gu[at2 + I + e]) : 0.0f;
            }
            v4f dg, du, h;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x, z, w;
                glu_gradient(sum[e], g[e], u[e], x, z, w);
                dg[e] = x, du[e] = z, h[e] = w;
            }
            store(C + at2, dg, left, true);
            store(C + at2 + I, du, left, true);
            if (plan.h_out) store(plan.h_out + at, h, left, false);
        }
    }
    if (amax_bits) {
        mag = wave_max_u32((mag & 0xFFFFu) > (mag >> 16) ? mag & 0xFFFFu : mag >> 16);
        const unsigned bits = amax_bits_from_bf16_mag(mag);
        if (lane == 0 && bits > __hip_atomic_load(amax_bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(amax_bits, bits);
    }
}

// Workgroups of four waves and four slots fill a CU and are a chain of a quarter of the steps; workgroups of one wave and three slots lie eight to a CU and have nothing to wait for one another: better where all
// of them have work and no wave's chain is the whole time.  Four waves / one, us, I x T: 16 rows 18944 x 3584 35.0 / 26.7, 11008 x 2048 14.0 / 9.6, 5504 x 2048 9.3 / 7.7, 8192 x 512 5.2 / 3.7; the other way
// 2736 x 2048 4.92 / 7.43, 4096 x 2048 6.1 / 7.6, 5504 x 8192 22.8 / 29.4; 32 rows 18944 x 3584 40.7 / 31.2, 5504 x 3584 13.3 / 13.9.  Through registers (four waves with four slots, one with two): 16 rows 18944 x 3581 49.4 / 40.8,
// 5504 x 2047 12.2 / 12.2, 24 rows 11007 x 1023 15.1 / 10.1, 450 rows 438 x 223 backward 7.9 / 5.9.
template <int FA, int FB, int DIR, int RB, int CB>
static void launch_glu_few(const GluOperands& p, hipStream_t stream, int num_cus) {
    constexpr int kCols = DIR == kGluForward ? 8 * CB : 16 * CB;
    const int64_t groups = (p.I + kCols - 1) / kCols, row_groups = (p.M + 16 * RB - 1) / (16 * RB);
    auto launch = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups, (unsigned)row_groups), dim3(waves * kWave), 0, stream, p.A, p.sA, p.B, p.sB, p.c, p.plan, (int)p.M, (int)p.I, (int)p.T, p.amax);
    };
    const char* alone = tuning_env("LLMQ_GLU_FEW_ALONE");
    if (p.T % 4 != 0) {
        if constexpr (CB == 1 || DIR == kGluForward) {
            if (alone ? atoi(alone) != 0 : groups * row_groups > num_cus && (groups * row_groups >= 2 * num_cus || p.T <= 24 * BK)) launch(gemm_glu_few_kernel<FA, FB, DIR, RB, CB, 1, 2, false>, 1);
            else launch(gemm_glu_few_kernel<FA, FB, DIR, RB, CB, 4, 4, false>, 4);
        }
    } else if (alone ? atoi(alone) != 0 : groups * row_groups > num_cus && (groups * row_groups >= 2 * num_cus || p.T <= 24 * BK)) {
        launch(gemm_glu_few_kernel<FA, FB, DIR, RB, CB, 1, 3, true>, 1);
    } else {
        launch(gemm_glu_few_kernel<FA, FB, DIR, RB, CB, 4, 4, true>, 4);
    }
}

// Launches the kernel of the choice; gemm_glu_*.hip instantiate it for a pair of formats and a direction each.
template <int FA, int FB, int DIR>
void launch_glu(const GluOperands& p, const GluChoice& choice, hipStream_t stream, int num_cus) {
    if (choice.few) {
        if constexpr (DIR == kGluForward) {
            p.M <= 16 ? launch_glu_few<FA, FB, DIR, 1, 2>(p, stream, num_cus) : launch_glu_few<FA, FB, DIR, 2, 2>(p, stream, num_cus);
        } else {
            // (as in the plain contraction)
            const bool two = p.T % 4 == 0 && (p.I + 31) / 32 >= num_cus / 2;
            if (p.M <= 16) two ? launch_glu_few<FA, FB, DIR, 1, 2>(p, stream, num_cus) : launch_glu_few<FA, FB, DIR, 1, 1>(p, stream, num_cus);
            else two ? launch_glu_few<FA, FB, DIR, 2, 2>(p, stream, num_cus) : launch_glu_few<FA, FB, DIR, 2, 1>(p, stream, num_cus);
        }
        return;
    }
#define LLMQ_GLU_CASE(I, J, KIND)                                                        \
    case KIND * 64 + I * 8 + J:                                                          \
        launch_glu_tile<FA, FB, DIR, I, J, KIND>(p, choice.loose, stream, num_cus);      \
        return;
    switch (choice.tile.edge * 64 + choice.tile.ni * 8 + choice.tile.nj) {
        LLMQ_GLU_CASE(4, 4, kNoEdge) LLMQ_GLU_CASE(4, 2, kNoEdge) LLMQ_GLU_CASE(3, 4, kNoEdge) LLMQ_GLU_CASE(2, 4, kNoEdge) LLMQ_GLU_CASE(2, 2, kNoEdge)
        LLMQ_GLU_CASE(4, 4, kEdge) LLMQ_GLU_CASE(3, 4, kEdge) LLMQ_GLU_CASE(4, 2, kEdge) LLMQ_GLU_CASE(2, 4, kEdge) LLMQ_GLU_CASE(2, 2, kEdge)
        LLMQ_GLU_CASE(2, 2, kEdgeUnaligned)
        default: break;
    }
#undef LLMQ_GLU_CASE
}
extern template void launch_glu<0, 0, kGluForward>(const GluOperands&, const GluChoice&, hipStream_t, int);
extern template void launch_glu<1, 0, kGluForward>(const GluOperands&, const GluChoice&, hipStream_t, int);
extern template void launch_glu<0, 0, kGluBackward>(const GluOperands&, const GluChoice&, hipStream_t, int);
extern template void launch_glu<1, 0, kGluBackward>(const GluOperands&, const GluChoice&, hipStream_t, int);

}  // namespace llmq
