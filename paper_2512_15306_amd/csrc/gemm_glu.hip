// Choice of kernel and entry points of the contractions joined with a SwiGLU.
#include "gemm_glu.h"

#include "api_checks.h"

namespace llmq {

// M x I x T as in GluOperands.  LLMQ_GLU_FEW=0 / 1 (tests): the kernel for few rows never, or for up to 4096 rows always; else LLMQ_GLU_TILE=IxJ: that tile where it is built for
// the shape.
//
// The kernel for few rows reads its operands straight from memory and divides the contraction between waves, so it has no tile to fill and ends one short wait after it began.  It
// takes what is bounded by reading the weights, and problems of up to four of its workgroups a CU.  Tiles / few, us, M x I x T: forward 16 x 18944 x 3584 45.0 / 26.6, 128 x 512 x 1024 7.6 / 3.9,
// 300 x 800 x 400 6.2 / 4.7, 256 x 1024 x 3584 16.8 / 15.6, 2048 x 256 x 512 6.05 / 5.2, 128 x 4096 x 2048 11.7 / 11.2, 96 x 5024 x 1024 8.6 / 8.7, 64 x 3000 x 2001 20.3 / 13.9; backward 128 x 512 x 1024
// 8.8 / 3.7, 1000 x 512 x 1024 9.6 / 7.9, 64 x 4096 x 3584 17.8 / 7.1, 248 x 1839 x 167 16.3 / 9.25; beyond the rule, forward: 64 x 18944 x 3584 45.3 / 49.4, 65 x 6675 x 868 9.5 / 11.5, 40 x 12000 x 2001 19.3 / 24.1.
template <int DIR>
static GluChoice choose_glu(int64_t M, int64_t I, int64_t T, int num_cus) {
    GluChoice choice{false, {0, 0, kNoEdge}, DIR == kGluForward && I % 32 != 0};
    const char* few = tuning_env("LLMQ_GLU_FEW");
    const int64_t cols = DIR == kGluForward ? 2 * I : I, steps = (T + BK - 1) / BK, groups = (M + 31) / 32 * ((I + 15) / 16);
    const bool small = M <= 32 || groups <= num_cus || (groups <= 4 * num_cus && groups * steps <= 64 * num_cus);
    // (Rows of whole dwords go straight to LDS.  Through registers, in tiles of 128 x 128 / straight: forward 1777 x 2720 x 1000 28.5 / 22.5 us, 4001 x 8000 with T = 2001 / 2004 265 / 154; backward
    // 1777 x 2720 x 1000 21.9 / 19.85, 4001 x 8001 with T = 2001 / 2004 210 / 175.  Through registers a tile of twice the size is 5 % faster on 4001 x 8000 x 2001 and takes 35 for 1777 x 2720 x 1000.)
    auto form = [&](int ni, int nj) {
        const bool whole = M % (64 * ni) == 0 && cols % (64 * nj) == 0 && T % BK == 0 && !choice.loose;
        return TilePlan{ni, nj, whole ? kNoEdge : T % 4 == 0 ? kEdge : kEdgeUnaligned};
    };
    // 128 x 128 is built for everything; the others for chunks that go straight to LDS, and forward where the codes of two blocks of rows can share a register
    auto built = [&](const TilePlan& p) { return (p.ni == 2 && p.nj == 2) || (p.edge != kEdgeUnaligned && !choice.loose); };
    const char* e = tuning_env("LLMQ_GLU_TILE");
    choice.few = few ? atoi(few) != 0 && M <= 4096 : small && !e;
    if (choice.few) return choice;
    if (e) {
        if (e[0] >= '2' && e[0] <= '4' && e[1] == 'x' && (e[2] == '2' || e[2] == '4') && !(e[0] == '3' && e[2] == '2')) {
            const TilePlan p = form(e[0] - '0', e[2] - '0');
            if (built(p)) { choice.tile = p; return choice; }
        }
    }
    if (((M + 127) / 128) * ((cols + 127) / 128) <= resident_slots(num_cus, 2, 2) / 2) { choice.tile = form(2, 2); return choice; }
    static const int forms[][2] = {{4, 4}, {3, 4}, {4, 2}, {2, 4}, {2, 2}};
    double best_us = 0.0;
    for (const auto& f : forms) {
        const TilePlan p = form(f[0], f[1]);
        const int64_t tiles = ((M + 64 * p.ni - 1) / (64 * p.ni)) * ((cols + 64 * p.nj - 1) / (64 * p.nj));
        if (!built(p) || tiles > kMaxWorkgroups) continue;
        const double us = tile_us(p, tiles, steps, DIR == kGluBackward, cols % 8 != 0, resident_slots(num_cus, p.ni, p.nj));
        if (choice.tile.ni == 0 || us < best_us) { choice.tile = p; best_us = us; }
    }
    return choice;
}

}  // namespace llmq

namespace {

// 32-bit offsets from the first row of a tile, of operands, scales and outputs; sixteen bytes in every row of an operand
int check_glu(const uint8_t* A, const uint8_t* sA, int fmtA, const uint8_t* B, const uint8_t* sB, int fmtB, int64_t M, int64_t I, int64_t T, int64_t rows_of_b, const void* gu, const void* out, const void* other,
              const float* d_amax) {
    if (!dim_ok(M) || !dim_ok(I) || !dim_ok(T) || T < 16 || T >= (1ll << 22) || I >= (1ll << 21)) return LLMQ_ERR_SHAPE;
    const int64_t steps = (T + 127) / 128, rows = M > rows_of_b ? M : rows_of_b;
    if (steps * ((rows + 127) / 128 * 128) >= 0x7FFFF000ll || M * I >= kMaxElems / 2 || ((M + 127) / 128) * ((I + 63) / 64) > (int64_t)llmq::kMaxWorkgroups) return LLMQ_ERR_SHAPE;
    if (!fmt_ok(fmtA) || fmtB != LLMQ_E4M3) return LLMQ_ERR_FORMAT;
    if (!aligned(A, 16) || !aligned(sA, 16) || !aligned(B, 16) || !aligned(sB, 16) || !aligned(gu, 16) || !aligned(out, 16) || !aligned(other, 16) || !aligned(d_amax, 4)) return LLMQ_ERR_ALIGN;
    return LLMQ_OK;
}

template <int DIR>
int run_glu(const llmq::GluOperands& p, int fmtA, void* stream) {
    const int cus = num_cus();
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (p.amax) llmq::launch_gemm_amax_reset(p.amax, s);
    const llmq::GluChoice choice = llmq::choose_glu<DIR>(p.M, p.I, p.T, cus);
    if (fmtA == LLMQ_E4M3) llmq::launch_glu<0, 0, DIR>(p, choice, s, cus);
    else llmq::launch_glu<1, 0, DIR>(p, choice, s, cus);
    return hipGetLastError() == hipSuccess ? LLMQ_OK : LLMQ_ERR_DEVICE;
}

}  // namespace

extern "C" {

int llmq_fp8_gemm_blocks_swiglu_fwd(const uint8_t* A, const uint8_t* sA, int fmtA, const uint8_t* W, const uint8_t* sW, int fmtW, int64_t M, int64_t I, int64_t T, void* h_bf16, void* gu_bf16, float* d_amax_h,
                                    void* stream) {
    if (!A || !sA || !W || !sW || !h_bf16) return LLMQ_ERR_NULL;
    const int st = check_glu(A, sA, fmtA, W, sW, fmtW, M, I, T, 2 * I, gu_bf16, h_bf16, nullptr, d_amax_h);
    if (st != LLMQ_OK) return st;
    return run_glu<llmq::kGluForward>({A, sA, W, sW, M, I, T, static_cast<uint16_t*>(h_bf16), {0, nullptr, static_cast<uint16_t*>(gu_bf16), nullptr}, reinterpret_cast<unsigned*>(d_amax_h)}, fmtA, stream);
}

int llmq_fp8_gemm_blocks_swiglu_bwd(const uint8_t* A, const uint8_t* sA, int fmtA, const uint8_t* B, const uint8_t* sB, int fmtB, const void* gu_bf16, int64_t M, int64_t I, int64_t T, void* dgu_bf16,
                                    void* h_bf16, float* d_amax_dgu, void* stream) {
    if (!A || !sA || !B || !sB || !gu_bf16 || !dgu_bf16) return LLMQ_ERR_NULL;
    const int st = check_glu(A, sA, fmtA, B, sB, fmtB, M, I, T, I, gu_bf16, dgu_bf16, h_bf16, d_amax_dgu);
    if (st != LLMQ_OK) return st;
    return run_glu<llmq::kGluBackward>({A, sA, B, sB, M, I, T, static_cast<uint16_t*>(dgu_bf16), {0, static_cast<const uint16_t*>(gu_bf16), nullptr, static_cast<uint16_t*>(h_bf16)},
                                        reinterpret_cast<unsigned*>(d_amax_dgu)}, fmtA, stream);
}

}  // extern "C"
