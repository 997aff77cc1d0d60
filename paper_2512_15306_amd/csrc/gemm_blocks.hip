// Choice of kernel and entry point of the contraction with block scales.
#include "gemm_blocks.h"

#include "api_checks.h"

namespace llmq {

// Whether a contraction of few rows takes the kernel for those: more than one K step, and where its workgroups come in several rounds, enough of them.  The kernels below /
// it, R x C x T, microseconds: 1 x 4608 x 3584 8.2 / 5.8, 16 x 1024 x 8192 13.8 / 7.3, 16 x 18944 x 3584 23.8 / 19.9, 5 x 39782 x 6960 80.5 / 50.6, 32 x 512 x 512 4.2 / 3.1,
// 5 x 700 x 333 9.9 / 3.2, 9 x 5305 x 4643 40.2 / 17.0, 2 x 11141 x 12797 122 / 81;  and where they are faster 3 x 26124 x 1632 12.6 / 15.2, 28 x 20369 x 1120 10.9 / 12.8,
// 3 x 9669 x 480 4.8 / 5.0, 2 x 6136 x 128 2.9 / 3.4, 2 x 25206 x 2203 26.4 / 31.8.
// Rows that are no whole 16-byte chunks leave other contractions of few outputs to 128 x 128 tiles or to bytes one by one: those take this kernel too, in groups of 32 rows, where two
// rounds of its workgroups at most are the faster ones by the fitted times below.  The others / it: 99 x 406 x 612 11.9 / 5.4, 500 x 500 x 333 13.3 / 8.2, 100 x 512 x 9999 63.6 / 41.5,
// 1 x 333 x 20 6.2 / 4.0, 300 x 300 x 127 7.5 / 5.1;  145 x 2091 x 890 15.3 / 17.6, 777 x 333 x 1999 24.3 / 28.7, 1000 x 1000 x 200 8.7 / 24.4.
// LLMQ_FEW=0 / 1 (tests): never, or for up to 4096 rows always.
static bool takes_few(int64_t R, int64_t C, int64_t T, int num_cus) {
    if (const char* e = tuning_env("LLMQ_FEW")) return atoi(e) != 0 && R <= 4096;
    const int64_t steps = (T + BK - 1) / BK;
    if (R <= 32 && steps > 1 && (C <= 8192 || steps >= (T % 16 == 0 ? 20 : 40))) return true;
    const int64_t rounds = ((R + 31) / 32 * ((C + 15) / 16) + num_cus - 1) / num_cus;
    return T % 16 != 0 && rounds <= (steps > 1 ? 2 : 1) && 1.9 + 2.6 * (double)rounds + (rounds == 1 ? 0.39 : 0.95) * (double)steps < 5.5 + 0.85 * (double)steps + (C % 8 != 0 ? 2.5 : 0.0);
}

// Whether full rounds of 256 x 256 tiles and a strip of the last rows or columns, in tiles of its own, take less time together than `least`: a round of a few large
// tiles takes nearly as long as a full one, although less than the model says where the power of the idle CUs goes to the others: hence a margin of 7 %.  All sides multiples of
// 128, T too, 8 K steps at least.  R x C x T, one launch / two, microseconds: 3584 x 18944 x 8192 (4.05 rounds) 458 / 428, 11264 x 1536 x 11264 214 / 177, 3456 x 15616 x 11648
// 521 / 475, 6272 x 11264 x 1280 114 / 103, 9984 x 5120 x 2048 110 / 104, 16000 x 13312 x 1664 402 / 403, 11008 x 13184 x 5120 541 / 552;  10880 x 1792 x 896 31.1 / 33.4.  Of shapes of
// 512 to 19072 rows and columns, T of 512 to 12288, a fifth is cut, and takes 1.8 % less time on average.
// LLMQ_BLOCKS_STRIP=0, rN, cN (tests): no strip, or one of N rows or columns wherever it leaves whole tiles.
static void cut_strip(BlocksPlan& plan, int64_t R, int64_t C, int64_t steps, bool accumulate, int num_cus, double least) {
    const char* const forced = tuning_env("LLMQ_BLOCKS_STRIP");
    if (forced ? forced[0] == '0' : steps < 8) return;
    const int64_t slots = resident_slots(num_cus, 4, 4);
    for (const bool by_rows : {false, true}) {
        const int64_t across = by_rows ? C : R, along = by_rows ? R : C, tiles_across = across / 256, rounds = tiles_across * (along / 256) / slots;
        if (across % 256 != 0) continue;
        int64_t first = rounds * slots / tiles_across * 256;
        if (forced) first = forced[0] == (by_rows ? 'r' : 'c') ? along - atoi(forced + 1) : 0;
        const int64_t strip = along - first, tiles = tiles_across * (first / 256);
        if (first <= 0 || first % 256 != 0 || strip <= 0 || strip % 128 != 0 || tiles > kMaxWorkgroups) continue;
        // the strip's tile and time
        double us = 0.0;
        TilePlan tile{};
        for (int i = 4; i >= 2; --i)
            for (int j = 4; j >= 2; --j) {
                if ((by_rows ? strip : across) % (64 * i) != 0 || (by_rows ? across : strip) % (64 * j) != 0) continue;
                const int64_t n = across * strip / (4096 * i * j);
                const double t = i == 2 && j == 2 && n <= resident_slots(num_cus, 2, 2) / 2 ? 4.5 + 0.39 * (double)steps             // (four LDS stages)
                                                                                            : tile_us({i, j, kNoEdge}, n, steps, accumulate, false, resident_slots(num_cus, i, j));
                if (us == 0.0 || t < us) { us = t; tile = TilePlan{i, j, kNoEdge}; }
            }
        us += tile_us({4, 4, kNoEdge}, tiles, steps, accumulate, false, slots);
        if (forced || us < least) {
            least = us;
            plan.tile = TilePlan{4, 4, kNoEdge}, plan.strip = tile, plan.strip_rows = by_rows ? strip : 0, plan.strip_cols = by_rows ? 0 : strip;
        }
    }
}

static BlocksPlan plan_blocks(int64_t R, int64_t C, int64_t T, bool accumulate, bool with_amax, int num_cus) {
    BlocksPlan plan{false, 0, {0, 0, kNoEdge}, 0, 0, {}};
    const int64_t steps = (T + BK - 1) / BK, rounded = ((R > C ? R : C) + 127) / 128 * 128;
    // 32-bit offsets from the first row of a tile, of operands, scales and output; sixteen bytes in every row of an operand
    if (T < 16 || T >= (1ll << 22) || C >= (1ll << 22) || steps * rounded >= 0x7FFFF000ll) return plan;
    const bool aligned_rows = T % 16 == 0;
    auto form = [&](int ni, int nj) {
        const bool whole = R % (64 * ni) == 0 && C % (64 * nj) == 0 && T % BK == 0;
        return TilePlan{ni, nj, whole ? kNoEdge : aligned_rows ? kEdge : kEdgeUnaligned};
    };
    // guarded tiles are not built 192 columns wide, nor 192 rows high or 256 x 256 with chunks that go through registers (those would spill accumulators)
    auto built = [&](const TilePlan& p) { return p.edge == kNoEdge || (p.nj != 3 && (p.edge == kEdge || (p.ni != 3 && p.ni * p.nj < 16))); };
    if (const char* e = tuning_env("LLMQ_GEMM_ANY_TILE")) {
        if (e[0] >= '2' && e[0] <= '4' && e[1] == 'x' && e[2] >= '2' && e[2] <= '4') {
            const TilePlan p = form(e[0] - '0', e[2] - '0');
            if (built(p)) { plan.tile = p; return plan; }
        }
        if (e[0] == '0') return plan;
    }
    const bool ragged = R % 128 != 0 || C % 128 != 0 || T % BK != 0;
    if (tuning_env("LLMQ_BLOCKS_STRIP") && !ragged) {
        cut_strip(plan, R, C, steps, accumulate, num_cus, 0.0);
        if (plan.tile.ni) return plan;
    }
    plan.few = takes_few(R, C, T, num_cus);
    if (plan.few) return plan;
    plan.side = aligned_rows ? takes_mini(R, C, T, false, false, accumulate, with_amax, false, num_cus) : 0;
    if (plan.side) return plan;
    if (ragged && generic_is_faster(R, C, T, false, false, accumulate, with_amax, false, num_cus)) return plan;
    if (((R + 127) / 128) * ((C + 127) / 128) <= resident_slots(num_cus, 2, 2) / 2) { plan.tile = form(2, 2); return plan; }
    double best_us = 0.0;
    for (int ni = 4; ni >= 2; --ni)
        for (int nj = 4; nj >= 2; --nj) {
            const int64_t tiles = ((R + 64 * ni - 1) / (64 * ni)) * ((C + 64 * nj - 1) / (64 * nj));
            if (tiles > kMaxWorkgroups) continue;
            const TilePlan p = form(ni, nj);
            if (!built(p)) continue;
            const double us = tile_us(p, tiles, steps, accumulate, C % 8 != 0, resident_slots(num_cus, ni, nj));
            if (plan.tile.ni == 0 || us < best_us) { plan.tile = p; best_us = us; }
        }
    if (!ragged) cut_strip(plan, R, C, steps, accumulate, num_cus, 0.93 * best_us);
    return plan;
}

}  // namespace llmq

extern "C" int llmq_fp8_gemm_blocks(const uint8_t* A, const uint8_t* sA, int fmtA, const uint8_t* B, const uint8_t* sB, int fmtB, int64_t R, int64_t C,
                                    int64_t T, void* c_bf16, int accumulate, float* d_amax_c, void* stream) {
    if (!A || !sA || !B || !sB || !c_bf16) return LLMQ_ERR_NULL;
    if (!dim_ok(R) || !dim_ok(C) || !dim_ok(T)) return LLMQ_ERR_SHAPE;
    if (R * T >= kMaxElems || C * T >= kMaxElems || R * C >= kMaxElems) return LLMQ_ERR_SHAPE;
    if (!fmt_ok(fmtA) || !fmt_ok(fmtB)) return LLMQ_ERR_FORMAT;
    if (!aligned(A, 16) || !aligned(sA, 16) || !aligned(B, 16) || !aligned(sB, 16) || !aligned(c_bf16, 16) || !aligned(d_amax_c, 4)) return LLMQ_ERR_ALIGN;
    const int cus = num_cus();
    const llmq::BlocksPlan plan = llmq::plan_blocks(R, C, T, accumulate != 0, d_amax_c != nullptr, cus);
    // the generic kernel's grid has a workgroup of 32 x 32 outputs for each of its two dimensions
    if (plan.side == 0 && plan.tile.ni == 0 && (R >= (1ll << 21) || C >= (1ll << 28))) return LLMQ_ERR_SHAPE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    unsigned* amax = reinterpret_cast<unsigned*>(d_amax_c);
    if (amax) llmq::launch_gemm_amax_reset(amax, s);
    const llmq::BlocksOperands p{A, sA, B, sB, R, C, T, R, C, c_bf16, accumulate != 0, amax};
    if (fmtA == LLMQ_E4M3 && fmtB == LLMQ_E4M3) llmq::launch_blocks<0, 0>(p, plan, s, cus);
    else if (fmtA == LLMQ_E5M2 && fmtB == LLMQ_E4M3) llmq::launch_blocks<1, 0>(p, plan, s, cus);
    else if (fmtA == LLMQ_E4M3 && fmtB == LLMQ_E5M2) llmq::launch_blocks<0, 1>(p, plan, s, cus);
    else llmq::launch_blocks<1, 1>(p, plan, s, cus);
    return hipGetLastError() == hipSuccess ? LLMQ_OK : LLMQ_ERR_DEVICE;
}
