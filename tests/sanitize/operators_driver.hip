// Host code of the block-scaled contraction and of AdamW's plans under the sanitizers: what a plan launches computes every output once and addresses no operand or scale out of range; a table of
// pieces covers every tensor once; arrays that overlap are found as a comparison of all pairs finds them.  Nothing is launched.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <random>
#include <vector>

#include "../../paper_2512_15306_amd/csrc/gemm_blocks.hip"
#include "../../paper_2512_15306_amd/csrc/adamw.hip"

// (the launchers are never called here)
namespace llmq {
void launch_gemm_amax_reset(unsigned*, hipStream_t) {}
}

using namespace llmq;

static int g_fail = 0;
#define CHECK(cond, ...)                                  \
    do {                                                  \
        if (!(cond)) {                                    \
            if (g_fail < 20) { printf("FAIL %s:%d %s: ", __FILE__, __LINE__, #cond); printf(__VA_ARGS__); printf("\n"); } \
            ++g_fail;                                     \
        }                                                 \
    } while (0)

// One launch of tiles of 64 ni x 64 nj over rows x cols outputs that begin at (r0, c0): counts every square of 64 x 64
static void walk_tiles(const TilePlan& t, int64_t r0, int64_t c0, int64_t rows, int64_t cols, std::vector<int>& seen, int64_t wide) {
    const int tiles_r = (int)((rows + 64 * t.ni - 1) / (64 * t.ni)), tiles_c = (int)((cols + 64 * t.nj - 1) / (64 * t.nj)), n = tiles_r * tiles_c, grid = (n + kXcds - 1) / kXcds * kXcds;
    CHECK(grid <= (int)kMaxWorkgroups, "%d workgroups", grid);
    if (t.edge == kNoEdge) CHECK(rows % (64 * t.ni) == 0 && cols % (64 * t.nj) == 0, "%lld x %lld in whole tiles of %d x %d", (long long)rows, (long long)cols, 64 * t.ni, 64 * t.nj);
    for (int id = 0; id < grid; ++id) {
        const int pos = walk_position(id, n);
        if (pos < 0) continue;
        int tr, tc;
        tile_of_position(pos, tiles_r, tiles_c, 4, tr, tc);
        for (int i = 0; i < t.ni; ++i)
            for (int j = 0; j < t.nj; ++j) {
                const int64_t r = (r0 + (int64_t)tr * 64 * t.ni) / 64 + i, c = (c0 + (int64_t)tc * 64 * t.nj) / 64 + j;
                if (r * 64 < r0 + rows && c * 64 < c0 + cols) ++seen[r * wide + c];
            }
    }
}

static int g_strips = 0, g_few = 0, g_mini = 0, g_generic = 0, g_guarded = 0;
static void check_blocks(int64_t R, int64_t C, int64_t T, bool accumulate, bool amax) {
    const BlocksPlan p = plan_blocks(R, C, T, accumulate, amax, 256);
    const int64_t steps = (T + BK - 1) / BK, pitch_a = (R + 127) / 128 * 128, pitch_b = (C + 127) / 128 * 128;
    const bool generic = !p.few && !p.side && !p.tile.ni;
    if (!generic) {          // 32-bit offsets of scales, from the first code on, and of an operand's rows from the first row of a tile on
        CHECK(T >= 16 || p.few, "%lld x %lld x %lld", (long long)R, (long long)C, (long long)T);
        CHECK(steps * pitch_a < 0x7FFFF000ll && steps * pitch_b < 0x7FFFF000ll && T < (1ll << 22) && C < (1ll << 22), "%lld x %lld x %lld: scales out of range", (long long)R, (long long)C, (long long)T);
    }
    if (p.few) {
        ++g_few;
        const bool two = T % 16 == 0 && (C + 31) / 32 >= 128;
        const int64_t gx = two ? (C + 31) / 32 : (C + 15) / 16, gy = R <= 16 ? 1 : (R + 31) / 32;
        CHECK(gx <= (int64_t)kMaxWorkgroups && gy <= 65536 && gx * gy <= (int64_t)kMaxWorkgroups, "%lld x %lld x %lld: grid %lld x %lld", (long long)R, (long long)C, (long long)T, (long long)gx, (long long)gy);
        CHECK(T % 16 == 0 || !two, "%lld x %lld x %lld: no such kernel", (long long)R, (long long)C, (long long)T);
    } else if (p.side) {
        ++g_mini;
        CHECK(T % 16 == 0 && R < (1ll << 23) && C < (1ll << 23), "%lld x %lld x %lld: side %d", (long long)R, (long long)C, (long long)T, p.side);
    } else if (generic) {
        ++g_generic;
    } else {
        const int64_t wide = (C + 63) / 64, high = (R + 63) / 64;
        if (p.tile.edge != kNoEdge) ++g_guarded;
        CHECK(p.tile.edge != kEdge || T % 16 == 0, "%lld x %lld x %lld: chunks across rows", (long long)R, (long long)C, (long long)T);
        CHECK(!(p.strip_rows && p.strip_cols), "two strips");
        const bool strip = p.strip_rows || p.strip_cols;
        if (strip) {
            ++g_strips;
            CHECK(p.tile.edge == kNoEdge && p.strip.edge == kNoEdge && p.tile.ni == 4 && p.tile.nj == 4, "a strip beside guarded tiles");
            CHECK(p.strip_rows >= 0 && p.strip_rows < R && p.strip_cols >= 0 && p.strip_cols < C, "strip %lld, %lld", (long long)p.strip_rows, (long long)p.strip_cols);
        }
        const int64_t r = p.strip_rows ? R - p.strip_rows : 0, c = p.strip_cols ? C - p.strip_cols : 0;
        // the strip's scales: from its first row's code on, those of the whole operand
        CHECK(r % 128 == 0 && c % 128 == 0, "strip at (%lld, %lld)", (long long)r, (long long)c);
        for (int64_t i : {(int64_t)0, (int64_t)17, (int64_t)127}) {
            if (p.strip_rows) CHECK(r + block_scale_offset(i, 0, R) == block_scale_offset(r + i, 0, R) && r + block_scale_offset(i, steps - 1, R) == block_scale_offset(r + i, steps - 1, R), "codes of row %lld", (long long)(r + i));
            if (p.strip_cols) CHECK(c + block_scale_offset(i, 0, C) == block_scale_offset(c + i, 0, C) && c + block_scale_offset(i, steps - 1, C) == block_scale_offset(c + i, steps - 1, C), "codes of column %lld", (long long)(c + i));
        }
        if (wide * high > 4000000) return;
        std::vector<int> seen((size_t)(wide * high), 0);
        if (strip) {
            walk_tiles(p.tile, 0, 0, r ? r : R, c ? c : C, seen, wide);
            walk_tiles(p.strip, r, c, p.strip_rows ? p.strip_rows : R, p.strip_cols ? p.strip_cols : C, seen, wide);
        } else {
            walk_tiles(p.tile, 0, 0, R, C, seen, wide);
        }
        int64_t bad = 0;
        for (int n : seen) bad += n != 1;
        CHECK(bad == 0, "%lld x %lld x %lld: %lld squares not computed once (tile %d x %d, strip %lld, %lld)", (long long)R, (long long)C, (long long)T, (long long)bad, p.tile.ni, p.tile.nj, (long long)p.strip_rows,
              (long long)p.strip_cols);
    }
}

// Codes of all rows and steps lie in llmq_block_scales_bytes, each at a place of its own
static void check_places(int64_t rows, int64_t T) {
    const int64_t steps = (T + 127) / 128, n = (rows + 127) / 128 * 128 * steps;
    std::vector<char> seen((size_t)n, 0);
    for (int64_t r = 0; r < rows; ++r)
        for (int64_t k = 0; k < steps; ++k) {
            const int64_t at = block_scale_offset(r, k, rows);
            CHECK(at >= 0 && at < n, "row %lld step %lld at %lld of %lld", (long long)r, (long long)k, (long long)at, (long long)n);
            if (at >= 0 && at < n) { CHECK(!seen[at], "row %lld step %lld: the place of another", (long long)r, (long long)k); seen[at] = 1; }
        }
}

// ---- AdamW

static llmq_adamw_tensor entry(uint64_t& at, int64_t n, int flags) {
    auto take = [&](int64_t bytes) { const uint64_t p = at; at += ((uint64_t)bytes + 31) & ~(uint64_t)15; return p; };
    const bool codes = flags & LLMQ_ADAMW_STATES_8BIT;
    llmq_adamw_tensor t{};
    t.n = n, t.flags = flags;
    t.w_bf16 = (void*)take(2 * n), t.w_f32 = (float*)take(4 * n), t.grad = (void*)take(flags & LLMQ_ADAMW_GRAD_F32 ? 4 * n : 2 * n);
    t.m = (void*)take(codes ? n : 4 * n), t.v = (void*)take(codes ? n : 4 * n);
    if (codes) t.m_scale = (uint8_t*)take((n + 127) / 128), t.v_scale = (uint8_t*)take((n + 127) / 128);
    return t;
}

static void check_table(const std::vector<llmq_adamw_tensor>& ts) {
    const size_t bytes = llmq_adamw_plan_bytes(ts.data(), (int64_t)ts.size());
    std::vector<uint8_t> plan(bytes);                        // exactly as large as asked for
    int64_t info[4];
    const int st = llmq_adamw_plan(ts.data(), (int64_t)ts.size(), plan.data(), plan.size(), info);
    CHECK(st == LLMQ_OK && info[0] == (int64_t)ts.size(), "status %d", st);
    if (st != LLMQ_OK) return;
    CHECK(llmq_adamw_plan(ts.data(), (int64_t)ts.size(), plan.data(), plan.size() - 1, info) == LLMQ_ERR_WORKSPACE, "a plan that is too small");
    CHECK(bytes == adamw_table(info[0]) + (size_t)info[1] * sizeof(AdamWPiece), "%zu bytes for %lld pieces", bytes, (long long)info[1]);
    std::vector<int64_t> next(ts.size(), 0);
    for (int64_t p = 0; p < info[1]; ++p) {
        AdamWPiece piece;
        memcpy(&piece, plan.data() + adamw_table(info[0]) + (size_t)p * sizeof(piece), sizeof(piece));
        CHECK(piece.tensor >= 0 && piece.tensor < (int)ts.size() && piece.piece == next[piece.tensor], "piece %lld: %d of tensor %d", (long long)p, piece.piece, piece.tensor);
        if (piece.tensor >= 0 && piece.tensor < (int)ts.size()) ++next[piece.tensor];
    }
    for (size_t i = 0; i < ts.size(); ++i) {
        AdamWTensor t;
        memcpy(&t, plan.data() + i * sizeof(t), sizeof(t));
        CHECK(t.n == ts[i].n && t.w == ts[i].w_bf16 && t.m == ts[i].m && t.v_scale == ts[i].v_scale && t.flags == ts[i].flags, "tensor %zu", i);
        CHECK(next[i] == (t.n + kAdamPiece - 1) / kAdamPiece, "tensor %zu: %lld pieces", i, (long long)next[i]);
    }
}

// Overlaps by a comparison of all pairs
static bool overlap(const std::vector<llmq_adamw_tensor>& ts) {
    struct Range { uintptr_t first, end; bool written; };
    std::vector<Range> r;
    for (const llmq_adamw_tensor& t : ts) {
        const bool codes = t.flags & LLMQ_ADAMW_STATES_8BIT;
        auto add = [&](const void* p, int64_t bytes, bool written) { if (p) r.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written}); };
        add(t.w_bf16, 2 * t.n, true), add(t.w_f32, 4 * t.n, true), add(t.grad, (t.flags & LLMQ_ADAMW_GRAD_F32 ? 4 : 2) * t.n, false), add(t.m, (codes ? 1 : 4) * t.n, true), add(t.v, (codes ? 1 : 4) * t.n, true);
        if (codes) add(t.m_scale, (t.n + 127) / 128, true), add(t.v_scale, (t.n + 127) / 128, true);
    }
    for (size_t i = 0; i < r.size(); ++i)
        for (size_t j = 0; j < i; ++j)
            if ((r[i].written || r[j].written) && r[i].first < r[j].end && r[j].first < r[i].end) return true;
    return false;
}

int main() {
    std::mt19937_64 rng(5);
    auto spread = [&](double low, double high) { return (int64_t)(low * pow(high / low, std::uniform_real_distribution<double>(0, 1)(rng))); };
    // contractions of all kinds, multiples of 128 (where strips are cut) and others
    for (int i = 0; i < 3000; ++i) check_blocks(spread(1, 20000), spread(1, 20000), spread(1, 12000), i & 1, i & 2);
    for (int i = 0; i < 1500; ++i) check_blocks(128 * (int64_t)(1 + rng() % 150), 128 * (int64_t)(1 + rng() % 150), 128 * (int64_t)(1 + rng() % 96), i & 1, i & 2);
    for (int i = 0; i < 500; ++i) check_blocks(spread(1, 2e9), spread(1, 1000), spread(1, 5e6), false, false), check_blocks(spread(1, 1000), spread(1, 2e9), spread(1, 5e6), false, false);
    CHECK(g_strips > 20 && g_few > 100 && g_mini > 50 && g_generic > 50 && g_guarded > 100, "strips %d few %d mini %d generic %d guarded %d", g_strips, g_few, g_mini, g_generic, g_guarded);
    // forced strips, as the GPU tests use them
    for (const char* how : {"r128", "r384", "c128", "c640"}) {
        setenv("LLMQ_BLOCKS_STRIP", how, 1);
        for (int i = 0; i < 100; ++i) check_blocks(128 * spread(1, 30), 128 * spread(1, 30), 128 * spread(1, 30), false, false);
    }
    unsetenv("LLMQ_BLOCKS_STRIP");
    for (int64_t rows : {1, 15, 16, 127, 128, 129, 300, 1000}) for (int64_t T : {1, 127, 128, 129, 1000}) check_places(rows, T);
    // what the generic kernel is given: within the grid's dimensions, refused behind them
    CHECK(((1ll << 21) - 1 + 31) / 32 <= 65536 && ((1ll << 28) - 1 + 31) / 32 <= (int64_t)kMaxWorkgroups, "the generic kernel's grid");

    for (int i = 0; i < 300; ++i) {
        uint64_t at = 4096;
        std::vector<llmq_adamw_tensor> ts;
        for (int k = 1 + (int)(rng() % 12); k > 0; --k) ts.push_back(entry(at, spread(1, 20000), (int)(rng() & 7)));
        check_table(ts);
        // one array moved to a random place near another, of its own tensor or the next
        llmq_adamw_tensor &a = ts[rng() % ts.size()], &b = ts[rng() % ts.size()];
        const uintptr_t where = ((uintptr_t)(rng() & 1 ? a.m : a.grad) & ~(uintptr_t)15) + 16 * (rng() % 64) - (rng() & 1 ? 2 * (uintptr_t)b.n & ~(uintptr_t)15 : 0);
        if (where >= ((uintptr_t)1 << 40)) continue;         // (below zero)
        if (rng() & 1) b.v = (void*)where; else b.grad = (void*)where;
        std::vector<uint8_t> plan(llmq_adamw_plan_bytes(ts.data(), (int64_t)ts.size()));
        int64_t info[4];
        const int st = llmq_adamw_plan(ts.data(), (int64_t)ts.size(), plan.data(), plan.size(), info);
        CHECK(st == (overlap(ts) ? LLMQ_ERR_VALUE : LLMQ_OK), "status %d, overlap %d", st, (int)overlap(ts));
    }
    // the largest tensors are refused or counted, not overflown
    {
        uint64_t at = 4096;
        std::vector<llmq_adamw_tensor> ts(3, entry(at, 100, 0));
        int64_t pieces = 0;
        for (llmq_adamw_tensor& t : ts) t.n = kMaxElems - 1;
        CHECK(check_adamw(ts.data(), 1, pieces) == LLMQ_OK && pieces == (1ll << 30), "%lld pieces", (long long)pieces);
        CHECK(check_adamw(ts.data(), 3, pieces) == LLMQ_ERR_SHAPE && llmq_adamw_plan_bytes(ts.data(), 3) == 0, "more pieces than a launch counts");
        ts[0].n = kMaxElems;
        CHECK(check_adamw(ts.data(), 1, pieces) == LLMQ_ERR_SHAPE, "too many elements");
    }
    uint32_t words[LLMQ_ADAMW_HYPER_WORDS];
    CHECK(llmq_adamw_hyper(INT64_MAX, 1e-3, 0.999999, 0.9999999, 1e-8, 0.1, ~0ull, words) == LLMQ_OK, "a late step");
    if (g_fail) { printf("%d failures\n", g_fail); return 1; }
    printf("operators driver ok\n");
    return 0;
}
