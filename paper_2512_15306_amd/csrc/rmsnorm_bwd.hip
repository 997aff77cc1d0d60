// Gradient of RMSNorm and of the residual addition in front of it (llmq_rmsnorm_bwd).
//
//   n = res' rstd,  g = dy w;   dx = dres + rstd (g - n mean(g n)),   dw[c] = sum over the rows of dy n
//
// HBM-bound: dy, res' and dres are read once, dx is written once (8 bytes an element).  A workgroup walks over rows: a row's lanes hold it in registers between the
// mean and the result, and the sums of dw of their columns from row to row in binary32, so that they leave the workgroup once, as a row of the workspace.  A second
// kernel adds those rows in an order that the sizes decide.
//
// 8192 x 5120 with dres (336 MB): 70.9 us, of them 4 for the second kernel, where a large copy's rate is 57; 1777 x 2730 17.5, 256 x 2048 6.3, half of it the second launch.  Two workgroups of 512 lanes
// a CU hide each other's waits: asking for the next row while one is worked on takes the registers of the second (ragged 17.9 -> 25.9 us, large 72.7 -> 73.8).
#include "api_checks.h"
#include "rmsnorm.h"

namespace llmq {

constexpr int kBwdThreads = 512, kBwdWaves = kBwdThreads / kWave;
constexpr int kBwdMaxBlocks = 512;              // workgroups: rows of sums in the workspace
constexpr int64_t kBwdMaxC = 16384;             // widest row that is kept in registers
constexpr int kBwdChunks = 64;                  // rows of sums of wider ones

struct NormBwd {
    // dx may be dy or dres: no lane stores of a row before the row's loads have been requested
    const uint16_t *dy, *dres, *res, *w;
    const float* rstd;
    uint16_t* dx;
    float* dw_partial;                          // [workgroups][C], or NULL
    unsigned* amax_partial;                     // a word for each workgroup, or NULL
    int64_t M;
    int C;
};

// Sum over the wave in all lanes, in an order that is the same for all of them
__device__ inline float wave_sum_all(float v) {
    auto moved = [](float x, auto ctrl) { return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, false)); };
    v += moved(v, std::integral_constant<int, 0xB1>{});          // quad_perm [1,0,3,2]
    v += moved(v, std::integral_constant<int, 0x4E>{});          // quad_perm [2,3,0,1]
    v += moved(v, std::integral_constant<int, 0x141>{});         // row_half_mirror
    v += moved(v, std::integral_constant<int, 0x140>{});         // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <bool EDGE>
__device__ inline v4u bwd_load(const uint16_t* row, int idx, int C) {
    if constexpr (!EDGE) return __builtin_nontemporal_load(reinterpret_cast<const v4u*>(row) + idx);
    else return load8_upto(row + 8 * idx, 8 * idx, C - 8 * idx);
}

// LANES lanes to a row, VPL vectors of eight elements to a lane.
template <int LANES, int VPL, bool EDGE, bool DRES>
__global__ __launch_bounds__(kBwdThreads) void rmsnorm_bwd_kernel(const NormBwd a) {
    constexpr int kGroups = kBwdThreads / LANES, kWavesOfRow = LANES / kWave;
    __shared__ float s_sum[2][kBwdWaves];
    __shared__ __attribute__((aligned(16))) float s_dw[kGroups > 1 ? LANES * VPL * 8 : 4];
    __shared__ unsigned s_part[kBwdWaves];
    const int group = threadIdx.x / LANES, t = threadIdx.x % LANES, wave = threadIdx.x / kWave, C = a.C, nvec = EDGE ? (C + 7) / 8 : C / 8;
    v4u wv[VPL];
    float dw[VPL][8];
#pragma unroll
    for (int k = 0; k < VPL; ++k) {
        const int idx = k * LANES + t;
        wv[k] = v4u{0, 0, 0, 0};
        if (idx < nvec) wv[k] = EDGE ? load8_upto(a.w + 8 * idx, 8 * idx, C - 8 * idx) : reinterpret_cast<const v4u*>(a.w)[idx];
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[k][e] = 0.0f;
    }
    unsigned mag = 0;
    int parity = 0;
    // (the same number of trips for the whole workgroup)
    for (int64_t first = (int64_t)blockIdx.x * kGroups; first < a.M; first += (int64_t)gridDim.x * kGroups, parity ^= 1) {
        const int64_t row = first + group;
        const bool there = row < a.M;
        const int64_t at = (there ? row : 0) * C;
        v4u dy[VPL], res[VPL], dres[VPL];
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int idx = k * LANES + t;
            dy[k] = res[k] = dres[k] = v4u{0, 0, 0, 0};
            if (there && idx < nvec) {
                dy[k] = bwd_load<EDGE>(a.dy + at, idx, C);
                res[k] = bwd_load<EDGE>(a.res + at, idx, C);
                if constexpr (DRES) dres[k] = bwd_load<EDGE>(a.dres + at, idx, C);
            }
        }
        const float rstd = there ? a.rstd[row] : 0.0f;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < VPL; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float n0 = rn_lo(res[k][j]) * rstd, n1 = rn_hi(res[k][j]) * rstd, y0 = rn_lo(dy[k][j]), y1 = rn_hi(dy[k][j]);
                sum = __builtin_fmaf(y0 * rn_lo(wv[k][j]), n0, sum);
                sum = __builtin_fmaf(y1 * rn_hi(wv[k][j]), n1, sum);
                dw[k][2 * j] = __builtin_fmaf(y0, n0, dw[k][2 * j]);
                dw[k][2 * j + 1] = __builtin_fmaf(y1, n1, dw[k][2 * j + 1]);
            }
        sum = wave_sum_all(sum);
        if constexpr (kWavesOfRow > 1) {
            if ((threadIdx.x & (kWave - 1)) == 0) s_sum[parity][wave] = sum;
            __syncthreads();
            sum = s_sum[parity][group * kWavesOfRow];
#pragma unroll
            for (int i = 1; i < kWavesOfRow; ++i) sum += s_sum[parity][group * kWavesOfRow + i];
        }
        const float mean = sum / (float)C;
        if (!there) continue;
        // (opaque here, or the compiler keeps what it has computed of every element over the barrier: 186 registers instead of 146 with three vectors)
#pragma unroll
        for (int k = 0; k < VPL; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(dy[k][j]), "+v"(res[k][j]), "+v"(wv[k][j]));
#pragma unroll
        for (int k = 0; k < VPL; ++k) {
            const int idx = k * LANES + t;
            if (idx >= nvec) continue;
            v4u out;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float d[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float n = (h ? rn_hi(res[k][j]) : rn_lo(res[k][j])) * rstd, g = (h ? rn_hi(dy[k][j]) : rn_lo(dy[k][j])) * (h ? rn_hi(wv[k][j]) : rn_lo(wv[k][j]));
                    const float inner = __builtin_fmaf(-n, mean, g);
                    d[h] = DRES ? __builtin_fmaf(rstd, inner, h ? rn_hi(dres[k][j]) : rn_lo(dres[k][j])) : rstd * inner;
                }
                out[j] = rn_pack(d[0], d[1]);
            }
            if (EDGE && idx == nvec - 1) out = keep_upto(out, C % 8);
#pragma unroll
            for (int j = 0; j < 4; ++j) mag = pk_max_mag(mag, out[j]);
            if constexpr (EDGE) store8_upto(a.dx + at + 8 * idx, out, C - 8 * idx);
            else *reinterpret_cast<v4u*>(a.dx + at + 8 * idx) = out;
        }
    }
    if (a.amax_partial) {
        mag = block_max_u32<kBwdThreads>((mag & 0xFFFFu) > (mag >> 16) ? mag & 0xFFFFu : mag >> 16, s_part);
        if (threadIdx.x == 0) a.amax_partial[blockIdx.x] = mag;
    }
    if (!a.dw_partial) return;
    float* const out = a.dw_partial + (int64_t)blockIdx.x * C;
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int k = 0; k < VPL; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (8 * (k * LANES + t) + e < C) out[8 * (k * LANES + t) + e] = dw[k][e];
    } else {
        // the groups one after the other
        for (int g = 0; g < kGroups; ++g) {
            if (g == group) {
#pragma unroll
                for (int k = 0; k < VPL; ++k) {
                    v4f* p = reinterpret_cast<v4f*>(&s_dw[8 * (k * LANES + t)]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        v4f v = {dw[k][4 * h], dw[k][4 * h + 1], dw[k][4 * h + 2], dw[k][4 * h + 3]};
                        if (g > 0) {
                            const v4f before = p[h];
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = before[e] + v[e];
                        }
                        p[h] = v;
                    }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < C; c += kBwdThreads) out[c] = s_dw[c];
    }
}

// Rows of more than 16384 elements, element by element; the row is read a second time for the result.  A workgroup takes a row.
template <bool DRES>
__global__ __launch_bounds__(kBwdThreads) void rmsnorm_bwd_wide_kernel(const NormBwd a) {
    __shared__ float s_sum[2][kBwdWaves];
    __shared__ unsigned s_part[kBwdWaves];
    unsigned mag = 0;
    int parity = 0;
    auto value = [](uint16_t v) { return __uint_as_float((unsigned)v << 16); };
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x, parity ^= 1) {
        const int64_t at = row * a.C;
        const float rstd = a.rstd[row];
        float sum = 0.0f;
        for (int c = threadIdx.x; c < a.C; c += kBwdThreads) sum = __builtin_fmaf(value(a.dy[at + c]) * value(a.w[c]), value(a.res[at + c]) * rstd, sum);
        sum = wave_sum_all(sum);
        if ((threadIdx.x & (kWave - 1)) == 0) s_sum[parity][threadIdx.x / kWave] = sum;
        __syncthreads();
        sum = s_sum[parity][0];
#pragma unroll
        for (int i = 1; i < kBwdWaves; ++i) sum += s_sum[parity][i];
        const float mean = sum / (float)a.C;
        for (int c = threadIdx.x; c < a.C; c += kBwdThreads) {
            const float inner = __builtin_fmaf(-(value(a.res[at + c]) * rstd), mean, value(a.dy[at + c]) * value(a.w[c]));
            const unsigned o = rn_pack(DRES ? __builtin_fmaf(rstd, inner, value(a.dres[at + c])) : rstd * inner, 0.0f) & 0xFFFFu;
            a.dx[at + c] = (uint16_t)o;
            mag = pk_max_mag(mag, o);
        }
    }
    if (a.amax_partial) {
        mag = block_max_u32<kBwdThreads>(mag & 0xFFFFu, s_part);
        if (threadIdx.x == 0) a.amax_partial[blockIdx.x] = mag;
    }
}
// Their sums of dw: a lane takes a column of every kBwdChunks-th row.  In front of the kernel above, which may write over dy.
__global__ __launch_bounds__(kBwdThreads) void rmsnorm_bwd_wide_sums_kernel(const NormBwd a) {
    const int c = blockIdx.x * kBwdThreads + threadIdx.x;
    if (c >= a.C) return;
    float sum = 0.0f;
    for (int64_t row = blockIdx.y; row < a.M; row += gridDim.y)
        sum = __builtin_fmaf(__uint_as_float((unsigned)a.dy[row * a.C + c] << 16), __uint_as_float((unsigned)a.res[row * a.C + c] << 16) * a.rstd[row], sum);
    a.dw_partial[(int64_t)blockIdx.y * a.C + c] = sum;
}

// The rows of sums: a workgroup has 32 columns (a line) and 32 lanes to each, which take every 32nd row in turn and are then added pairwise: an order that the
// number of rows alone decides.  The last workgroup finds the absmax.
constexpr int kSumCols = 32, kSumRows = 32, kSumThreads = kSumCols * kSumRows;
__global__ __launch_bounds__(kSumThreads) void rmsnorm_bwd_final_kernel(const float* dw_partial, int rows, const unsigned* amax_partial, int words, int C, float* dw, int accumulate, float fmax,
                                                                       float* d_amax, float* d_scale) {
    __shared__ float s_sum[kSumRows][kSumCols + 1];
    __shared__ unsigned s_part[kSumThreads / kWave];
    if (blockIdx.x == gridDim.x - 1) {
        if (!amax_partial) return;
        unsigned m = 0;
        for (int i = threadIdx.x; i < words; i += kSumThreads) m = m > amax_partial[i] ? m : amax_partial[i];
        m = block_max_u32<kSumThreads>(m, s_part);
        if (threadIdx.x == 0) {
            const float amax = __uint_as_float(amax_bits_from_bf16_mag(m));
            *d_amax = amax;
            if (d_scale) *d_scale = scale_of_amax(amax, fmax);
        }
        return;
    }
    const int c = threadIdx.x % kSumCols, r = threadIdx.x / kSumCols, col = blockIdx.x * kSumCols + c;
    constexpr int kAtOnce = kBwdMaxBlocks / kSumRows;       // all of a lane's loads are on their way together
    static_assert(kBwdChunks <= kBwdMaxBlocks, "a lane takes every row of sums there may be");
    float v[kAtOnce], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) v[k] = col < C && r + kSumRows * k < rows ? dw_partial[(int64_t)(r + kSumRows * k) * C + col] : 0.0f;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) sum += v[k];
    s_sum[r][c] = sum;
#pragma unroll
    for (int step = kSumRows / 2; step >= 1; step /= 2) {
        __syncthreads();
        if (r < step) s_sum[r][c] += s_sum[r + step][c];
    }
    if (r == 0 && col < C) dw[col] = accumulate ? dw[col] + s_sum[0][c] : s_sum[0][c];
}

// Lanes to a row and workgroups of a launch, and rows of sums: functions of the sizes alone.
struct NormBwdGrid { int lanes, blocks, rows_of_sums; };
static NormBwdGrid norm_bwd_grid(int64_t M, int64_t C) {
    const int lanes = C > kBwdMaxC ? kBwdThreads : C <= 512 ? 64 : C <= 2048 && M >= 4096 ? 64 : C <= 8192 ? 256 : 512;
    const int64_t wanted = (M + kBwdThreads / lanes - 1) / (kBwdThreads / lanes);
    const int blocks = (int)(wanted < kBwdMaxBlocks ? wanted : kBwdMaxBlocks);
    return {lanes, blocks, C > kBwdMaxC ? (int)(M < kBwdChunks ? M : kBwdChunks) : blocks};
}

static int launch_norm_bwd(const NormBwd& a, const NormBwdGrid& g, float* dw, int accumulate, int fmt, float* d_amax, float* d_scale, hipStream_t stream) {
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(g.blocks), dim3(kBwdThreads), 0, stream, a); };
    if (a.C > kBwdMaxC) {
        if (a.dw_partial) hipLaunchKernelGGL(rmsnorm_bwd_wide_sums_kernel, dim3((unsigned)((a.C + kBwdThreads - 1) / kBwdThreads), g.rows_of_sums), dim3(kBwdThreads), 0, stream, a);
        if (a.dres) launch(rmsnorm_bwd_wide_kernel<true>); else launch(rmsnorm_bwd_wide_kernel<false>);
    } else {
        const bool edge = a.C % 8 != 0;
        auto of = [&](auto lanes, auto vpl) {
            constexpr int L = decltype(lanes)::value, V = decltype(vpl)::value;
            if (a.dres) edge ? launch(rmsnorm_bwd_kernel<L, V, true, true>) : launch(rmsnorm_bwd_kernel<L, V, false, true>);
            else edge ? launch(rmsnorm_bwd_kernel<L, V, true, false>) : launch(rmsnorm_bwd_kernel<L, V, false, false>);
        };
        typedef std::integral_constant<int, 64> L64;
        typedef std::integral_constant<int, 256> L256;
        typedef std::integral_constant<int, 512> L512;
        typedef std::integral_constant<int, 1> V1;
        typedef std::integral_constant<int, 2> V2;
        typedef std::integral_constant<int, 3> V3;
        typedef std::integral_constant<int, 4> V4;
        const int vectors = (int)((a.C + 8 * g.lanes - 1) / (8 * g.lanes));
        if (g.lanes == 64) vectors == 1 ? of(L64{}, V1{}) : vectors == 2 ? of(L64{}, V2{}) : of(L64{}, V4{});
        else if (g.lanes == 256) vectors == 1 ? of(L256{}, V1{}) : vectors == 2 ? of(L256{}, V2{}) : vectors == 3 ? of(L256{}, V3{}) : of(L256{}, V4{});
        else of(L512{}, V4{});
    }
    if (a.dw_partial || a.amax_partial) {
        const unsigned cols = a.dw_partial ? (unsigned)((a.C + kSumCols - 1) / kSumCols) : 0;
        hipLaunchKernelGGL(rmsnorm_bwd_final_kernel, dim3(cols + 1), dim3(kSumThreads), 0, stream, a.dw_partial, g.rows_of_sums, a.amax_partial, g.blocks, a.C, dw, accumulate, fp8_max(fmt), d_amax, d_scale);
    }
    return hipGetLastError() == hipSuccess ? LLMQ_OK : LLMQ_ERR_DEVICE;
}

}  // namespace llmq

namespace {

bool norm_bwd_shape_ok(int64_t M, int64_t C) { return dim_ok(M) && dim_ok(C) && C < ((int64_t)1 << 24) && M * C < kMaxElems; }

size_t sums_bytes(int64_t M, int64_t C) { return round256((size_t)llmq::norm_bwd_grid(M, C).rows_of_sums * (size_t)C * sizeof(float)); }

}  // namespace

extern "C" {

size_t llmq_rmsnorm_bwd_workspace_bytes(int64_t M, int64_t C) {
    if (!norm_bwd_shape_ok(M, C)) return 0;
    return sums_bytes(M, C) + (size_t)llmq::kBwdMaxBlocks * sizeof(unsigned);
}

int llmq_rmsnorm_bwd(const void* dy_bf16, const void* dres_bf16, const void* res_bf16, const void* w_bf16, const float* rstd, int64_t M, int64_t C, void* dx_bf16, float* dw, int accumulate, int fmt,
                     float* d_amax, float* d_scale, void* ws, size_t ws_bytes, void* stream) {
    if (!dy_bf16 || !res_bf16 || !w_bf16 || !rstd || !dx_bf16 || (d_scale && !d_amax) || ((dw || d_amax) && !ws)) return LLMQ_ERR_NULL;
    if (!norm_bwd_shape_ok(M, C)) return LLMQ_ERR_SHAPE;
    if (d_amax && !fmt_ok(fmt)) return LLMQ_ERR_FORMAT;
    if (!aligned(dy_bf16, 16) || !aligned(dres_bf16, 16) || !aligned(res_bf16, 16) || !aligned(w_bf16, 16) || !aligned(rstd, 4) || !aligned(dx_bf16, 16) || !aligned(dw, 4) || !aligned(d_amax, 4) ||
        !aligned(d_scale, 4) || !aligned(ws, 16))
        return LLMQ_ERR_ALIGN;
    if ((dw || d_amax) && ws_bytes < llmq_rmsnorm_bwd_workspace_bytes(M, C)) return LLMQ_ERR_WORKSPACE;
    llmq::NormBwd a{};
    a.dy = static_cast<const uint16_t*>(dy_bf16), a.dres = static_cast<const uint16_t*>(dres_bf16), a.res = static_cast<const uint16_t*>(res_bf16), a.w = static_cast<const uint16_t*>(w_bf16);
    a.rstd = rstd, a.dx = static_cast<uint16_t*>(dx_bf16), a.M = M, a.C = (int)C;
    a.dw_partial = dw ? static_cast<float*>(ws) : nullptr;
    a.amax_partial = d_amax ? reinterpret_cast<unsigned*>(static_cast<uint8_t*>(ws) + sums_bytes(M, C)) : nullptr;
    return llmq::launch_norm_bwd(a, llmq::norm_bwd_grid(M, C), dw, accumulate != 0, d_amax ? fmt : 0, d_amax, d_scale, static_cast<hipStream_t>(stream));
}

}  // extern "C"
