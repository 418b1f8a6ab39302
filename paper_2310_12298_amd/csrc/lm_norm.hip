// Layer norm, forward and backward, for gfx950.
//
// Both directions are bound by HBM: two elements moved per element forward, three backward.
// A row is read once and stays in registers between the statistics and the result, held by
// one wave (short rows: no barrier at all) or by the whole workgroup. Element c of a row
// belongs to the lane that owns its 16-byte piece, so every load and store of a wave is
// 1 KB of consecutive bytes.
//
// The backward pass also sums over the rows, for the gain's and the bias's gradient. Each
// workgroup takes every grid-th group of rows and keeps its columns' two sums in registers
// over all of them; the sums go to the workspace once per workgroup, and a second launch
// adds them column by column in a fixed order (no atomics: the same bits every time).
//
// Measured, 16384 x 4096 bf16: forward 58 us (4.6 TB/s of what it has to move; a large copy
// reaches 5.0-5.15), backward 86 us (4.7 TB/s), the second launch 6 us. 5003 x 1999 fp32
// (rows at odd addresses): 17.3, 27.5 and 5.7 us (4.6 and 4.4 TB/s).
#include "lm_common.hpp"

namespace jorge_lm {
namespace {

// Sum over the lanes that share a row: a wave, or the workgroup of WAVES waves through LDS.
// `red` alternates between two halves, so one barrier per sum is enough.
template <int WAVES>
struct RowSum {
    float* red;  // 2 x WAVES x 2 floats
    int turn = 0;
    __device__ __forceinline__ void two(float& a, float& b) {
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (WAVES > 1) {
            float* const r = red + turn * 2 * WAVES;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) {
                r[2 * (threadIdx.x >> 6)] = a;
                r[2 * (threadIdx.x >> 6) + 1] = b;
            }
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                a += r[2 * w];
                b += r[2 * w + 1];
            }
        }
    }
    __device__ __forceinline__ float one(float a) {
        float b = 0.0f;
        two(a, b);
        return a;
    }
};

// WAVES waves share a row (a workgroup of max(4, WAVES) waves takes 4 / WAVES rows at a
// time); ITEMS 16-byte pieces per lane.
template <typename T, typename P, int WAVES, int ITEMS>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void norm_forward_kernel(
    const T* x, int64_t ldx, const P* __restrict__ weight, const P* __restrict__ bias, T* y, int64_t ldy,
    float* __restrict__ mean_out, float* __restrict__ rstd_out, int64_t rows, int cols, float eps) {
    constexpr int N = Wide<T>::N, TEAMS = WAVES > 4 ? 1 : 4 / WAVES, LANES = WAVES * 64;
    __shared__ float red[TEAMS * 4 * WAVES];
    const int team = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * TEAMS + team;
    static_assert(WAVES == 1 || TEAMS == 1, "a barrier is for a whole workgroup");
    if (TEAMS > 1 && row >= rows) return;
    const T* const xr = x + row * ldx;
    typename Wide<T>::V in[ITEMS];
    load_row<LANES>(xr, cols, lane, in);
    float v[ITEMS][N];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            v[i][e] = (float)in[i][e];
            sum += v[i][e];
        }
    RowSum<WAVES> rs{red};
    const float n = (float)cols, mean = rs.one(sum) / n;
    // Squares of the differences, from the registers: no cancellation however far the mean is from zero.
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int left = cols - (i * LANES + lane) * N;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            v[i][e] = v[i][e] - mean;
            sq += e < left ? v[i][e] * v[i][e] : 0.0f;
        }
    }
    const float rstd = 1.0f / sqrtf(rs.one(sq) / n + eps);
    if (mean_out && lane == 0) {
        mean_out[row] = mean;
        rstd_out[row] = rstd;
    }
    T* const yr = y + row * ldy;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * LANES + lane) * N, left = cols - c;
        if (left <= 0) break;
        float w[N], b[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            w[e] = 1.0f;
            b[e] = 0.0f;
        }
        if (weight) load_param<N>(weight + c, left, w);
        if (bias) load_param<N>(bias + c, left, b);
#pragma unroll
        for (int e = 0; e < N; ++e) v[i][e] = v[i][e] * rstd * w[e] + b[e];
        store_wide(yr + c, left, v[i]);
    }
}

// partial: [gridDim.x][2][cols] sums of dy xhat and of dy (SUMS).
template <typename T, typename P, int WAVES, int ITEMS, bool SUMS>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void norm_backward_kernel(
    const T* dy, int64_t lddy, const T* __restrict__ x, int64_t ldx, const float* __restrict__ mean,
    const float* __restrict__ rstd, const P* __restrict__ weight, T* dx, int64_t lddx,
    float* __restrict__ partial, int64_t rows, int cols) {
    constexpr int N = Wide<T>::N, TEAMS = WAVES > 4 ? 1 : 4 / WAVES, LANES = WAVES * 64;
    static_assert(WAVES == 1 || TEAMS == 1, "a barrier is for a whole workgroup");
    __shared__ float red[4 * WAVES];
    const int team = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    // The gain stays in registers where they reach; the widest rows read it again for every row.
    constexpr bool HOLD = ITEMS * N < 32;
    float w[HOLD ? ITEMS : 1][N], sw[SUMS ? ITEMS : 1][N], sb[SUMS ? ITEMS : 1][N];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * LANES + lane) * N;
#pragma unroll
        for (int e = 0; e < N; ++e)
            if constexpr (HOLD) w[i][e] = 1.0f;
        if constexpr (HOLD)
            if (weight) load_param<N>(weight + c, cols - c, w[i]);
        if constexpr (SUMS)
#pragma unroll
            for (int e = 0; e < N; ++e) sw[i][e] = sb[i][e] = 0.0f;
    }
    const float n = (float)cols;
    RowSum<WAVES> rs{red};
    const int64_t step = (int64_t)gridDim.x * TEAMS;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < rows; row += step) {
        const float mu = mean[row], r = rstd[row];
        typename Wide<T>::V xi[ITEMS], di[ITEMS];
        load_row<LANES>(x + row * ldx, cols, lane, xi);
        load_row<LANES>(dy + row * lddy, cols, lane, di);
        float gx[ITEMS][N], xv[ITEMS][N];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if constexpr (!HOLD) {
                const int c = (i * LANES + lane) * N;
#pragma unroll
                for (int e = 0; e < N; ++e) w[0][e] = 1.0f;
                if (weight) load_param<N>(weight + c, cols - c, w[0]);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                // Past the row's end dy is 0, and so is all that its xhat enters.
                const float xh = ((float)xi[i][e] - mu) * r, d = (float)di[i][e];
                if constexpr (SUMS) {
                    sw[i][e] += d * xh;
                    sb[i][e] += d;
                }
                xv[i][e] = xh;
                gx[i][e] = d * w[HOLD ? i : 0][e];
                s1 += gx[i][e];
                s2 += gx[i][e] * xh;
            }
        }
        rs.two(s1, s2);
        const float m1 = s1 / n, m2 = s2 / n;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * LANES + lane) * N;
            if (cols - c <= 0) break;
            float o[N];
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = r * (gx[i][e] - m1 - xv[i][e] * m2);
            store_wide(dx + row * lddx + c, cols - c, o);
        }
    }
    if constexpr (SUMS) {
        float* const out = partial + (int64_t)blockIdx.x * 2 * cols;
        if constexpr (TEAMS > 1) {
            // The waves' sums of the same columns, added in wave order.
            __shared__ float lds[TEAMS][LANES * N];
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int which = 0; which < 2; ++which) {
                    __syncthreads();
#pragma unroll
                    for (int e = 0; e < N; ++e) lds[team][e * LANES + lane] = which ? sb[i][e] : sw[i][e];
                    __syncthreads();
                    for (int k = threadIdx.x; k < LANES * N; k += TEAMS * LANES) {
                        const int c = i * LANES * N + (k % LANES) * N + k / LANES;
                        float t = 0.0f;
#pragma unroll
                        for (int m = 0; m < TEAMS; ++m) t += lds[m][k];
                        if (c < cols) out[which * cols + c] = t;
                    }
                }
        } else {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int c = (i * LANES + lane) * N;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (c + e < cols) {
                        out[c + e] = sw[i][e];
                        out[cols + c + e] = sb[i][e];
                    }
            }
        }
    }
}

// Sums the partial sums of 64 columns of one of the two gradients: 16 waves take every 16th
// partial each, in ascending order, and their sums are added in wave order.
constexpr int kSumWaves = 16;
template <typename P>
__global__ __launch_bounds__(kSumWaves * 64) void norm_sums_kernel(const float* __restrict__ partial, int parts,
                                                                   int cols, P* __restrict__ dweight,
                                                                   P* __restrict__ dbias) {
    __shared__ float lds[kSumWaves][64];
    P* const out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const float* const p = partial + (int64_t)blockIdx.y * cols + min(c, cols - 1);
    float s[4] = {};
    int k = wave;
    for (; k + 3 * kSumWaves < parts; k += 4 * kSumWaves)
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] += p[(int64_t)(k + u * kSumWaves) * 2 * cols];
    for (; k < parts; k += kSumWaves) s[0] += p[(int64_t)k * 2 * cols];
    lds[wave][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (wave == 0 && c < cols) {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < kSumWaves; ++w) t += lds[w][lane];
        out[c] = (P)t;
    }
}

// Waves per row and pieces per lane for rows of `cols` elements: the fewest waves whose lanes hold
// the row in at most four pieces.
struct Split {
    int waves, items;
};
Split split_of(int64_t cols, int wide) {
    const int64_t pieces = ceil_div(cols, wide);
    if (pieces <= 64) return {1, 1};
    if (pieces <= 128) return {1, 2};
    if (pieces <= 256) return {1, 4};
    if (pieces <= 512) return {4, 2};
    if (pieces <= 1024) return {4, 4};
    if (pieces <= 2048) return {8, 4};
    return {8, 8};
}

// Workgroups of the backward pass: each leaves 2 * cols partial sums, so there are no more than it
// takes to keep the memory busy: three per CU hold six rows' worth of loads (25 MB of sums for 4096
// columns, beside 403 MB of rows). Rows above 8192 take a workgroup of eight waves, one per CU.
constexpr int kGroups = 768;
int groups_of(int64_t rows, int64_t cols, int32_t dtype) {
    const Split s = split_of(cols, dtype == JORGE_BF16 ? 8 : 4);
    const int64_t teams = s.waves == 1 ? 4 : 1;
    const int64_t most = s.waves == 8 ? 256 : kGroups;
    const int64_t want = ceil_div(rows, teams);
    return (int)(want < most ? want : most);
}

template <typename F>
void with_split(Split s, F&& f) {
    if (s.waves == 1) {
        if (s.items == 1) f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
        else if (s.items == 2) f(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
        else f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
    } else if (s.waves == 4) {
        if (s.items == 2) f(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
        else f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
    } else {
        if (s.items == 4) f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
        else f(std::integral_constant<int, 8>(), std::integral_constant<int, 8>());
    }
}

template <typename T, typename P>
void forward(const void* x, int64_t ldx, const void* weight, const void* bias, void* y, int64_t ldy, float* mean,
             float* rstd, int64_t rows, int cols, float eps, hipStream_t stream) {
    const Split s = split_of(cols, Wide<T>::N);
    with_split(s, [&](auto W, auto I) {
        constexpr int waves = decltype(W)::value, items = decltype(I)::value, teams = waves == 1 ? 4 : 1;
        // Eight pieces per lane are for fp32: bf16 rows end at JORGE_NORM_MAX_COLS before.
        if constexpr (items < 8 || Wide<T>::N == 4)
            // A grid holds fewer than 2^32 threads.
            for (int64_t r0 = 0; r0 < rows; r0 += kRowsPerLaunch) {
                const int64_t n = rows - r0 < kRowsPerLaunch ? rows - r0 : kRowsPerLaunch;
                norm_forward_kernel<T, P, waves, items>
                    <<<dim3((unsigned)ceil_div(n, teams)), dim3(waves > 4 ? waves * 64 : 256), 0, stream>>>(
                        (const T*)x + r0 * ldx, ldx, (const P*)weight, (const P*)bias, (T*)y + r0 * ldy, ldy,
                        mean ? mean + r0 : nullptr, rstd ? rstd + r0 : nullptr, n, cols, eps);
            }
    });
}

template <typename T, typename P>
void backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd,
              const void* weight, void* dx, int64_t lddx, float* partial, int groups, int64_t rows, int cols,
              hipStream_t stream) {
    const Split s = split_of(cols, Wide<T>::N);
    with_split(s, [&](auto W, auto I) {
        constexpr int waves = decltype(W)::value, items = decltype(I)::value;
        if constexpr (items < 8 || Wide<T>::N == 4) {
            const dim3 grid(groups), block(waves > 4 ? waves * 64 : 256);
            if (partial)
                norm_backward_kernel<T, P, waves, items, true><<<grid, block, 0, stream>>>(
                    (const T*)dy, lddy, (const T*)x, ldx, mean, rstd, (const P*)weight, (T*)dx, lddx, partial, rows,
                    cols);
            else
                norm_backward_kernel<T, P, waves, items, false><<<grid, block, 0, stream>>>(
                    (const T*)dy, lddy, (const T*)x, ldx, mean, rstd, (const P*)weight, (T*)dx, lddx, partial, rows,
                    cols);
        }
    });
}

// What every call of the pass checks.
jorge_status check(int64_t rows, int64_t cols, int32_t dtype, int32_t param_dtype, const void* weight,
                   const void* bias) {
    if (!known_dtype(dtype) || !known_dtype(param_dtype)) return bad("layer norm: unknown element type");
    if (rows < 0 || cols < 1) return bad("layer norm: rows >= 0 and cols >= 1 are needed");
    if (cols > JORGE_NORM_MAX_COLS) return refuse(JORGE_ERR_UNSUPPORTED, "layer norm: cols above JORGE_NORM_MAX_COLS");
    if (rows > (int64_t)1 << 31) return refuse(JORGE_ERR_UNSUPPORTED, "layer norm: more than 2^31 rows");
    const int64_t pe = dtype_bytes(param_dtype);
    if (!aligned(weight, pe) || !aligned(bias, pe)) return bad("layer norm: a parameter is not aligned to its element");
    return JORGE_OK;
}

}  // namespace
}  // namespace jorge_lm

using namespace jorge_lm;

extern "C" {

jorge_status jorge_layernorm_forward(const void* x, int64_t ldx, int32_t dtype, const void* weight, const void* bias,
                                     int32_t param_dtype, void* y, int64_t ldy, float* mean, float* rstd, int64_t rows,
                                     int64_t cols, double eps, void* hip_stream) {
    jorge_status st = check(rows, cols, dtype, param_dtype, weight, bias);
    if (st != JORGE_OK) return st;
    if (!(eps >= 0.0) || eps > 1e30) return bad("layer norm: eps must be finite and not negative");
    if (!mean != !rstd) return bad("layer norm: mean and rstd are written both or neither");
    if (ldx < cols || ldy < cols) return bad("layer norm: a row stride is below cols");
    if (rows == 0) return JORGE_OK;
    if (!x || !y) return bad("layer norm: x and y are needed");
    const int64_t e = dtype_bytes(dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(mean, 4) || !aligned(rstd, 4))
        return bad("layer norm: a pointer is not aligned to its element");
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    const auto go = [&](auto t, auto p) {
        forward<decltype(t), decltype(p)>(x, ldx, weight, bias, y, ldy, mean, rstd, rows, (int)cols, (float)eps, s);
    };
    if (dtype == JORGE_F32) param_dtype == JORGE_F32 ? go(float(), float()) : go(float(), bf16());
    else param_dtype == JORGE_F32 ? go(bf16(), float()) : go(bf16(), bf16());
    return launched("layer norm");
}

jorge_status jorge_layernorm_workspace(int64_t rows, int64_t cols, int64_t* bytes) {
    if (!bytes) return bad("layer norm: bytes is needed");
    const jorge_status st = check(rows, cols, JORGE_F32, JORGE_F32, nullptr, nullptr);
    if (st != JORGE_OK) return st;
    // The larger of the two element types' needs.
    const int64_t a = groups_of(rows, cols, JORGE_F32), b = groups_of(rows, cols, JORGE_BF16);
    *bytes = round_up((a > b ? a : b) * 2 * cols * (int64_t)sizeof(float), kAlign);
    return JORGE_OK;
}

jorge_status jorge_layernorm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int32_t dtype,
                                      const float* mean, const float* rstd, const void* weight, int32_t param_dtype,
                                      void* dx, int64_t lddx, void* dweight, void* dbias, int64_t rows, int64_t cols,
                                      void* workspace, int64_t workspace_bytes, void* hip_stream) {
    jorge_status st = check(rows, cols, dtype, param_dtype, weight, nullptr);
    if (st != JORGE_OK) return st;
    if (ldx < cols || lddy < cols || lddx < cols) return bad("layer norm: a row stride is below cols");
    const int64_t e = dtype_bytes(dtype), pe = dtype_bytes(param_dtype);
    if (rows > 0 && (!dy || !x || !mean || !rstd || !dx)) return bad("layer norm: dy, x, mean, rstd and dx are needed");
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(dx, e) || !aligned(mean, 4) || !aligned(rstd, 4) ||
        !aligned(dweight, pe) || !aligned(dbias, pe))
        return bad("layer norm: a pointer is not aligned to its element");
    const bool sums = dweight || dbias;
    const int groups = groups_of(rows, cols, dtype);
    if (sums && rows > 0) {
        if (!workspace || !aligned(workspace, kAlign))
            return bad("layer norm: a workspace aligned to 256 bytes is needed");
        if (workspace_bytes < round_up((int64_t)groups * 2 * cols * 4, kAlign))
            return bad("layer norm: the workspace is too small");
    }
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    float* const partial = sums ? (float*)workspace : nullptr;
    if (rows > 0) {
        const auto go = [&](auto t, auto p) {
            backward<decltype(t), decltype(p)>(dy, lddy, x, ldx, mean, rstd, weight, dx, lddx, partial, groups, rows,
                                               (int)cols, s);
        };
        if (dtype == JORGE_F32) param_dtype == JORGE_F32 ? go(float(), float()) : go(float(), bf16());
        else param_dtype == JORGE_F32 ? go(bf16(), float()) : go(bf16(), bf16());
        if ((st = launched("layer norm")) != JORGE_OK) return st;
    }
    if (sums) {
        const dim3 grid((unsigned)ceil_div(cols, 64), 2), block(kSumWaves * 64);
        if (param_dtype == JORGE_F32)
            norm_sums_kernel<float><<<grid, block, 0, s>>>(partial, groups, (int)cols, (float*)dweight, (float*)dbias);
        else
            norm_sums_kernel<bf16><<<grid, block, 0, s>>>(partial, groups, (int)cols, (bf16*)dweight, (bf16*)dbias);
        return launched("layer norm");
    }
    return JORGE_OK;
}

}  // extern "C"
