// What the operators that are made of matrix products share around the product itself (lm_loss_gemm.hpp): the copies
// that make an operand's rows K-contiguous, which tile a workgroup takes, and which tile and how many ranges of K a
// product takes.
#pragma once

#include "lm_common.hpp"
#include "lm_loss_gemm.hpp"

#include <algorithm>

namespace jorge_lm {
namespace {

constexpr int kPadK = 64;      // K of every product is a multiple of two stages

// ---------------------------------------------------------------- operands
// Copies of a matrix that the products read: `flat`, its rows padded with zeros to a multiple of 64, and `turned`, its
// transpose, padded alike with zeros, which also stand in for the rows that `targets` (if given) has no target for:
// what such a row holds must not reach a sum that it has no part in. Either may be null; the terms of a row follow one
// another.
struct Copies {
    const void* src;
    int64_t ld, rows;
    int cols, tiles_c;       // 64 x 64 tiles along the columns
    bf16 *flat, *turned;
    int64_t padded_f, padded_t;  // of one term of a row
    const int64_t* targets;
    int64_t vocab, ignore;
    int64_t tiles;           // of the whole job
};
constexpr int kCopyJobs = 3;
struct CopyJobs {
    Copies job[kCopyJobs];
};

// The next term of a split value, of which the terms before it have been subtracted. One that is infinite, or would be
// rounded to that, is its last term alone: the last term meets only the first one of the other operand, whose sign is the
// element's, while an infinite first term would meet the others' zeros and signs and make a NaN.
__device__ __forceinline__ bf16 term_of(float f, bool last) {
    return (bf16)(last || __builtin_fabsf(f) < 0x1.ffp127f ? f : 0.0f);  // from there on bfloat16 rounds to infinity
}
template <int TERMS>
__device__ __forceinline__ void store_terms(bf16* dst, int64_t plane, float (&f)[8]) {
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o[e] = term_of(f[e], t == TERMS - 1);
            f[e] -= (float)o[e];
        }
        *reinterpret_cast<bf16x8*>(dst + t * plane) = o;
    }
}

// One workgroup per 64 x 64 tile: read once, eight elements of a row per lane, and written both ways.
template <typename T, int TERMS>
__global__ __launch_bounds__(256) void copies_kernel(CopyJobs jobs) {
    __shared__ T tile[64][64 + 4 / sizeof(T)];  // the odd row length spreads a column over the banks
    int which = 0;
    int64_t g = blockIdx.x;
    while (which < kCopyJobs - 1 && g >= jobs.job[which].tiles) g -= jobs.job[which++].tiles;
    const Copies& j = jobs.job[which];
    const int64_t r0 = g / j.tiles_c * 64;
    const int c0 = (int)(g % j.tiles_c) * 64, part = (threadIdx.x & 7) * 8;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int y = (threadIdx.x >> 3) + 32 * k, c = c0 + part, left = j.cols - c;
        const int64_t r = r0 + y;
        float f[8] = {};
        bool live = r < j.rows;
        if (live) {
            typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
            const T* const p = (const T*)j.src + r * j.ld + c;
            if (left >= 8) {
                const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = (float)v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = e < left ? (float)p[e] : 0.0f;
            }
            if (j.targets) {
                const int64_t t = j.targets[r];
                live = t >= 0 && t < j.vocab && t != j.ignore;
            }
        }
        if (j.turned)
#pragma unroll
            for (int e = 0; e < 8; ++e) tile[y][part + e] = live ? (T)f[e] : (T)0.0f;
        if (j.flat && r < j.rows) store_terms<TERMS>(j.flat + r * TERMS * j.padded_f + c, j.padded_f, f);
    }
    if (!j.turned) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = (threadIdx.x >> 3) + 32 * k;
        if (c0 + c >= j.cols) continue;
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)tile[part + e][c];
        store_terms<TERMS>(j.turned + (int64_t)(c0 + c) * TERMS * j.padded_t + r0 + part, j.padded_t, f);
    }
}

// ---------------------------------------------------------------- tiles
// The tile of workgroup g of a grid of ta x tb tiles. Workgroup g runs on XCD g mod 8; each XCD takes a
// contiguous share of an order in which 32 neighbours span 8 tiles of b and 4 of a: what its CUs work on at a time
// shares operands in its L2.
struct Place {
    int a, b;
};
__device__ __forceinline__ Place place_of(int g, int ta, int tb) {
    const int total = ta * tb, q = total / 8, r = total % 8, x = g % 8;
    const int id = x * q + min(x, r) + g / 8;
    const int band = id / (8 * ta), nb = min(8, tb - band * 8), in = id - band * 8 * ta;
    return {in / nb, band * 8 + in % nb};
}

struct Product {
    Operand A, B;
    int stages;      // of 32 k
    int ta, tb;
};

// Of a lane's N elements of a row, how many exist where `left` do from its first one on.
template <int N>
__device__ __forceinline__ int left_of(int64_t left) {
    return left < 0 ? 0 : left < N ? (int)left : N;
}

// ---------------------------------------------------------------- host
constexpr int kCus = 256;

// Which tile a product of `a` x `b` takes, and over how many ranges of K it is cut.
struct Shape {
    int blocks;   // 8, 4 or 2: tiles of 256 x 256, 128 x 128 or 64 x 64
    int ranges;
    bool deep;    // a tile has its CU to itself: a ring of eight stages, else of four
    double us;    // what the model expects
};
// The tile and the number of ranges that a model of the launch puts first: rounds of workgroups over the CUs, each the
// stages of its range and a fixed part (the ring's first loads, the epilogue), and adding the ranges' sums up. A stage
// takes 0.88, 0.36 and 0.15 us (tiles of 256, 128 and 64, all CUs busy; per flop the large one is 1.6 and 2.7 times
// as fast: 4096 x 4096 x 8192 takes 238 us in large tiles and 395 in middle ones), the fixed part 12, 6 and 4 us. The
// small ones win where the large ones leave CUs idle or are mostly padding: 64 tokens, 8192 words of 512 in fp32 30 ->
// 17 us for the logits.
// least_ranges: a power of two, the fewest ranges that the caller takes.
Shape shape_of(int64_t a, int64_t b, int64_t k, int products, bool may_cut, int64_t least_ranges = 1) {
    constexpr double kStage[3] = {0.88, 0.36, 0.15}, kFixed[3] = {12.0, 6.0, 4.0};
    Shape best{};
    double least = 1e300;
    for (int t = 0; t < 3; ++t) {
        const int64_t blocks = 8 >> t, tiles = ceil_div(a, 32 * blocks) * ceil_div(b, 32 * blocks);
        // A range keeps at least eight stages' products, and two stages.
        const int64_t stages = k / kStageK * products, most = std::min(stages / 8, k / kStageK / 2);
        for (int64_t r = least_ranges; r == least_ranges || (may_cut && r <= most && tiles * r <= 2 * kCus); r *= 2) {
            double us = (double)ceil_div(tiles * r, kCus) * ((double)ceil_div(stages, r) * kStage[t] + kFixed[t]);
            if (r > 1) us += 4.0 + (double)(r * a * b) * 8.0 / 4.5e6;
            if (us < least) {
                least = us;
                best = {(int)blocks, (int)r, tiles * r <= kCus, us};
            }
        }
    }
    return best;
}

template <typename F>
void with_tile(const Shape& s, F&& f) {
    if (s.blocks == 8) f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
    else if (s.blocks == 2) f(std::integral_constant<int, 2>(), std::integral_constant<int, 8>());
    else if (s.deep) f(std::integral_constant<int, 4>(), std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
}
Product product_of(const Shape& sh, const Operand& A, const Operand& B, int64_t k) {
    const int64_t t = 32 * sh.blocks;
    return {A, B, (int)(k / kStageK), (int)ceil_div(A.rows, t), (int)ceil_div(B.rows, t)};
}
// Lets a kernel use the LDS of its ring (more than the default limit).
template <typename K>
jorge_status allow_lds(K* kernel, int bytes, const char* why) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) !=
        hipSuccess) {
        (void)hipGetLastError();
        return refuse(JORGE_ERR_HIP, why);
    }
    return JORGE_OK;
}

// The copies of a matrix of rows x cols; flat and turned may be null, padded is the transpose's row length.
Copies copies_of(const void* src, int64_t ld, int64_t rows, int64_t cols, bf16* flat, int64_t kd, bf16* turned,
                 int64_t padded) {
    Copies c{};
    if (!flat && !turned) return c;
    c.src = src;
    c.ld = ld;
    c.rows = rows;
    c.cols = (int)cols;
    c.tiles_c = (int)(kd / 64);
    c.flat = flat;
    c.turned = turned;
    c.padded_f = kd;
    c.padded_t = padded;
    c.tiles = ceil_div(rows, 64) * c.tiles_c;
    return c;
}
template <typename T>
void copy(const Copies& a, const Copies& b, hipStream_t s, const Copies& c = Copies{}) {
    const int64_t tiles = a.tiles + b.tiles + c.tiles;
    if (tiles == 0) return;
    copies_kernel<T, sizeof(T) == 4 ? kTerms : 1><<<dim3((unsigned)tiles), dim3(256), 0, s>>>({{a, b, c}});
}

}  // namespace
}  // namespace jorge_lm
