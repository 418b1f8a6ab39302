// Softmax cross entropy of logits z = hidden weight^T over a vocabulary, forward and backward, for gfx950.
//
// Bound by the matrix products: 2 tokens vocab cols flops forward, and backward as many again for the
// logits, which are not kept, and twice that for the two gradients. All of them run on the bfloat16
// matrix instructions (lm_loss_gemm.hpp).
//
// Forward: a workgroup forms a tile of logits and leaves, for each of its tokens, the maximum of its
// words' logits, the sum of their exponentials relative to it and (label smoothing) their sum; a second
// kernel joins the tiles' statistics of a token in a fixed order.
//
// Backward, a piece of the vocabulary at a time:
//   dz = p - (target distribution), from a tile of logits formed again, rounded to bfloat16 (bf16 inputs) and
//   written both ways round, so that both products below have K-contiguous operands;
//   dhidden += dz weight      (K: the piece's words; the sum over the pieces in fp32)
//   dweight  = dz^T hidden    (K: the tokens; whole, as a piece holds all tokens)
// A piece is as large as keeps dz, and the copies of weight that the products read, within a fixed number of elements,
// so the memory does not grow with the vocabulary.
//
// dz of bf16 inputs is the one value here that is held in fewer than 32 bits, because the matrix instructions take it
// so; in two bfloat16 terms it would double both gradients' products (2.9 ms more of 6.0 for 8192 tokens of 2048, 50001
// words). Who pays: dweight's rows of words that are nobody's target in the batch. Their sums of p h have an error of
// up to 2^-8 in each term, which is 1.5e-3 of such a row before its own rounding to bfloat16 and 2.2e-3 after it,
// where an exact dz leaves 1.66e-3 (46820 of those 50001 rows, measured). dhidden and the rows of words that are
// targets stay at 1.66e-3, their own rounding: the target's -1 is exact and makes up most of them. fp32 inputs have
// dz in three terms.
//
// The copies of weight's piece and of hidden, padded, transposed or split, cost 4% of the time of the gradients'
// products in bf16 and 15% in fp32 at the sizes below, and more the fewer tokens there are: of 64 tokens' 84 us with
// 8192 words of 512 in fp32 they are a quarter.
//
// fp32 operands are split into three bfloat16 terms that sum to them exactly (in bfloat16's range), and a
// product is the six products of terms down to 2^-16 of the whole: the same K loop, six times as long.
// dz is split alike. This is the scheme of the Jorge step's products; there the terms are formed while a
// slab is staged, here once before the product, because every operand enters many tiles.
//
// Measured (a library product of 8192 x 8192 x 8192 in bf16 reaches 1350-1400 TFLOP/s here, x 2048 1140-1200, in fp32
// 153). Rates are over a pass's whole product, all pieces of the vocabulary together:
//   bf16, 8192 tokens, cols 2048, 50001 words: forward 1.33-1.38 ms (1210-1260 TFLOP/s); in seven pieces dz 1.66 ms
//   (1010), each gradient 1.49 ms (1120), transposes 0.12 ms; both passes 6.0 ms.
//   fp32, 2001 tokens, cols 1001, 30011 words (six products each): forward 0.50-0.56 ms (215-240 TFLOP/s of fp32
//   products); in two pieces dz 0.70 ms (172), each gradient 0.57 ms (211), copies 0.17 ms; both passes 2.4 ms.
// The MFMAs are busy 59% of the bf16 forward's wave cycles and 80% of the fp32 one's, which loads half as much for
// each: the former is bound by the way from L2 to LDS as well. Power bounds both: a loop of these MFMAs on registers
// alone reaches 1850-1970 TFLOP/s with random operands, 2430 with zeros.
#include "lm_common.hpp"
#include "lm_product.hpp"

#include <math.h>

#include <algorithm>

namespace jorge_lm {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
struct LossRows {
    const int64_t* targets;
    int64_t tokens, vocab, ignore;
    __device__ __forceinline__ int64_t target(int64_t i) const {
        if (i >= tokens) return -1;
        const int64_t t = targets[i];
        return t >= 0 && t < vocab && t != ignore ? t : -1;
    }
};

// Which of a lane's 4 WA words word `target` is, -1 if none.
template <int WA>
__device__ __forceinline__ int lane_word(int64_t target, int64_t first) {
    const int64_t k = target - first;
    return target >= 0 && k >= 0 && k < 4 * WA ? (int)k : -1;
}

__device__ __forceinline__ float across_groups_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float across_groups_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// Statistics of one part (the 16 WA words of a wave) of the logits: planes [parts][tokens].
struct Stats {
    float *top, *sum, *all;  // all: the plain sum of logits, if wanted
    float* at_target;        // [tokens]
};

// A: words from word0 on; B: tokens.
template <int WA, int WB, int RING, bool SPLIT>
__global__ __launch_bounds__(256, 1) void loss_forward_kernel(Product p, LossRows rows, Stats out, int64_t word0) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using T = Tile<WA, WB, RING, SPLIT>;
    const Place at = place_of(blockIdx.x, p.ta, p.tb);
    T t;
    t.multiply(p.A, p.B, (int64_t)at.a * T::kA, (int64_t)at.b * T::kB, 0, p.stages, p.stages, lds);
    const int64_t a0 = (int64_t)at.a * T::kA + T::lane_a(), b0 = (int64_t)at.b * T::kB + T::lane_b();
    const int left = left_of<4 * WA>(p.A.rows - a0);  // words of this lane that exist
    const int64_t part = (word0 + (int64_t)at.a * T::kA) / (16 * WA) + (threadIdx.x >> 7);
    float top[WB], sum[WB], all[WB];
#pragma unroll
    for (int j = 0; j < WB; ++j) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < WA; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (4 * i + r >= left) t.acc[i][j][r] = -INFINITY;
                m = fmaxf(m, t.acc[i][j][r]);
            }
        m = across_groups_max(m);
        // With nothing above minus infinity the sum is 0, not NaN.
        const float base = m == -INFINITY ? 0.0f : m;
        float s = 0.0f, u = 0.0f;
#pragma unroll
        for (int i = 0; i < WA; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s += __builtin_amdgcn_exp2f((t.acc[i][j][r] - base) * kLog2e);
        if (out.all)
#pragma unroll
            for (int i = 0; i < WA; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) u += 4 * i + r < left ? t.acc[i][j][r] : 0.0f;
        top[j] = m;
        sum[j] = across_groups_sum(s);
        all[j] = out.all ? across_groups_sum(u) : 0.0f;
        // The target's logit, by the one lane that has it.
        const int here = lane_word<WA>(rows.target(b0 + j), word0 + a0);
        const bool hit = here >= 0 && here < left;
        if (__ballot(hit)) {
            float z = 0.0f;
#pragma unroll
            for (int i = 0; i < WA; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) z = here == 4 * i + r ? t.acc[i][j][r] : z;
            if (hit) out.at_target[b0 + j] = z;
        }
    }
    if ((threadIdx.x & 63) < 16) {
#pragma unroll
        for (int j = 0; j < WB; ++j)
            if (b0 + j < p.B.rows) {
                out.top[part * rows.tokens + b0 + j] = top[j];
                out.sum[part * rows.tokens + b0 + j] = sum[j];
                if (out.all) out.all[part * rows.tokens + b0 + j] = all[j];
            }
    }
}

// Joins the parts' statistics of 64 tokens: 16 waves take every 16th part, ascending, and are joined in order.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves * 64) void loss_join_kernel(Stats in, int64_t parts, LossRows rows,
                                                                    float smoothing, float* __restrict__ loss,
                                                                    float* __restrict__ lse) {
    __shared__ float lt[kJoinWaves][64], ls[kJoinWaves][64], la[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i = (int64_t)blockIdx.x * 64 + lane, at = i < rows.tokens ? i : rows.tokens - 1;
    float top = -INFINITY, sum = 0.0f, all = 0.0f;
    const auto add = [&](float m, float s) {
        const float n = fmaxf(top, m);
        // A NaN anywhere stays: fmaxf passes it by, but its sum is NaN.
        const float base = n == -INFINITY ? 0.0f : n;
        sum = sum * __builtin_amdgcn_exp2f((top - base) * kLog2e) + s * __builtin_amdgcn_exp2f((m - base) * kLog2e);
        top = n;
    };
    for (int64_t k = wave; k < parts; k += kJoinWaves) {
        add(in.top[k * rows.tokens + at], in.sum[k * rows.tokens + at]);
        if (in.all) all += in.all[k * rows.tokens + at];
    }
    lt[wave][lane] = top;
    ls[wave][lane] = sum;
    la[wave][lane] = all;
    __syncthreads();
    if (wave || i >= rows.tokens) return;
    for (int w = 1; w < kJoinWaves; ++w) {
        add(lt[w][lane], ls[w][lane]);
        all += la[w][lane];
    }
    const float l = top + logf(sum);
    lse[i] = l;
    float v = 0.0f;
    if (rows.target(i) >= 0) {
        v = l - (1.0f - smoothing) * in.at_target[i];
        if (in.all) v -= smoothing * (all / (float)rows.vocab);
    }
    loss[i] = v;
}

// total = [sum of the losses, rows with a target, mean], by one workgroup, in fp64.
__global__ __launch_bounds__(1024) void loss_total_kernel(const float* __restrict__ loss, LossRows rows,
                                                          float* __restrict__ total) {
    __shared__ double rs[16], rc[16];
    double s = 0.0, c = 0.0;
    for (int64_t i = threadIdx.x; i < rows.tokens; i += 1024)
        if (rows.target(i) >= 0) {
            s += loss[i];
            c += 1.0;
        }
    s = wave_sum(s);
    c = wave_sum(c);
    if ((threadIdx.x & 63) == 0) {
        rs[threadIdx.x >> 6] = s;
        rc[threadIdx.x >> 6] = c;
    }
    __syncthreads();
    if (threadIdx.x) return;
    s = c = 0.0;
    for (int w = 0; w < 16; ++w) {
        s += rs[w];
        c += rc[w];
    }
    total[0] = (float)s;
    total[1] = (float)c;
    total[2] = c > 0.0 ? (float)(s / c) : 0.0f;
}

// ---------------------------------------------------------------- backward
struct DzOut {
    bf16 *dz, *dzt;            // [tokens][terms][words], [words][terms][tokens]
    int64_t words, tokens;     // padded to multiples of 64
};

// dz of a piece: words word0 .. word0 + A.rows; the padding of both copies is written as 0.
template <int WA, int WB, int RING, bool SPLIT>
__global__ __launch_bounds__(256, 1) void loss_dz_kernel(Product p, LossRows rows, const float* __restrict__ lse,
                                                         const float* __restrict__ row_grad, float smoothing,
                                                         int64_t word0, DzOut out) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using T = Tile<WA, WB, RING, SPLIT>;
    const Place at = place_of(blockIdx.x, p.ta, p.tb);
    T t;
    t.multiply(p.A, p.B, (int64_t)at.a * T::kA, (int64_t)at.b * T::kB, 0, p.stages, p.stages, lds);
    const int64_t a0 = (int64_t)at.a * T::kA + T::lane_a(), b0 = (int64_t)at.b * T::kB + T::lane_b();
    const int left = left_of<4 * WA>(p.A.rows - a0);
    const float even = smoothing / (float)rows.vocab;
#pragma unroll
    for (int j = 0; j < WB; ++j) {
        const int64_t target = rows.target(b0 + j);
        const bool live = target >= 0;
        const int here = lane_word<WA>(target, word0 + a0);
        const float l = live ? lse[b0 + j] : 0.0f, g = live && row_grad ? row_grad[b0 + j] : 1.0f;
        const float hit = 1.0f - smoothing;
#pragma unroll
        for (int i = 0; i < WA; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = __builtin_amdgcn_exp2f((t.acc[i][j][r] - l) * kLog2e) - even;
                if (here == 4 * i + r) v -= hit;
                // Selected, not multiplied by 0: what stands in a row without a target may be anything.
                t.acc[i][j][r] = live && 4 * i + r < left ? g * v : 0.0f;
            }
    }
#pragma unroll
    for (int term = 0; term < (SPLIT ? kTerms : 1); ++term) {
        constexpr int terms = SPLIT ? kTerms : 1;
        bf16* const dz = out.dz + term * out.words + a0;
        bf16* const dzt = out.dzt + term * out.tokens + b0;
#pragma unroll
        for (int j = 0; j < WB; ++j)
            if (b0 + j < rows.tokens)
#pragma unroll
                for (int i = 0; i < WA; i += 2) {
                    bf16x8 o;
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = term_of(t.acc[i + e / 4][j][e & 3], term == terms - 1);
                    if (a0 + 4 * i < out.words)
                        *reinterpret_cast<bf16x8*>(dz + (b0 + j) * terms * out.words + 4 * i) = o;
                }
        if (b0 < out.tokens)
#pragma unroll
            for (int i = 0; i < WA; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (4 * i + r < left) {
                        typedef __bf16 V __attribute__((ext_vector_type(WB)));
                        V o;
#pragma unroll
                        for (int j = 0; j < WB; ++j) o[j] = term_of(t.acc[i][j][r], term == terms - 1);
                        *reinterpret_cast<V*>(dzt + (a0 + 4 * i + r) * terms * out.tokens) = o;
                    }
        if constexpr (SPLIT)
#pragma unroll
            for (int j = 0; j < WB; ++j)
#pragma unroll
                for (int i = 0; i < WA; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) t.acc[i][j][r] -= (float)term_of(t.acc[i][j][r], false);
    }
}

// What a gradient is multiplied by after its product: grad[0] (or 1), over the number of rows with a target for a mean;
// 0 where no row has one, whatever grad is.
struct Scale {
    const float *grad, *count;
    bool mean;
    __device__ __forceinline__ float value() const {
        const float n = *count;
        return n > 0.0f ? (grad ? *grad : 1.0f) / (mean ? n : 1.0f) : 0.0f;
    }
};

// C[b][a] over one of gridDim.y ranges of K, to out (whole: one range) or to the range's slice of fp32 sums
// [ranges][B.rows][lda], added to it where `add`. rows: of B's rows, where those are tokens; one without a target gets
// 0, not 0 times what the scale or A may hold.
template <int WA, int WB, int RING, bool SPLIT, typename O>
__global__ __launch_bounds__(256, 1) void loss_grad_kernel(Product p, O* __restrict__ out, int64_t ldo,
                                                           float* __restrict__ slices, int64_t lda, int add,
                                                           Scale scale, LossRows rows) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using T = Tile<WA, WB, RING, SPLIT>;
    const Place at = place_of(blockIdx.x, p.ta, p.tb);
    const int pairs = p.stages / 2;
    const int s0 = (int)((int64_t)pairs * blockIdx.y / gridDim.y) * 2;
    const int s1 = (int)((int64_t)pairs * (blockIdx.y + 1) / gridDim.y) * 2;
    T t;
    t.multiply(p.A, p.B, (int64_t)at.a * T::kA, (int64_t)at.b * T::kB, s0, s1, p.stages, lds);
    const int64_t a0 = (int64_t)at.a * T::kA + T::lane_a(), b0 = (int64_t)at.b * T::kB + T::lane_b();
    const int left = left_of<4 * WA>(p.A.rows - a0);
    if (slices) {
        float* const to = slices + (int64_t)blockIdx.y * p.B.rows * lda;
#pragma unroll
        for (int j = 0; j < WB; ++j)
            if (b0 + j < p.B.rows) {
                f32x4* const q = reinterpret_cast<f32x4*>(to + (b0 + j) * lda + a0);
                // Past the last column up to lda there is room for a whole piece.
                if (add)
#pragma unroll
                    for (int i = 0; i < WA; ++i)
                        if (4 * i < left) t.acc[i][j] += q[i];
#pragma unroll
                for (int i = 0; i < WA; ++i)
                    if (4 * i < left) q[i] = t.acc[i][j];
            }
        return;
    }
    const float f = scale.value();
    constexpr int N = Wide<O>::N;
#pragma unroll
    for (int j = 0; j < WB; ++j)
        if (b0 + j < p.B.rows) {
            const bool none = rows.targets && rows.target(b0 + j) < 0;
#pragma unroll
            for (int i = 0; i < WA; i += N / 4) {
                float v[N];
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = none ? 0.0f : t.acc[i + e / 4][j][e & 3] * f;
                if (4 * i < left) store_wide(out + (b0 + j) * ldo + a0 + 4 * i, left - 4 * i, v);
            }
        }
}

// out[r][c] = scale times the sum of the slices, in order (rows: as above).
template <typename O>
__global__ __launch_bounds__(256) void loss_slices_kernel(const float* __restrict__ slices, int n, int64_t rows,
                                                          int cols, int64_t lda, O* __restrict__ out, int64_t ldo,
                                                          Scale scale, LossRows targets) {
    const int64_t r = blockIdx.x;
    const float f = scale.value();
    const bool none = targets.targets && targets.target(r) < 0;
    for (int c = (blockIdx.y * 256 + threadIdx.x) * 4; c < cols; c += gridDim.y * 1024) {
        const float* p = slices + r * lda + c;
        f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
        int k = 0;
        for (; k + 8 <= n; k += 8) {
            f32x4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const f32x4*>(p + (k + u) * rows * lda);
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        for (; k < n; ++k) s += *reinterpret_cast<const f32x4*>(p + k * rows * lda);
        O* const o = out + r * ldo + c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < cols) o[e] = (O)(none ? 0.0f : s[e] * f);
    }
}

// ---------------------------------------------------------------- host
constexpr const char* kNoLds = "cross entropy: no LDS for a tile";

struct Plan {
    int terms, products;
    int64_t kd, kn, piece;       // padded cols, padded tokens, words of a piece
    bool direct_x, direct_w;     // hidden and weight serve as operands as they are
    Shape logits, dh, dw;
};

bool direct(const jorge_loss_shape& s, const void* p, int64_t ld) {
    return s.dtype == JORGE_BF16 && s.cols % kPadK == 0 && ld % 8 == 0 && aligned(p, 16);
}

// What bounds the workspaces, whatever the vocabulary: elements of one layout of dz (forward: of weight's copy), and,
// where tokens are few and weight outgrows dz, those of each of the backward pass's two copies of it, terms together:
// 1 GiB. In 2^29 elements a piece keeps enough tiles for the CUs: 64 tokens, 128256 words of 4096 in fp32 take 4.43 ms
// and 2.1 GB, in 2^28 4.80 and 1.1, with weight copied whole 4.26 and 6.4; 1 token, 262144 words of 8192 in bf16 5.42,
// 5.85 and 5.05 ms.
constexpr int64_t kPieceElements = 1 << 26;
constexpr int64_t kCopyElements = 1 << 29;
// Tiles of one launch: its threads have to stay below 2^32.
constexpr int64_t kMostTiles = 1 << 23;

// Words of a piece, a multiple of 256 up to `most`: where the tiles are large, those that leave the CUs idle least in
// the last round of a launch's tiles, over the whole vocabulary. A round of dz costs cols (and its exponentials, about
// 400 elements of K), one of dweight tokens; a piece's other launches about a thousand. (8192 tokens, 50001 words of
// 2048: pieces of 8192 words rather than seven equal ones, 6.67 -> 6.50 ms.)
int64_t piece_of(const jorge_loss_shape& s, int64_t most, bool backward) {
    const int64_t even = round_up(ceil_div(s.vocab, ceil_div(s.vocab, most)), 256);
    const int64_t tokens = ceil_div(s.tokens, 256), cols = ceil_div(s.cols, 256);
    if (!backward || even >= s.vocab || tokens * ceil_div(even, 256) < kCus) return even;
    const auto cost = [&](int64_t n) {
        const int64_t w = ceil_div(n, 256);
        return ceil_div(tokens * w, kCus) * (s.cols + 400) + ceil_div(cols * w, kCus) * s.tokens + 1000;
    };
    int64_t best = even, least = INT64_MAX;
    for (int64_t n = most; n >= std::max<int64_t>(512, most / 2); n -= 256) {
        const int64_t last = s.vocab % n, c = s.vocab / n * cost(n) + (last ? cost(last) : 0);
        if (c < least) {
            least = c;
            best = n;
        }
    }
    return best;
}

Plan plan_of(const jorge_loss_shape& s, bool backward, bool direct_x, bool direct_w) {
    Plan p{};
    p.terms = s.dtype == JORGE_F32 ? kTerms : 1;
    p.products = s.dtype == JORGE_F32 ? 6 : 1;
    p.kd = round_up(s.cols, kPadK);
    p.kn = round_up(s.tokens, kPadK);
    p.direct_x = direct_x;
    p.direct_w = direct_w;
    // Without copies of weight the forward pass needs no pieces. A piece may take another tile than the whole
    // vocabulary does, which groups the words of a row's sums otherwise: lse's last bits depend on whether bf16 weight
    // lies so that it can be read in place. The whole vocabulary's tile for its pieces too would cost those (500 tokens
    // of 8192, 128256 words at an odd address: 3.62 against 2.23 ms), the pieces' tile for the whole the usual call.
    int64_t most = kPieceElements / (s.dtype == JORGE_F32 ? 2 : 1) / std::max<int64_t>(1, backward ? p.kn : p.kd);
    if (backward) most = std::min(most, kCopyElements / (p.terms * p.kd));
    if (!backward && direct_w) most = s.vocab;
    most = std::min(most, kMostTiles / ceil_div(std::max<int64_t>(1, s.tokens), 128) * 128);
    most = most < s.vocab ? most / 256 * 256 : round_up(most, 256);
    p.piece = piece_of(s, std::max<int64_t>(512, most), backward);
    const int64_t words = std::min(p.piece, s.vocab);
    p.logits = shape_of(words, s.tokens, p.kd, p.products, false);
    p.dh = shape_of(s.cols, s.tokens, round_up(words, kPadK), p.products, true);
    p.dw = shape_of(s.cols, words, p.kn, p.products, true);
    return p;
}

struct Work {
    bf16 *x, *w;                          // K-contiguous copies: hidden, a piece of weight
    bf16 *xt, *wt;                        // transposed copies
    bf16 *dz, *dzt;
    float *top, *sum, *all, *at_target;   // forward
    float *dh, *dw;                       // slices
    int64_t bytes;
};
Work carve(void* base, const jorge_loss_shape& s, const Plan& p, bool backward) {
    Carve c{(char*)base};
    Work w{};
    const int64_t words = std::min(p.piece, s.vocab), ld = round_up(s.cols, 4);
    if (!p.direct_x) w.x = c.take<bf16>(p.terms * s.tokens * p.kd);
    if (!p.direct_w) w.w = c.take<bf16>(p.terms * words * p.kd);
    if (!backward) {
        const int64_t parts = ceil_div(s.vocab, 16 * p.logits.blocks) + 1;
        w.top = c.take<float>(parts * s.tokens);
        w.sum = c.take<float>(parts * s.tokens);
        if (s.label_smoothing > 0.0) w.all = c.take<float>(parts * s.tokens);
        w.at_target = c.take<float>(s.tokens);
    } else {
        const int64_t ldz = round_up(words, kPadK);
        w.xt = c.take<bf16>(p.terms * s.cols * p.kn);
        w.wt = c.take<bf16>(p.terms * s.cols * ldz);
        w.dz = c.take<bf16>(p.terms * s.tokens * ldz);
        w.dzt = c.take<bf16>(p.terms * words * p.kn);
        if (p.dh.ranges > 1 || s.vocab > p.piece) w.dh = c.take<float>(p.dh.ranges * s.tokens * ld);
        if (p.dw.ranges > 1) w.dw = c.take<float>(p.dw.ranges * words * ld);
    }
    w.bytes = c.used;
    return w;
}
// Whether hidden and weight serve as they are depends on their addresses: room for copies is asked for where
// their type and strides alone do not rule it out.
int64_t workspace_bytes_of(const jorge_loss_shape& s, bool backward) {
    int64_t most = 0;
    for (int k = 0; k < 4; ++k)
        most = std::max(most, carve(nullptr, s, plan_of(s, backward, k & 1, k & 2), backward).bytes);
    return most;
}

// The copies of a matrix, rows without a target taken as zeros in its transpose.
Copies copies_of(const void* src, int64_t ld, int64_t rows, int64_t cols, bf16* flat, int64_t kd, bf16* turned,
                 int64_t padded, const LossRows* targets) {
    Copies c = copies_of(src, ld, rows, cols, flat, kd, turned, padded);
    if (targets && c.src) {
        c.targets = targets->targets;
        c.vocab = targets->vocab;
        c.ignore = targets->ignore;
    }
    return c;
}

// hidden, and a piece of n words of weight from `from` on, as operands.
Operand operand_x(const jorge_loss_shape& s, const Plan& p, const Work& w, const void* hidden) {
    if (p.direct_x) return {(const bf16*)hidden, s.ldh, 0, s.tokens};
    return {w.x, p.terms * p.kd, p.kd, s.tokens};
}
Operand operand_w(const jorge_loss_shape& s, const Plan& p, const Work& w, const void* from, int64_t n) {
    if (p.direct_w) return {(const bf16*)from, s.ldw, 0, n};
    return {w.w, p.terms * p.kd, p.kd, n};
}

template <typename T>
jorge_status forward(const jorge_loss_shape& s, const Plan& p, const Work& w, const void* hidden, const void* weight,
                     const LossRows& rows, float* loss, float* lse, float* total, hipStream_t st) {
    const Operand x = operand_x(s, p, w, hidden);
    const Stats stats{w.top, w.sum, w.all, w.at_target};
    jorge_status err = JORGE_OK;
    for (int64_t v0 = 0; v0 < s.vocab; v0 += p.piece) {
        const int64_t n = std::min(p.piece, s.vocab - v0);
        const T* const from = (const T*)weight + v0 * s.ldw;
        copy<T>(v0 ? Copies{} : copies_of(hidden, s.ldh, s.tokens, s.cols, w.x, p.kd, nullptr, 0, nullptr),
                copies_of(from, s.ldw, n, s.cols, w.w, p.kd, nullptr, 0, nullptr), st);
        const Product pr = product_of(p.logits, operand_w(s, p, w, from, n), x, p.kd);
        with_tile(p.logits, [&](auto W, auto R) {
            constexpr int WA = decltype(W)::value, RING = decltype(R)::value;
            const auto k = loss_forward_kernel<WA, WA, RING, sizeof(T) == 4>;
            if ((err = allow_lds(k, Tile<WA, WA, RING, sizeof(T) == 4>::kBytes, kNoLds)) != JORGE_OK) return;
            k<<<dim3(pr.ta * pr.tb), dim3(256), Tile<WA, WA, RING, sizeof(T) == 4>::kBytes, st>>>(pr, rows, stats, v0);
        });
        if (err != JORGE_OK) return err;
    }
    // Words of a part: every piece but the last is a whole number of parts, and the last one's tile
    // may have parts past its end, whose statistics are those of nothing.
    const int64_t per = 16 * p.logits.blocks, last = (ceil_div(s.vocab, p.piece) - 1) * p.piece;
    const int64_t parts = last / per + ceil_div(s.vocab - last, 2 * per) * 2;
    loss_join_kernel<<<dim3((unsigned)ceil_div(s.tokens, 64)), dim3(kJoinWaves * 64), 0, st>>>(
        stats, parts, rows, (float)s.label_smoothing, loss, lse);
    loss_total_kernel<<<dim3(1), dim3(1024), 0, st>>>(loss, rows, total);
    return launched("cross entropy");
}

// One gradient: out = scale * A-by-B, in slices where K is cut or the sum goes on (first, last: of the sum's pieces).
template <typename T>
jorge_status gradient(const Shape& sh, const Product& pr, T* out, int64_t ldo, int64_t cols, float* slices, bool first,
                      bool last, const Scale& scale, const LossRows& rows, hipStream_t st) {
    jorge_status err = JORGE_OK;
    const int64_t lda = round_up(cols, 4);
    with_tile(sh, [&](auto W, auto R) {
        constexpr int WA = decltype(W)::value, RING = decltype(R)::value;
        const auto k = loss_grad_kernel<WA, WA, RING, sizeof(T) == 4, T>;
        if ((err = allow_lds(k, Tile<WA, WA, RING, sizeof(T) == 4>::kBytes, kNoLds)) != JORGE_OK) return;
        // The first piece of a sum is the longest and fills every slice; a short last one may add to fewer.
        const int ranges = std::min(sh.ranges, pr.stages / 2);
        k<<<dim3(pr.ta * pr.tb, ranges), dim3(256), Tile<WA, WA, RING, sizeof(T) == 4>::kBytes, st>>>(
            pr, out, ldo, slices, lda, first ? 0 : 1, scale, rows);
    });
    if (err != JORGE_OK) return err;
    if (slices && last)
        loss_slices_kernel<T><<<dim3((unsigned)pr.B.rows, (unsigned)ceil_div(cols, 1024)), dim3(256), 0, st>>>(
            slices, sh.ranges, pr.B.rows, (int)cols, lda, out, ldo, scale, rows);
    return JORGE_OK;
}

template <typename T>
jorge_status backward(const jorge_loss_shape& s, const Plan& p, const Work& w, const float* grad, int32_t kind,
                      const void* hidden, const void* weight, const LossRows& rows, const float* lse,
                      const float* total, void* dhidden, void* dweight, hipStream_t st) {
    const Scale scale{kind == JORGE_LOSS_ROWS ? nullptr : grad, total + 1, kind == JORGE_LOSS_MEAN};
    const float* const row_grad = kind == JORGE_LOSS_ROWS ? grad : nullptr;
    const Operand x = operand_x(s, p, w, hidden);
    const Operand xt{w.xt, p.terms * p.kn, p.kn, s.cols};
    jorge_status err = JORGE_OK;
    for (int64_t v0 = 0; v0 < s.vocab; v0 += p.piece) {
        const int64_t n = std::min(p.piece, s.vocab - v0), ldz = round_up(n, kPadK);
        const T* const from = (const T*)weight + v0 * s.ldw;
        copy<T>(v0 ? Copies{}
                   : copies_of(hidden, s.ldh, s.tokens, s.cols, w.x, p.kd, dweight ? w.xt : nullptr, p.kn, &rows),
                copies_of(from, s.ldw, n, s.cols, w.w, p.kd, dhidden ? w.wt : nullptr, ldz, nullptr), st);
        const Product pr = product_of(p.logits, operand_w(s, p, w, from, n), x, p.kd);
        const DzOut dz{w.dz, w.dzt, ldz, p.kn};
        with_tile(p.logits, [&](auto W, auto R) {
            constexpr int WA = decltype(W)::value, RING = decltype(R)::value;
            const auto k = loss_dz_kernel<WA, WA, RING, sizeof(T) == 4>;
            if ((err = allow_lds(k, Tile<WA, WA, RING, sizeof(T) == 4>::kBytes, kNoLds)) != JORGE_OK) return;
            k<<<dim3(pr.ta * pr.tb), dim3(256), Tile<WA, WA, RING, sizeof(T) == 4>::kBytes, st>>>(
                pr, rows, lse, row_grad, (float)s.label_smoothing, v0, dz);
        });
        if (err != JORGE_OK) return err;
        if (dhidden) {
            const Operand wt{w.wt, p.terms * ldz, ldz, s.cols}, z{w.dz, p.terms * ldz, ldz, s.tokens};
            err = gradient(p.dh, product_of(p.dh, wt, z, ldz), (T*)dhidden, s.ldh, s.cols, w.dh, v0 == 0,
                           v0 + n == s.vocab, scale, rows, st);
            if (err != JORGE_OK) return err;
        }
        if (dweight) {
            const Operand zt{w.dzt, p.terms * p.kn, p.kn, n};
            err = gradient(p.dw, product_of(p.dw, xt, zt, p.kn), (T*)dweight + v0 * s.ldw, s.ldw, s.cols, w.dw, true,
                           true, scale, LossRows{}, st);
            if (err != JORGE_OK) return err;
        }
    }
    return launched("cross entropy");
}

template <typename T>
__global__ __launch_bounds__(256) void zero_rows_kernel(T* p, int64_t ld, int64_t cols) {
    for (int64_t c = threadIdx.x; c < cols; c += 256) p[blockIdx.x * ld + c] = (T)0.0f;
}

jorge_status check(const jorge_loss_shape* s) {
    if (!s) return bad("cross entropy: a shape is needed");
    if (!known_dtype(s->dtype)) return bad("cross entropy: unknown element type");
    if (s->tokens < 0 || s->cols < 1 || s->vocab < 1)
        return bad("cross entropy: tokens >= 0, cols >= 1 and vocab >= 1 are needed");
    if (s->tokens > JORGE_LOSS_MAX_TOKENS)
        return refuse(JORGE_ERR_UNSUPPORTED, "cross entropy: tokens above JORGE_LOSS_MAX_TOKENS");
    if (s->vocab > JORGE_LOSS_MAX_VOCAB)
        return refuse(JORGE_ERR_UNSUPPORTED, "cross entropy: vocab above JORGE_LOSS_MAX_VOCAB");
    if (s->cols > JORGE_LOSS_MAX_COLS)
        return refuse(JORGE_ERR_UNSUPPORTED, "cross entropy: cols above JORGE_LOSS_MAX_COLS");
    if (ceil_div(s->tokens, 64) * ceil_div(s->cols, 64) > 1 << 23)
        return refuse(JORGE_ERR_UNSUPPORTED, "cross entropy: tokens * cols above 2^35");
    if (s->ldh < s->cols || s->ldw < s->cols) return bad("cross entropy: a row stride is below cols");
    if (s->ldh > JORGE_LOSS_MAX_STRIDE || s->ldw > JORGE_LOSS_MAX_STRIDE)
        return refuse(JORGE_ERR_UNSUPPORTED, "cross entropy: a row stride above JORGE_LOSS_MAX_STRIDE (2^22)");
    if (!(s->label_smoothing >= 0.0 && s->label_smoothing <= 1.0))
        return bad("cross entropy: label_smoothing must be in [0, 1]");
    return JORGE_OK;
}

}  // namespace
}  // namespace jorge_lm

using namespace jorge_lm;

extern "C" {

jorge_status jorge_cross_entropy_workspace(const jorge_loss_shape* shape, int32_t backward, int64_t* bytes) {
    if (!bytes) return bad("cross entropy: bytes is needed");
    const jorge_status st = check(shape);
    if (st != JORGE_OK) return st;
    *bytes = shape->tokens ? workspace_bytes_of(*shape, backward != 0) : 0;
    return JORGE_OK;
}

jorge_status jorge_cross_entropy_forward(const jorge_loss_shape* shape, const void* hidden, const void* weight,
                                         const int64_t* targets, float* loss, float* lse, float* total, void* workspace,
                                         int64_t workspace_bytes, void* hip_stream) {
    jorge_status st = check(shape);
    if (st != JORGE_OK) return st;
    const jorge_loss_shape& s = *shape;
    const int64_t e = dtype_bytes(s.dtype);
    if (!total || !aligned(total, 4)) return bad("cross entropy: total is needed");
    if (s.tokens > 0) {
        if (!hidden || !weight || !targets || !loss || !lse)
            return bad("cross entropy: hidden, weight, targets, loss and lse are needed");
        if (!aligned(hidden, e) || !aligned(weight, e) || !aligned(targets, 8) || !aligned(loss, 4) || !aligned(lse, 4))
            return bad("cross entropy: a pointer is not aligned to its element");
        if (!workspace || !aligned(workspace, kAlign))
            return bad("cross entropy: a workspace aligned to 256 bytes is needed");
        if (workspace_bytes < workspace_bytes_of(s, false)) return bad("cross entropy: the workspace is too small");
    }
    const LossRows rows{targets, s.tokens, s.vocab, s.ignore_index};
    const hipStream_t q = reinterpret_cast<hipStream_t>(hip_stream);
    if (s.tokens == 0) {
        loss_total_kernel<<<dim3(1), dim3(1024), 0, q>>>(loss, rows, total);
        return launched("cross entropy");
    }
    const Plan p = plan_of(s, false, direct(s, hidden, s.ldh), direct(s, weight, s.ldw));
    const Work w = carve(workspace, s, p, false);
    if (s.dtype == JORGE_F32) return forward<float>(s, p, w, hidden, weight, rows, loss, lse, total, q);
    return forward<bf16>(s, p, w, hidden, weight, rows, loss, lse, total, q);
}

jorge_status jorge_cross_entropy_backward(const jorge_loss_shape* shape, const float* grad, int32_t kind,
                                          const void* hidden, const void* weight, const int64_t* targets,
                                          const float* lse, const float* total, void* dhidden, void* dweight,
                                          void* workspace, int64_t workspace_bytes, void* hip_stream) {
    jorge_status st = check(shape);
    if (st != JORGE_OK) return st;
    const jorge_loss_shape& s = *shape;
    const int64_t e = dtype_bytes(s.dtype);
    if (kind != JORGE_LOSS_ROWS && kind != JORGE_LOSS_SUM && kind != JORGE_LOSS_MEAN)
        return bad("cross entropy: unknown kind of gradient");
    if (!aligned(dhidden, e) || !aligned(dweight, e))
        return bad("cross entropy: a pointer is not aligned to its element");
    const hipStream_t q = reinterpret_cast<hipStream_t>(hip_stream);
    if (s.tokens == 0) {
        if (dweight) {
            if (s.dtype == JORGE_F32)
                zero_rows_kernel<float><<<dim3((unsigned)s.vocab), dim3(256), 0, q>>>((float*)dweight, s.ldw, s.cols);
            else zero_rows_kernel<bf16><<<dim3((unsigned)s.vocab), dim3(256), 0, q>>>((bf16*)dweight, s.ldw, s.cols);
        }
        return launched("cross entropy");
    }
    if (!grad || !hidden || !weight || !targets || !lse || !total)
        return bad("cross entropy: grad, hidden, weight, targets, lse and total are needed");
    if (!aligned(grad, 4) || !aligned(hidden, e) || !aligned(weight, e) || !aligned(targets, 8) || !aligned(lse, 4) ||
        !aligned(total, 4))
        return bad("cross entropy: a pointer is not aligned to its element");
    if (!workspace || !aligned(workspace, kAlign))
        return bad("cross entropy: a workspace aligned to 256 bytes is needed");
    if (workspace_bytes < workspace_bytes_of(s, true)) return bad("cross entropy: the workspace is too small");
    if (!dhidden && !dweight) return JORGE_OK;
    const Plan p = plan_of(s, true, direct(s, hidden, s.ldh), direct(s, weight, s.ldw));
    const Work w = carve(workspace, s, p, true);
    const LossRows rows{targets, s.tokens, s.vocab, s.ignore_index};
    if (s.dtype == JORGE_F32)
        return backward<float>(s, p, w, grad, kind, hidden, weight, rows, lse, total, dhidden, dweight, q);
    return backward<bf16>(s, p, w, grad, kind, hidden, weight, rows, lse, total, dhidden, dweight, q);
}

}  // extern "C"
