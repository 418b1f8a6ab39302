// The linear layer y = act(x weight^T + bias) + residual and the gated projection y = act(x gate^T) * (x up^T), forward
// and backward, for gfx950.
//
// Bound by the matrix products: 2 tokens cols outs flops a matrix forward and twice that backward, and once more
// backward where an activation's argument is formed again rather than kept: kept in 32 bits it would take four bytes
// for every two of y, and rounded to bfloat16 it would put a second rounding into every gradient.
//
// Forward: a tile of products stays in registers for bias, activation, product of the pair and residual. The gated
// projection's tile is of the same columns of both matrices (Tile's PAIR), so that a lane holds both factors.
//
// Backward:
//   dz = dy act'(z)  (gated: dgate = dy u act'(g), dup = dy act(g), side by side as one matrix of 2 outs columns)
//   dx = dz weight       (K: the columns of dz)
//   dweight = dz^T x     (K: the tokens)
// bfloat16: dz is rounded to it, as the matrix instructions take it (a gradient, a sum of such terms, errs by up to
// 2.4e-3 of its size instead of the 1.7e-3 of its own rounding); weight, x and dz are read as they lie, K along their
// rows or across them (Tile's TA and TB). fp32: dz is written both ways round, in three terms, from the registers of the
// tile that forms z again, and x and weight are copied so. Without an activation dz is dy as it is. dbias is summed
// from the unrounded dz.
//
// Few tokens, forward: bound by reading the weights once. A workgroup takes 16 of their rows, its eight waves cut K,
// and nothing goes through LDS but the sums; fp32 then runs on the fp32 MFMAs, as splits would cost three times the
// bytes.
#include "lm_product.hpp"

#include <math.h>

namespace jorge_lm {
namespace {

constexpr float kLog2e = 1.44269504088896341f;

// ---------------------------------------------------------------- activations
// 1 / (1 + exp(-z)). exp(-z) = 2^t 2^r with t the rounded product -z log2(e) and r what its rounding left out (fp32).
template <bool EXACT>
__device__ __forceinline__ float logistic(float z) {
    const float t = -z * kLog2e;
    float e = __builtin_amdgcn_exp2f(t);
    if constexpr (EXACT) {
        const float r = __builtin_fmaf(-z, kLog2e, -t) - z * 1.925963033500e-8f;
        e = __builtin_fmaf(e, r * 0.693147180559945f, e);
    }
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    // Beyond 88 the steps above overflow, and the sigmoid is 0 or 1 to the last bit. A NaN passes both comparisons by.
    return z < -88.0f ? 0.0f : z > 88.0f ? 1.0f : s;
}
// The normal distribution's upper tail at m >= 0, erfc(x) / 2 with x = m / sqrt(2), and exp(-x^2).
struct Upper {
    float tail, bell;
};
template <bool EXACT>
__device__ __forceinline__ Upper upper(float m) {
    if constexpr (EXACT) {
        // gelu(-m) is as small as the tail, so the tail's relative error is the result's. erfc(x) = exp(-x^2) times a slow
        // function of x, which is Q(y) / (x + 3) with y = (x - 3) / (x + 3) and Q a polynomial fitted to it up to x = 9.4
        // (1.4e-9 of it; the map is Shepherd and Laframboise's), where both results leave fp32; in fp32 the tail is within
        // 12 roundings. x^2's own is made up for by a factor of the exponential. Beyond 20 both are 0. A NaN passes the
        // comparison by. A forward pass in fp32 of 8192 tokens, 1024 -> 4096, takes 315 us, 308 with the polynomial below and
        // 357 with erfcf.
        constexpr float kHalf = 0.5f * kLog2e, kHalfLow = 0.5f * 1.925963033500e-8f;
        m = m > 20.0f ? 20.0f : m;
        const float q = __builtin_amdgcn_rcpf(__builtin_fmaf(m, 0.707106781186547524f, 3.0f));
        const float y = __builtin_fmaf(q, -6.0f, 1.0f);
        float tail = __builtin_fmaf(-1.652540540e-4f, y, -2.465911536e-4f);
        tail = __builtin_fmaf(tail, y, 1.538947947e-3f);
        tail = __builtin_fmaf(tail, y, -6.108181731e-4f);
        tail = __builtin_fmaf(tail, y, -1.341892682e-2f);
        tail = __builtin_fmaf(tail, y, 5.976416205e-2f);
        tail = __builtin_fmaf(tail, y, -1.552331529e-1f);
        tail = __builtin_fmaf(tail, y, 2.951141701e-1f);
        tail = __builtin_fmaf(tail, y, -4.416972383e-1f);
        tail = __builtin_fmaf(tail, y, 5.370034537e-1f);
        const float s = m * m, t = -kHalf * s;
        const float r = __builtin_fmaf(-kHalf, s, -t) - kHalf * __builtin_fmaf(m, m, -s) - kHalfLow * s;
        float bell = __builtin_amdgcn_exp2f(t);
        bell = __builtin_fmaf(bell, r * 0.693147180559945f, bell);
        return {tail * q * bell, bell};
    } else {
        // The polynomial 7.1.26 of Abramowitz and Stegun in 1 / (1 + p x) times exp(-x^2), off by at most 0.75e-7 and in
        // fp32 by 2.7e-7; the same exponential is the density. That is of the tail's size from m = 5 on, where gelu is
        // below 2e-6: nothing next to bfloat16's other values, but not for fp32 results. A forward pass in bfloat16 of
        // 4096 tokens, 1024 -> 4096, took 84 us with erff and 72 us with this.
        const float x = 0.707106781186547524f * m;
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
        const float bell = __builtin_amdgcn_exp2f(-kLog2e * x * x);
        float tail = __builtin_fmaf(1.061405429f, t, -1.453152027f);
        tail = __builtin_fmaf(tail, t, 1.421413741f);
        tail = __builtin_fmaf(tail, t, -0.284496736f);
        tail = __builtin_fmaf(tail, t, 0.254829592f);
        return {tail * (0.5f * t * bell), bell};
    }
}
struct Acted {
    float a, d;  // act(z), act'(z)
};
// EXACT: fp32 results; otherwise they will be rounded to bfloat16.
template <int ACT, bool EXACT>
__device__ __forceinline__ Acted acted(float z) {
    switch (ACT) {
        case JORGE_ACT_RELU: return {z > 0.0f || z != z ? z : 0.0f, z > 0.0f ? 1.0f : z != z ? z : 0.0f};
        case JORGE_ACT_GELU: {
            const Upper u = upper<EXACT>(__builtin_fabsf(z));
            const float phi = z < 0.0f ? u.tail : 1.0f - u.tail;
            return {z * phi, __builtin_fmaf(z, 0.398942280401432678f * u.bell, phi)};
        }
        case JORGE_ACT_SILU: {
            const float s = logistic<EXACT>(z);
            return {z * s, s * (1.0f + z * (1.0f - s))};
        }
        case JORGE_ACT_SIGMOID: {
            const float s = logistic<EXACT>(z);
            return {s, s * (1.0f - s)};
        }
        default: return {z, 1.0f};
    }
}
// f(activation as a constant): the choice is made once for what f does, not for each element.
template <typename F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
    switch (act) {
        case JORGE_ACT_RELU: return f(std::integral_constant<int, JORGE_ACT_RELU>());
        case JORGE_ACT_GELU: return f(std::integral_constant<int, JORGE_ACT_GELU>());
        case JORGE_ACT_SILU: return f(std::integral_constant<int, JORGE_ACT_SILU>());
        case JORGE_ACT_SIGMOID: return f(std::integral_constant<int, JORGE_ACT_SIGMOID>());
        default: return f(std::integral_constant<int, JORGE_ACT_NONE>());
    }
}

// ---------------------------------------------------------------- epilogues
// M consecutive elements at p, of which `left` exist.
template <int M, typename T>
__device__ __forceinline__ void load_some(const T* p, int left, float (&f)[M]) {
    typedef T V __attribute__((ext_vector_type(M), aligned(sizeof(T))));
    if (left >= M) {
        const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
        for (int e = 0; e < M; ++e) f[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < M; ++e) f[e] = e < left ? (float)p[e] : 0.0f;
    }
}
template <int M, typename T>
__device__ __forceinline__ void store_some(T* p, int left, const float (&f)[M]) {
    typedef T V __attribute__((ext_vector_type(M), aligned(sizeof(T))));
    if (left >= M) {
        V v;
#pragma unroll
        for (int e = 0; e < M; ++e) v[e] = (T)f[e];
        *reinterpret_cast<V*>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < M; ++e)
            if (e < left) p[e] = (T)f[e];
    }
}

// A bias vector of either type, or none.
struct Bias {
    const void* p;
    int bf;
    template <int M>
    __device__ __forceinline__ void load(int64_t c, int left, float (&f)[M]) const {
        if (!p) {
#pragma unroll
            for (int e = 0; e < M; ++e) f[e] = 0.0f;
        } else if (bf) load_some<M>((const bf16*)p + c, left, f);
        else load_some<M>((const float*)p + c, left, f);
    }
};

// What a product becomes. z: x weight^T, u: x up^T (gated).
template <typename T>
struct Finish {
    Bias bias;
    const T* residual;
    T* y;
    int64_t ldr, ldy;
    int act;
    // M elements of row `row` from column c on, of which `left` exist. y may be residual: read before it is written.
    template <int M, bool PAIR>
    __device__ __forceinline__ void store(int64_t row, int64_t c, int left, const float (&z)[M],
                                          const float (&u)[M]) const {
        if (left <= 0) return;
        float b[M], r[M];
        if constexpr (!PAIR) {
            bias.template load<M>(c, left, b);
            if (residual) load_some<M>(residual + row * ldr + c, left, r);
        }
        store<M, PAIR>(row, c, left, z, u, b, r);
    }
    // b: the bias, r: the residual (where there is one).
    template <int M, bool PAIR>
    __device__ __forceinline__ void store(int64_t row, int64_t c, int left, const float (&z)[M], const float (&u)[M],
                                          const float (&b)[M], const float (&r)[M]) const {
        float f[M];
        with_activation(act, [&](auto A) {
#pragma unroll
            for (int e = 0; e < M; ++e) f[e] = acted<decltype(A)::value, sizeof(T) == 4>(PAIR ? z[e] : z[e] + b[e]).a;
        });
        if (PAIR || residual)
#pragma unroll
            for (int e = 0; e < M; ++e) f[e] = PAIR ? f[e] * u[e] : f[e] + r[e];
        store_some<M>(y + row * ldy + c, left, f);
    }
};

// A wave's part of a tile, row by row: the rows (tokens) of four columns j of its accumulators at a time go through LDS,
// so that a lane gets 8 consecutive columns of a row (8 of both matrices, PAIR) and a row's stores are whole cache lines.
// The body is in a loop: unrolled over all accumulators, activations would spill them. What a row needs from memory is
// loaded four passes ahead: a workgroup has its CU to itself, and nothing else would hide that time (dz of 8192 tokens,
// 2048 -> 2 x 8192: 574 us with every load waited for, 515 so).
template <int WA, bool PAIR>
struct Rows {
    static constexpr int kCols = PAIR ? 8 * WA : 16 * WA;          // of a row, of one matrix
    static constexpr int kLanes = kCols / 8, kPasses = kLanes / 4; // lanes to a row; passes of 64 / kLanes rows
    static constexpr int kJ = WA < 4 ? WA : 4, kAll = kJ * kPasses, kAhead = kAll < 4 ? kAll : 4;
    static_assert(kPasses >= 1 && kAll % kAhead == 0, "a pass takes whole rows");
    float* at;                                                     // this wave's area
    int c;                                                         // this lane's first column
    __device__ __forceinline__ explicit Rows(char* lds)
        : at(reinterpret_cast<float*>(lds) + (threadIdx.x >> 6) * kJ * 256 * WA),
          c((threadIdx.x & 63) % kLanes * 8) {}
    // Piece of 4 columns of a row of the jj-th of the columns j; the pieces are permuted so that 16 rows meet all banks.
    __device__ __forceinline__ f32x4* piece(int jj, int row, int n) const {
        const int swizzled = n ^ (WA == 2 ? row >> 1 & 7 : row & 15);
        return reinterpret_cast<f32x4*>(at + (jj * 16 + row) * 16 * WA + swizzled * 4);
    }
    // Piece i of this lane's own accumulators, of row lane % 16.
    __device__ __forceinline__ f32x4* own(int jj, int i) const {
        const int lane = threadIdx.x & 63;
        const int n = PAIR ? i / (WA / 2) * 2 * WA + (lane >> 4) * (WA / 2) + i % (WA / 2) : (lane >> 4) * WA + i;
        return piece(jj, lane & 15, n);
    }
    static __device__ __forceinline__ void fence() {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __device__ __forceinline__ void put(int jj, int row, const float (&z)[8], const float (&u)[8]) const {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            *piece(jj, row, c / 4 + n) = f32x4{z[4 * n], z[4 * n + 1], z[4 * n + 2], z[4 * n + 3]};
            if constexpr (PAIR)
                *piece(jj, row, (kCols + c) / 4 + n) = f32x4{u[4 * n], u[4 * n + 1], u[4 * n + 2], u[4 * n + 3]};
        }
    }
    // load(row, j): what row `row` of column j needs, started ahead; use(jj, row, j, z, u, that): its values. again: what
    // use() has put back is wanted in the accumulators.
    template <typename ACC, typename LOAD, typename USE>
    __device__ __forceinline__ void each(ACC& acc, bool again, LOAD&& load, USE&& use) const {
#pragma unroll
        for (int j0 = 0; j0 < WA; j0 += kJ) {
            decltype(load(0, 0)) ahead[kAhead];
            const int lane_row = (threadIdx.x & 63) / kLanes;
            const auto row_of = [&](int pass) { return pass % kPasses * (64 / kLanes) + lane_row; };
#pragma unroll
            for (int n = 0; n < kAhead; ++n) ahead[n] = load(row_of(n), j0 + n / kPasses);
            fence();
#pragma unroll
            for (int jj = 0; jj < kJ; ++jj)
#pragma unroll
                for (int i = 0; i < WA; ++i) *own(jj, i) = acc[i][j0 + jj];
            fence();
#pragma unroll 1
            for (int pass = 0; pass < kAll; pass += kAhead)
#pragma unroll
                for (int n = 0; n < kAhead; ++n) {
                    const int jj = (pass + n) / kPasses, row = row_of(pass + n);
                    float z[8], u[8];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const f32x4 a = *piece(jj, row, c / 4 + k);
                        const f32x4 b = PAIR ? *piece(jj, row, (kCols + c) / 4 + k) : a;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            z[4 * k + e] = a[e];
                            u[4 * k + e] = b[e];
                        }
                    }
                    const auto now = ahead[n];
                    if (pass + kAhead < kAll) ahead[n] = load(row_of(pass + kAhead + n), j0 + (pass + kAhead + n) / kPasses);
                    use(jj, row, j0 + jj, z, u, now);
                }
            if (again) {
                fence();
#pragma unroll
                for (int jj = 0; jj < kJ; ++jj)
#pragma unroll
                    for (int i = 0; i < WA; ++i) acc[i][j0 + jj] = *own(jj, i);
            }
        }
    }
};
struct Nothing {};

// 8 elements of a row as they lie, of which `left` exist.
template <typename T>
struct Raw {
    typedef T V __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    V v;
    __device__ __forceinline__ void load(const T* p, int left) {
        if (left >= 8) v = *reinterpret_cast<const V*>(p);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < left ? p[e] : (T)0.0f;
    }
    __device__ __forceinline__ void get(float (&f)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)v[e];
    }
};

// The stages of range n of `of` along K, if not given the workgroup's (blockIdx.y of gridDim.y).
struct Range {
    int s0, s1;
    __device__ __forceinline__ explicit Range(int stages) : Range(stages, blockIdx.y, gridDim.y) {}
    __device__ __forceinline__ Range(int stages, int n, int of) {
        const int pairs = stages / 2;
        s0 = (int)((int64_t)pairs * n / of) * 2;
        s1 = (int)((int64_t)pairs * (n + 1) / of) * 2;
    }
};

// A product of one matrix (A) or two (A and A2) with B's rows.
struct Dense {
    Product p;
    Operand A2;
};

// Tiles of y, or, where K is cut, of its sums: slices [ranges][tokens][lda], the second matrix's columns lda / 2 on.
template <int WA, int RING, bool SPLIT, bool PAIR, typename T>
__global__ __launch_bounds__(256, 1) void dense_forward_kernel(Dense d, Finish<T> out, float* __restrict__ slices,
                                                               int64_t lda) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using Q = Tile<WA, WA, RING, SPLIT, PAIR>;
    const Place at = place_of(blockIdx.x, d.p.ta, d.p.tb);
    const Range k(d.p.stages);
    Q t;
    t.multiply(d.p.A, d.A2, d.p.B, (int64_t)at.a * Q::kRowsA, (int64_t)at.b * Q::kB, k.s0, k.s1, d.p.stages, lds);
    const int64_t a0 = (int64_t)at.a * Q::kRowsA + Q::lane_a(), b0 = (int64_t)at.b * Q::kB + Q::lane_b();
    const int left = left_of<Q::kLaneA>(d.p.A.rows - a0);
    constexpr int kUp = PAIR ? WA / 2 : 0;
    if (slices) {
#pragma unroll
        for (int j = 0; j < WA; ++j)
            if (b0 + j < d.p.B.rows) {
                f32x4* const q = reinterpret_cast<f32x4*>(slices + (blockIdx.y * d.p.B.rows + b0 + j) * lda + a0);
                // Past the last column up to a multiple of four there is room.
#pragma unroll
                for (int i = 0; i < Q::kLaneA / 4; ++i)
                    if (4 * i < left) {
                        q[i] = t.acc[i][j];
                        if constexpr (PAIR) q[i + lda / 8] = t.acc[i + kUp][j];
                    }
            }
        return;
    }
    const Rows<WA, PAIR> rows(lds);
    const int64_t wa = (int64_t)at.a * Q::kRowsA + (threadIdx.x >> 7) * (Q::kRowsA / 2);
    const int64_t wb = (int64_t)at.b * Q::kB + ((threadIdx.x >> 6) & 1) * (Q::kB / 2);
    const int n = left_of<8>(d.p.A.rows - wa - rows.c);  // of this lane's columns
    float bias[8] = {};
    if constexpr (!PAIR) out.bias.template load<8>(wa + rows.c, n, bias);
    rows.each(
        t.acc, false,
        [&](int row, int j) {
            Raw<T> r{};
            const int64_t token = wb + row * WA + j;
            if (!PAIR && out.residual && n && token < d.p.B.rows) r.load(out.residual + token * out.ldr + wa + rows.c, n);
            return r;
        },
        [&](int, int row, int j, const float(&z)[8], const float(&u)[8], const Raw<T>& raw) {
            const int64_t token = wb + row * WA + j;
            float r[8];
            raw.get(r);
            if (n && token < d.p.B.rows) out.template store<8, PAIR>(token, wa + rows.c, n, z, u, bias, r);
        });
}

// The sum of n slices at p, a fixed distance apart, in order.
__device__ __forceinline__ f32x4 sum_slices(const float* p, int n, int64_t apart) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    int k = 0;
    for (; k + 4 <= n; k += 4) {
        f32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const f32x4*>(p + (k + u) * apart);
        s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    for (; k < n; ++k) s += *reinterpret_cast<const f32x4*>(p + k * apart);
    return s;
}

template <bool PAIR, typename T>
__global__ __launch_bounds__(256) void dense_join_kernel(const float* __restrict__ slices, int n, int64_t rows,
                                                         int cols, int64_t lda, Finish<T> out) {
    const int64_t r = blockIdx.x;
    for (int c = (blockIdx.y * 256 + threadIdx.x) * 4; c < cols; c += gridDim.y * 1024) {
        const float* const p = slices + r * lda + c;
        const f32x4 a = sum_slices(p, n, rows * lda), b = PAIR ? sum_slices(p + lda / 2, n, rows * lda) : a;
        const float z[4] = {a[0], a[1], a[2], a[3]}, u[4] = {b[0], b[1], b[2], b[3]};
        out.template store<4, PAIR>(r, c, cols - c, z, u);
    }
}

// ---------------------------------------------------------------- few tokens
constexpr int kFewWaves = 8, kFewTokens = JORGE_LINEAR_FEW_TOKENS;  // the most tokens of the kernel below
static_assert(kFewTokens == 64, "16 NT");

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));

// A lane's piece of a row for one step along K: 16 bytes, zeros past the end.
template <typename T>
struct Piece;
template <>
struct Piece<bf16> {
    static constexpr int K = 32, E = 8;  // elements of K of a step, of a lane's piece
    bf16x8 v;
    __device__ __forceinline__ void load(const bf16* p, int left) {
        if (left >= E) v = *reinterpret_cast<const bf16x8u*>(p);
        else
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = e < left ? p[e] : (bf16)0.0f;
    }
    static __device__ __forceinline__ void mma(f32x4& c, const Piece& a, const Piece& b) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
    }
};
template <>
struct Piece<float> {
    static constexpr int K = 16, E = 4;
    f32x4 v;
    __device__ __forceinline__ void load(const float* p, int left) {
        if (left >= E) v = *reinterpret_cast<const f32x4u*>(p);
        else
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = e < left ? p[e] : 0.0f;
    }
    // The four MFMAs take the same elements of both operands, so which k each is does not matter.
    static __device__ __forceinline__ void mma(f32x4& c, const Piece& a, const Piece& b) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e], b.v[e], c, 0, 0, 0);
    }
};

struct FewRows {
    const void *x, *w, *u;
    int64_t ldx, ldw, ldu, outs;
    int tokens, cols;
};

// Rows 16 blockIdx.x .. of the weights (of both), all tokens (up to 16 NT). An MFMA leaves lane l with rows
// 4 (l / 16) + r of the weights and token l % 16.
template <typename T, int NT, bool PAIR>
__global__ __launch_bounds__(kFewWaves * 64) void dense_few_kernel(FewRows in, Finish<T> out) {
    using P = Piece<T>;
    constexpr int MATS = PAIR ? 2 : 1, U = NT == 1 ? 4 : 2;  // steps whose loads are started together
    __shared__ float sums[kFewWaves][MATS][NT][64][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = (lane >> 4) * P::E;
    const int64_t row0 = (int64_t)blockIdx.x * 16, row = row0 + (lane & 15);
    const T* const w[2] = {(const T*)in.w + (row < in.outs ? row : in.outs - 1) * in.ldw + at,
                           PAIR ? (const T*)in.u + (row < in.outs ? row : in.outs - 1) * in.ldu + at : nullptr};
    const T* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int i = n * 16 + (lane & 15);
        x[n] = (const T*)in.x + (int64_t)(i < in.tokens ? i : in.tokens - 1) * in.ldx + at;
    }
    f32x4 acc[MATS][NT] = {};
    // Wave w takes the steps from w / 8 to (w + 1) / 8 of all.
    const int steps = (in.cols + P::K - 1) / P::K;
    const int s0 = steps * wave / kFewWaves, s1 = steps * (wave + 1) / kFewWaves;
    int s = s0;
    const auto some = [&](auto COUNT) {
        constexpr int C = decltype(COUNT)::value;
        P a[C][MATS], b[C][NT];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int k = (s + c) * P::K, left = in.cols - k - at;
#pragma unroll
            for (int m = 0; m < MATS; ++m) a[c][m].load(w[m] + k, left);
#pragma unroll
            for (int n = 0; n < NT; ++n) b[c][n].load(x[n] + k, left);
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int m = 0; m < MATS; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) P::mma(acc[m][n], a[c][m], b[c][n]);
        s += C;
    };
    while (s + U <= s1) some(std::integral_constant<int, U>());
    while (s < s1) some(std::integral_constant<int, 1>());
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) *reinterpret_cast<f32x4*>(sums[wave][m][n][lane]) = acc[m][n];
    __syncthreads();
    if ((int)threadIdx.x >= 64 * NT) return;
    const int n = threadIdx.x >> 6, token = n * 16 + (lane & 15);
    f32x4 v[2] = {};
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int k = 0; k < kFewWaves; ++k) v[m] += *reinterpret_cast<const f32x4*>(sums[k][m][n][lane]);
    if (token >= in.tokens) return;
    const int64_t c = row0 + (lane >> 4) * 4;
    const float z[4] = {v[0][0], v[0][1], v[0][2], v[0][3]}, u[4] = {v[1][0], v[1][1], v[1][2], v[1][3]};
    out.template store<4, PAIR>(token, c, left_of<4>(in.outs - c), z, u);
}

// ---------------------------------------------------------------- backward
struct DzOut {
    bf16 *dz, *dzt;            // [tokens][terms][matrices * kf], [matrices * outs][terms][kn] or null
    int64_t kf, kn;            // outs and tokens, padded to multiples of 64
    float* bias;               // [parts][outs] sums of dz over 16 WA tokens each, or null
    int chunks;                // fp32, tiles up to 128 x 128: parts of K that are summed by themselves
};

template <int WA, int RING, bool SPLIT, bool PAIR, typename T>
__global__ __launch_bounds__(256, 1) void dense_dz_kernel(Dense d, const T* __restrict__ dy, int64_t ldy, Bias bias,
                                                          int act, DzOut out) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using Q = Tile<WA, WA, RING, SPLIT, PAIR>;
    const Place at = place_of(blockIdx.x, d.p.ta, d.p.tb);
    Q t;
    const auto sum = [&](const Range& k) {
        t.multiply(d.p.A, d.A2, d.p.B, (int64_t)at.a * Q::kRowsA, (int64_t)at.b * Q::kB, k.s0, k.s1, d.p.stages, lds);
    };
    if constexpr (SPLIT && WA <= 4) {
        f32x4 total[WA][WA] = {};
#pragma unroll 1
        for (int n = 0; n < out.chunks; ++n) {
            sum(Range(d.p.stages, n, out.chunks));
#pragma unroll
            for (int i = 0; i < WA * WA; ++i) total[i / WA][i % WA] += t.acc[i / WA][i % WA];
        }
#pragma unroll
        for (int i = 0; i < WA * WA; ++i) t.acc[i / WA][i % WA] = total[i / WA][i % WA];
    } else sum(Range(d.p.stages, 0, 1));
    const int64_t a0 = (int64_t)at.a * Q::kRowsA + Q::lane_a(), b0 = (int64_t)at.b * Q::kB + Q::lane_b();
    const int64_t outs = d.p.A.rows, tokens = d.p.B.rows;
    constexpr int L = Q::kLaneA, kUp = PAIR ? WA / 2 : 0, MATS = PAIR ? 2 : 1;
    const int left = left_of<L>(outs - a0);
    constexpr int terms = SPLIT ? kTerms : 1;
    const bool again = out.dzt || out.bias;  // whether dz is needed back in the registers
    const Rows<WA, PAIR> rows(lds);
    const int64_t wa = (int64_t)at.a * Q::kRowsA + (threadIdx.x >> 7) * (Q::kRowsA / 2);
    const int64_t wb = (int64_t)at.b * Q::kB + ((threadIdx.x >> 6) & 1) * (Q::kB / 2);
    const int cols = left_of<8>(outs - wa - rows.c);     // of this lane's columns, how many exist
    float b[8] = {};
    if constexpr (!PAIR) bias.template load<8>(wa + rows.c, cols, b);
    rows.each(
        t.acc, again,
        [&](int row, int j) {
            Raw<T> r{};
            const int64_t token = wb + row * WA + j;
            if (cols && token < tokens) r.load(dy + token * ldy + wa + rows.c, cols);
            return r;
        },
        [&](int jj, int row, int j, float(&z)[8], float(&u)[8], const Raw<T>& raw) {
            const int64_t token = wb + row * WA + j;
            const int n = token < tokens ? cols : 0;
            float g[8];
            raw.get(g);
            with_activation(act, [&](auto A) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const Acted f = acted<decltype(A)::value, sizeof(T) == 4>(z[e] + b[e]);
                    // Selected: rows and columns past the end hold copies of the last one.
                    z[e] = e < n ? (PAIR ? g[e] * u[e] * f.d : g[e] * f.d) : 0.0f;
                    u[e] = e < n ? g[e] * f.a : 0.0f;
                }
            });
            if (again) rows.put(jj, row, z, u);
            if (out.dz && token < tokens && wa + rows.c < out.kf) {
                bf16* const dz = out.dz + token * terms * MATS * out.kf + wa + rows.c;
                store_terms<terms>(dz, MATS * out.kf, z);
                if constexpr (PAIR) store_terms<terms>(dz + out.kf, MATS * out.kf, u);
            }
        });
    if (!PAIR && out.bias) {
        const int64_t part = b0 / (16 * WA);
#pragma unroll
        for (int i = 0; i < WA; ++i) {
            f32x4 s = t.acc[i][0];
#pragma unroll
            for (int j = 1; j < WA; ++j) s += t.acc[i][j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
#pragma unroll
                for (int off = 1; off < 16; off *= 2) s[r] += __shfl_xor(s[r], off);
                if ((threadIdx.x & 15) == 0 && 4 * i + r < left) out.bias[part * outs + a0 + 4 * i + r] = s[r];
            }
        }
    }
#pragma unroll
    for (int term = 0; term < terms; ++term) {
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
            bf16* const dzt = out.dzt + term * out.kn + b0;
            if (out.dzt && b0 < out.kn)
#pragma unroll
                for (int i = 0; i < L; ++i)
                    if (i < left) {
                        typedef __bf16 V __attribute__((ext_vector_type(WA)));
                        V o;
#pragma unroll
                        for (int j = 0; j < WA; ++j) o[j] = term_of(t.acc[i / 4 + m * kUp][j][i & 3], term == terms - 1);
                        *reinterpret_cast<V*>(dzt + (m * outs + a0 + i) * terms * out.kn) = o;
                    }
        }
        if constexpr (SPLIT)
#pragma unroll
            for (int j = 0; j < WA; ++j)
#pragma unroll
                for (int i = 0; i < WA; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) t.acc[i][j][r] -= (float)term_of(t.acc[i][j][r], false);
    }
}

// fp32, K cut: dz (of both matrices) from the ranges' sums, in the place of the first range's.
template <bool PAIR>
__global__ __launch_bounds__(256) void dense_dz_join_kernel(float* slices, int n, int64_t rows, int cols, int64_t lda,
                                                            const float* __restrict__ dy, int64_t ldy, Bias bias,
                                                            int act) {
    const int64_t r = blockIdx.x;
    for (int c = (blockIdx.y * 256 + threadIdx.x) * 4; c < cols; c += gridDim.y * 1024) {
        float* const p = slices + r * lda + c;
        f32x4 z = sum_slices(p, n, rows * lda), u = PAIR ? sum_slices(p + lda / 2, n, rows * lda) : z;
        float g[4], b[4] = {};
        load_some<4>(dy + r * ldy + c, cols - c, g);
        if constexpr (!PAIR) bias.template load<4>(c, cols - c, b);
        with_activation(act, [&](auto A) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const Acted f = acted<decltype(A)::value, true>(z[e] + b[e]);
                z[e] = PAIR ? g[e] * u[e] * f.d : g[e] * f.d;
                u[e] = g[e] * f.a;
            }
        });
        // Past the last column up to a multiple of four there is room.
        *reinterpret_cast<f32x4*>(p) = z;
        if constexpr (PAIR) *reinterpret_cast<f32x4*>(p + lda / 2) = u;
    }
}

// Where a gradient goes: rows [0, rows) to one matrix, those from `second` on to another one.
template <typename T>
struct Target {
    T *one, *two;
    int64_t rows, second, ld;
    __device__ __forceinline__ T* row(int64_t r) const {  // null for a row that is none
        if (r >= second) return two && r - second < rows ? two + (r - second) * ld : nullptr;
        return r < rows ? one + r * ld : nullptr;
    }
};

// C[b][a] over one of gridDim.y ranges of K, whole (one range) or into the range's slice [ranges][B.rows][lda].
template <int WA, int RING, bool SPLIT, bool TA, bool TB, typename T>
__global__ __launch_bounds__(256, 1) void dense_grad_kernel(Product p, Target<T> out, float* __restrict__ slices,
                                                            int64_t lda) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using Q = Tile<WA, WA, RING, SPLIT, false, TA, TB>;
    const Place at = place_of(blockIdx.x, p.ta, p.tb);
    const Range k(p.stages);
    Q t;
    t.multiply(p.A, p.B, (int64_t)at.a * Q::kA, (int64_t)at.b * Q::kB, k.s0, k.s1, p.stages, lds);
    const int64_t a0 = (int64_t)at.a * Q::kA + Q::lane_a();
    const int64_t wa = (int64_t)at.a * Q::kA + (threadIdx.x >> 7) * (Q::kA / 2);
    const int64_t wb = (int64_t)at.b * Q::kB + ((threadIdx.x >> 6) & 1) * (Q::kB / 2);
    const int left = left_of<4 * WA>(p.A.rows - a0);
    if (slices) {
#pragma unroll
        for (int j = 0; j < WA; ++j) {
            const int64_t b = wb + Q::part_b(threadIdx.x & 15, j);
            if (b < p.B.rows) {
                f32x4* const q = reinterpret_cast<f32x4*>(slices + (blockIdx.y * p.B.rows + b) * lda + a0);
#pragma unroll
                for (int i = 0; i < WA; ++i)
                    if (4 * i < left) q[i] = t.acc[i][j];
            }
        }
        return;
    }
    const Rows<WA, false> rows(lds);
    const int n = left_of<8>(p.A.rows - wa - rows.c);
    rows.each(
        t.acc, false, [](int, int) { return Nothing(); },
        [&](int, int row, int j, const float(&z)[8], const float(&)[8], Nothing) {
            const int64_t b = wb + Q::part_b(row, j);
            T* const to = b < p.B.rows ? out.row(b) : nullptr;
            if (to && n) store_some<8>(to + wa + rows.c, n, z);
        });
}

template <typename T>
__global__ __launch_bounds__(256) void dense_slices_kernel(const float* __restrict__ slices, int n, int64_t rows,
                                                           int cols, int64_t lda, Target<T> out) {
    const int64_t r = blockIdx.x;
    T* const to = out.row(r);
    if (!to) return;
    for (int c = (blockIdx.y * 256 + threadIdx.x) * 4; c < cols; c += gridDim.y * 1024) {
        const f32x4 s = sum_slices(slices + r * lda + c, n, rows * lda);
        const float v[4] = {s[0], s[1], s[2], s[3]};
        store_some<4>(to + c, cols - c, v);
    }
}

// Sums of dy's columns over kBiasRows rows, four columns a lane: a part [outs] per blockIdx.y.
constexpr int kBiasRows = 128;
template <typename T>
__global__ __launch_bounds__(256) void dense_columns_kernel(const T* __restrict__ dy, int64_t ldy, int64_t tokens,
                                                            int64_t outs, float* __restrict__ parts) {
    __shared__ f32x4 sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * 4, r0 = (int64_t)blockIdx.y * kBiasRows;
    const int left = left_of<4>(outs - c);
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (left > 0)
        for (int64_t r = r0 + wave; r < r0 + kBiasRows && r < tokens; r += 4) {
            float f[4];
            load_some<4>(dy + r * ldy + c, left, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += f[e];
        }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave) return;
    s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) parts[blockIdx.y * outs + c + e] = s[e];
}
// dbias: the parts of 64 columns added up by 16 waves, each every 16th, and those in order.
__global__ __launch_bounds__(1024) void dense_bias_kernel(const float* __restrict__ parts, int64_t n, int64_t outs,
                                                          void* __restrict__ dbias, int bf) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < outs)
        for (int64_t k = wave; k < n; k += 16) s += parts[k * outs + c];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= outs) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    if (bf) ((bf16*)dbias)[c] = (bf16)s;
    else ((float*)dbias)[c] = s;
}

template <typename T>
__global__ __launch_bounds__(256) void dense_zero_kernel(T* p, int64_t ld, int64_t cols) {
    for (int64_t c = threadIdx.x; c < cols; c += 256) p[blockIdx.x * ld + c] = (T)0.0f;
}

// ---------------------------------------------------------------- host
constexpr const char* kNoLds = "dense product: no LDS for a tile";

struct Plan {
    int terms, products, mats;       // mats: 2 for the gated projection
    int64_t kd, kf, kn;              // cols, outs and tokens, padded
    bool few;                        // forward: the kernel for few tokens
    bool direct_x, direct_w, direct_dy;
    bool dz;                         // dz differs from dy
    bool turn;                       // bfloat16: operands are read across their rows, not transposed first
    int64_t rows_w;                  // rows of the weights' gradients as one matrix
    int chunks;                      // of K, in dense_dz_kernel
    bool cut;                        // fp32, backward: dz from ranges of K over workgroups
    Shape z, dx, dw;
};
struct Wanted {
    bool backward, dx, dw, db;
};

bool readable(int32_t dtype, int64_t cols, const void* p, int64_t ld) {
    return dtype == JORGE_BF16 && cols % kPadK == 0 && ld % 8 == 0 && aligned(p, 16);
}

bool weights_readable(const jorge_linear_shape& s, int mats, const void* weight, const void* up) {
    return readable(s.dtype, s.cols, weight, s.ldw) &&
           (mats == 1 || (readable(s.dtype, s.cols, up, s.ldu) && s.ldw == s.ldu));
}

// fp32: the fewest ranges of a sum over K, a power of two. The accumulator's roundings leave an error that grows with the
// root of K, 7e-7 of the sum at 2048 and 1.4e-6 at 8192; ranges of 1024 stay at 5e-7. Eight at most, and no more than
// 1 GiB of them, as each is kept in 32 bits (`sums` of them to a range, with the padding of its rows; 0: in registers).
int64_t ranges_for(int64_t k, int64_t sums) {
    int64_t r = 1;
    while (r < 8 && r * 1024 < k && 2 * r * sums * 4 <= int64_t(1) << 30) r *= 2;
    return r;
}

Plan plan_of(const jorge_linear_shape& s, int mats, const Wanted& want, bool direct_x, bool direct_w, bool direct_dy) {
    Plan p{};
    p.terms = s.dtype == JORGE_F32 ? kTerms : 1;
    p.products = s.dtype == JORGE_F32 ? 6 : 1;
    p.mats = mats;
    p.kd = round_up(s.cols, kPadK);
    p.kf = round_up(s.outs, kPadK);
    p.kn = round_up(s.tokens, kPadK);
    p.direct_x = direct_x;
    p.direct_w = direct_w;
    p.direct_dy = direct_dy;
    p.few = !want.backward && s.tokens <= kFewTokens;
    p.dz = mats == 2 || s.activation != JORGE_ACT_NONE;
    p.turn = p.terms == 1;
    p.rows_w = mats * (p.turn ? p.kf : s.outs);
    const auto least = [&](int64_t k, int64_t sums) { return p.terms == 1 ? 1 : ranges_for(k, sums); };
    const int64_t sums_z = mats * round_up(s.outs, 4) * s.tokens, wide = round_up(s.cols, 4);
    p.z = shape_of(mats * s.outs, s.tokens, p.kd, p.products, !want.backward, want.backward ? 1 : least(p.kd, sums_z));
    p.chunks = 1;
    if (want.backward && least(p.kd, 0) > 2) {
        // dz needs its sums whole, and a tile of 256 x 256 leaves no registers for sums of two parts of K.
        p.chunks = (int)least(p.kd, 0);
        if (p.z.blocks == 8) p.z.blocks = 4;
        p.z.deep = ceil_div(mats * s.outs, 32 * p.z.blocks) * ceil_div(s.tokens, 32 * p.z.blocks) <= kCus;
    }
    if (want.backward && p.dz && p.terms > 1) {
        // Where tiles leave CUs idle K is cut for dz too, which is then formed by a launch of its own and split by
        // another: 1515 tokens, 7854 -> 230, silu, both passes: 385 us whole, 324 cut.
        const Shape cut = shape_of(mats * s.outs, s.tokens, p.kd, p.products, true, least(p.kd, sums_z));
        const double more = 10.0 + (double)sums_z * 28.0 / 4.5e6;
        p.cut = cut.ranges > 1 && cut.us + more < p.z.us;
        if (p.cut) {
            p.z = cut;
            p.chunks = 1;
        }
    }
    // A pair's tile of 64 x 64 holds 32 columns of each, which padding to 64 would leave without a tile.
    if (mats == 2 && p.z.blocks == 2) p.z.blocks = 4;
    if (want.backward) {
        p.dx = shape_of(s.cols, s.tokens, mats * p.kf, p.products, true, least(mats * p.kf, wide * s.tokens));
        p.dw = shape_of(s.cols, p.rows_w, p.kn, p.products, true, least(p.kn, wide * p.rows_w));
    }
    return p;
}

struct Work {
    bf16 *x, *w, *u;          // K-contiguous copies
    bf16 *xt, *wt;            // transposes; wt: of both matrices side by side
    bf16 *dz, *dzt;
    float *z, *dx, *dw;       // slices; the three of a backward pass, each used up before the next, in one place
    float* bias;
    int64_t bytes, ldz, ldc;
};
int64_t bias_parts(const jorge_linear_shape& s, const Plan& p) {
    return p.dz && !p.cut ? ceil_div(s.tokens, 32 * p.z.blocks) * 2 : ceil_div(s.tokens, kBiasRows);
}
Work carve(void* base, const jorge_linear_shape& s, const Plan& p, const Wanted& want) {
    Carve c{(char*)base};
    Work w{};
    w.ldz = p.mats * round_up(s.outs, 4);
    w.ldc = round_up(s.cols, 4);
    const bool z = !want.backward || (p.dz && (want.dx || want.dw || want.db));
    if (!p.few) {
        if (!p.direct_x && (z || (p.turn && want.dw))) w.x = c.take<bf16>(p.terms * s.tokens * p.kd);
        if (!p.direct_w && (z || (p.turn && want.dx))) {
            w.w = c.take<bf16>(p.terms * s.outs * p.kd);
            if (p.mats == 2) w.u = c.take<bf16>(p.terms * s.outs * p.kd);
        }
    }
    if (!want.backward) {
        if (!p.few && p.z.ranges > 1) w.z = c.take<float>(p.z.ranges * s.tokens * w.ldz);
    } else {
        const bool dz = want.dx || (p.turn && want.dw);
        const int64_t slices_z = p.cut && z ? p.z.ranges * s.tokens * w.ldz : 0;
        const int64_t slices_dx = want.dx && p.dx.ranges > 1 ? p.dx.ranges * s.tokens * w.ldc : 0;
        const int64_t slices_dw = want.dw && p.dw.ranges > 1 ? p.dw.ranges * p.rows_w * w.ldc : 0;
        if (want.dw && !p.turn) w.xt = c.take<bf16>(p.terms * s.cols * p.kn);
        if (want.dx && !p.turn) w.wt = c.take<bf16>(p.terms * s.cols * p.mats * p.kf);
        if (dz && (p.dz || !p.direct_dy)) w.dz = c.take<bf16>(p.terms * s.tokens * p.mats * p.kf);
        if (want.dw && !p.turn) w.dzt = c.take<bf16>(p.terms * p.mats * s.outs * p.kn);
        float* const slices = c.take<float>(std::max({slices_z, slices_dx, slices_dw}));
        if (slices_z) w.z = slices;
        if (slices_dx) w.dx = slices;
        if (slices_dw) w.dw = slices;
        if (want.db) w.bias = c.take<float>(bias_parts(s, p) * s.outs);
    }
    w.bytes = c.used;
    return w;
}
// The plan of a call: what lies in whole pieces of 16 bytes is read in place. dy null: forward.
Plan plan_of(const jorge_linear_shape& s, const Wanted& want, const void* dy, const void* x, const void* weight,
             const void* up) {
    const int mats = up ? 2 : 1;
    return plan_of(s, mats, want, readable(s.dtype, s.cols, x, s.ldx), weights_readable(s, mats, weight, up),
                   dy && readable(s.dtype, s.outs, dy, s.ldy));
}
// Of any addresses and all gradients.
int64_t workspace_of(const jorge_linear_shape& s, int mats, bool backward) {
    const Wanted want{backward, backward, backward, backward && mats == 1};
    return carve(nullptr, s, plan_of(s, mats, want, false, false, false), want).bytes;
}

template <typename F>
void with_pair_tile(const Shape& s, F&& f) {
    if (s.blocks == 8) f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>());
    else if (s.deep) f(std::integral_constant<int, 4>(), std::integral_constant<int, 8>());
    else f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
}

// x and the weights as operands, K along their rows.
struct Operands {
    Operand x, w, u;
};
Operands operands_of(const jorge_linear_shape& s, const Plan& p, const Work& w, const void* x, const void* weight,
                     const void* up) {
    const auto of = [&](bool direct, const void* at, int64_t ld, const bf16* copy, int64_t rows) {
        return direct ? Operand{(const bf16*)at, ld, 0, rows} : Operand{copy, p.terms * p.kd, p.kd, rows};
    };
    return {of(p.direct_x, x, s.ldx, w.x, s.tokens), of(p.direct_w, weight, s.ldw, w.w, s.outs),
            of(p.direct_w, up, s.ldu, w.u, s.outs)};
}
// An operand of `depth` rows, K across them; of `cols` elements each.
Operand turned(const Operand& o, int64_t cols, int64_t depth, const bf16* p2 = nullptr, int64_t part = 0) {
    return {o.p, o.ld, 0, cols, p2, depth, part};
}
// The product of x with the weights: ta counts tiles of kRowsA rows.
Dense dense_of(const jorge_linear_shape& s, const Plan& p, const Operands& o) {
    Dense d{product_of(p.z, o.w, o.x, p.kd), p.mats == 2 ? o.u : o.w};
    d.p.ta = (int)ceil_div(s.outs, 32 * p.z.blocks / p.mats);
    return d;
}

template <typename T, bool PAIR>
jorge_status forward(const jorge_linear_shape& s, const Plan& p, const Work& w, const void* x, const void* weight,
                     const void* up, const Finish<T>& out, hipStream_t st) {
    if (p.few) {
        const FewRows in{x, weight, up, s.ldx, s.ldw, s.ldu, s.outs, (int)s.tokens, (int)s.cols};
        const dim3 grid((unsigned)ceil_div(s.outs, 16)), block(kFewWaves * 64);
        if (s.tokens <= 16) dense_few_kernel<T, 1, PAIR><<<grid, block, 0, st>>>(in, out);
        else if (s.tokens <= 32) dense_few_kernel<T, 2, PAIR><<<grid, block, 0, st>>>(in, out);
        else dense_few_kernel<T, 4, PAIR><<<grid, block, 0, st>>>(in, out);
        return launched("dense product");
    }
    copy<T>(copies_of(x, s.ldx, s.tokens, s.cols, w.x, p.kd, nullptr, 0),
            copies_of(weight, s.ldw, s.outs, s.cols, w.w, p.kd, nullptr, 0), st,
            copies_of(up, s.ldu, s.outs, s.cols, w.u, p.kd, nullptr, 0));
    const Dense d = dense_of(s, p, operands_of(s, p, w, x, weight, up));
    jorge_status err = JORGE_OK;
    const int ranges = p.z.ranges;
    const auto run = [&](auto WA, auto RING) {
        constexpr int B = decltype(WA)::value, R = decltype(RING)::value, bytes = Tile<B, B, R, sizeof(T) == 4>::kBytes;
        const auto k = dense_forward_kernel<B, R, sizeof(T) == 4, PAIR, T>;
        if ((err = allow_lds(k, bytes, kNoLds)) != JORGE_OK) return;
        k<<<dim3(d.p.ta * d.p.tb, ranges), dim3(256), bytes, st>>>(d, out, w.z, w.ldz);
    };
    if constexpr (PAIR) with_pair_tile(p.z, run);
    else with_tile(p.z, run);
    if (err != JORGE_OK) return err;
    if (w.z)
        dense_join_kernel<PAIR, T><<<dim3((unsigned)s.tokens, (unsigned)ceil_div(s.outs, 1024)), dim3(256), 0, st>>>(
            w.z, ranges, s.tokens, (int)s.outs, w.ldz, out);
    return launched("dense product");
}

template <typename T, bool TA, bool TB>
jorge_status gradient(const Shape& sh, const Product& pr, const Target<T>& out, int64_t cols, float* slices,
                      hipStream_t st) {
    jorge_status err = JORGE_OK;
    const int64_t lda = round_up(cols, 4);
    with_tile(sh, [&](auto WA, auto RING) {
        constexpr int B = decltype(WA)::value, R = decltype(RING)::value, bytes = Tile<B, B, R, sizeof(T) == 4>::kBytes;
        const auto k = dense_grad_kernel<B, R, sizeof(T) == 4, TA, TB, T>;
        if ((err = allow_lds(k, bytes, kNoLds)) != JORGE_OK) return;
        k<<<dim3(pr.ta * pr.tb, sh.ranges), dim3(256), bytes, st>>>(pr, out, slices, lda);
    });
    if (err == JORGE_OK && slices)
        dense_slices_kernel<T><<<dim3((unsigned)pr.B.rows, (unsigned)ceil_div(cols, 1024)), dim3(256), 0, st>>>(
            slices, sh.ranges, pr.B.rows, (int)cols, lda, out);
    return err;
}

struct Gradients {
    void *dx, *dweight, *dup, *dbias;
    int64_t lddx, lddw;
};

template <typename T, bool PAIR>
jorge_status backward(const jorge_linear_shape& s, const Plan& p, const Work& w, const void* dy, const void* x,
                      const void* weight, const void* up, const Bias& bias, const Gradients& out, hipStream_t st) {
    const int64_t kz = p.mats * p.kf;
    bf16* const ut = w.wt && PAIR ? w.wt + p.kf : nullptr;
    copy<T>(copies_of(x, s.ldx, s.tokens, s.cols, w.x, p.kd, w.xt, p.kn),
            copies_of(weight, s.ldw, s.outs, s.cols, w.w, p.kd, w.wt, kz), st,
            PAIR ? copies_of(up, s.ldu, s.outs, s.cols, w.u, p.kd, ut, kz)
                 : p.dz ? Copies{} : copies_of(dy, s.ldy, s.tokens, s.outs, w.dz, p.kf, w.dzt, p.kn));
    const Operands in = operands_of(s, p, w, x, weight, up);
    jorge_status err = JORGE_OK;
    if constexpr (sizeof(T) == 4) {
        if (p.cut) {
            const Dense d = dense_of(s, p, in);
            const auto run = [&](auto WA, auto RING) {
                constexpr int B = decltype(WA)::value, R = decltype(RING)::value, bytes = Tile<B, B, R, true>::kBytes;
                const auto k = dense_forward_kernel<B, R, true, PAIR, T>;
                if ((err = allow_lds(k, bytes, kNoLds)) != JORGE_OK) return;
                k<<<dim3(d.p.ta * d.p.tb, p.z.ranges), dim3(256), bytes, st>>>(d, Finish<T>{}, w.z, w.ldz);
            };
            if constexpr (PAIR) with_pair_tile(p.z, run);
            else with_tile(p.z, run);
            if (err != JORGE_OK) return err;
            dense_dz_join_kernel<PAIR><<<dim3((unsigned)s.tokens, (unsigned)ceil_div(s.outs, 1024)), dim3(256), 0, st>>>(
                w.z, p.z.ranges, s.tokens, (int)s.outs, w.ldz, (const T*)dy, s.ldy, bias, s.activation);
            Copies split[2] = {};
            for (int m = 0; m < p.mats; ++m) {
                split[m] = copies_of(w.z + m * (w.ldz / 2), w.ldz, s.tokens, s.outs, w.dz ? w.dz + m * p.kf : nullptr,
                                     p.kf, w.dzt ? w.dzt + m * s.outs * p.terms * p.kn : nullptr, p.kn);
                split[m].padded_f = kz;
            }
            copy<T>(split[0], split[1], st);
            if (w.bias)
                dense_columns_kernel<T><<<dim3((unsigned)ceil_div(s.outs, 256), (unsigned)bias_parts(s, p)), dim3(256),
                                          0, st>>>(w.z, w.ldz, s.tokens, s.outs, w.bias);
        }
    }
    if (p.dz && !p.cut) {
        const Dense d = dense_of(s, p, in);
        const DzOut z{w.dz, w.dzt, p.kf, p.kn, w.bias, p.chunks};
        const auto run = [&](auto WA, auto RING) {
            constexpr int B = decltype(WA)::value, R = decltype(RING)::value;
            constexpr int bytes = Tile<B, B, R, sizeof(T) == 4>::kBytes;
            const auto k = dense_dz_kernel<B, R, sizeof(T) == 4, PAIR, T>;
            if ((err = allow_lds(k, bytes, kNoLds)) != JORGE_OK) return;
            k<<<dim3(d.p.ta * d.p.tb), dim3(256), bytes, st>>>(d, (const T*)dy, s.ldy, bias, s.activation, z);
        };
        if constexpr (PAIR) with_pair_tile(p.z, run);
        else with_tile(p.z, run);
        if (err != JORGE_OK) return err;
    } else if (!p.dz && w.bias) {
        dense_columns_kernel<T><<<dim3((unsigned)ceil_div(s.outs, 256), (unsigned)bias_parts(s, p)), dim3(256), 0,
                                  st>>>((const T*)dy, s.ldy, s.tokens, s.outs, w.bias);
    }
    if (out.dbias)
        dense_bias_kernel<<<dim3((unsigned)ceil_div(s.outs, 64)), dim3(1024), 0, st>>>(
            w.bias, bias_parts(s, p), s.outs, out.dbias, bias.bf);
    constexpr bool TURN = sizeof(T) == 2;
    const Operand z = w.dz ? Operand{w.dz, p.terms * kz, kz, s.tokens} : Operand{(const bf16*)dy, s.ldy, 0, s.tokens};
    if (out.dx) {
        const Operand a = TURN ? turned(in.w, s.cols, s.outs, PAIR ? in.u.p : nullptr, p.kf)
                               : Operand{w.wt, p.terms * kz, kz, s.cols};
        const Target<T> to{(T*)out.dx, nullptr, s.tokens, INT64_MAX, out.lddx};
        err = gradient<T, TURN, false>(p.dx, product_of(p.dx, a, z, kz), to, s.cols, w.dx, st);
        if (err != JORGE_OK) return err;
    }
    if (out.dweight) {
        const Operand a = TURN ? turned(in.x, s.cols, s.tokens) : Operand{w.xt, p.terms * p.kn, p.kn, s.cols};
        const Operand zt = TURN ? turned(z, p.rows_w, s.tokens) : Operand{w.dzt, p.terms * p.kn, p.kn, p.rows_w};
        const Target<T> to{(T*)out.dweight, (T*)out.dup, s.outs, p.rows_w / p.mats, out.lddw};
        err = gradient<T, TURN, TURN>(p.dw, product_of(p.dw, a, zt, p.kn), to, s.cols, w.dw, st);
        if (err != JORGE_OK) return err;
    }
    return launched("dense product");
}

jorge_status check(const jorge_linear_shape* s, bool gated) {
    if (!s) return bad("linear: a shape is needed");
    if (!known_dtype(s->dtype)) return bad("linear: unknown element type");
    if (!gated && !known_dtype(s->bias_dtype)) return bad("linear: unknown element type of the bias");
    if (s->activation < JORGE_ACT_NONE || s->activation > JORGE_ACT_SIGMOID) return bad("linear: unknown activation");
    if (s->tokens < 0 || s->cols < 1 || s->outs < 1)
        return bad("linear: tokens >= 0, cols >= 1 and outs >= 1 are needed");
    if (s->tokens > JORGE_LINEAR_MAX_TOKENS)
        return refuse(JORGE_ERR_UNSUPPORTED, "linear: tokens above JORGE_LINEAR_MAX_TOKENS");
    if (s->cols > JORGE_LINEAR_MAX_COLS) return refuse(JORGE_ERR_UNSUPPORTED, "linear: cols above JORGE_LINEAR_MAX_COLS");
    if (s->outs > JORGE_LINEAR_MAX_OUTS) return refuse(JORGE_ERR_UNSUPPORTED, "linear: outs above JORGE_LINEAR_MAX_OUTS");
    if (ceil_div(s->tokens, 64) * ceil_div(std::max(s->cols, s->outs), 64) > 1 << 22)
        return refuse(JORGE_ERR_UNSUPPORTED, "linear: tokens * max(cols, outs) above 2^34");
    const int64_t strides[] = {s->ldx, s->ldw, gated ? s->ldu : s->ldw, s->ldy}, least[] = {s->cols, s->cols, s->cols,
                                                                                            s->outs};
    for (int i = 0; i < 4; ++i) {
        if (strides[i] < least[i]) return bad("linear: a row stride is below its columns");
        if (strides[i] > JORGE_LINEAR_MAX_STRIDE)
            return refuse(JORGE_ERR_UNSUPPORTED, "linear: a row stride above JORGE_LINEAR_MAX_STRIDE (2^22)");
    }
    return JORGE_OK;
}
jorge_status check_workspace(int64_t need, const void* workspace, int64_t bytes) {
    if (need == 0) return JORGE_OK;
    if (!workspace || !aligned(workspace, kAlign)) return bad("linear: a workspace aligned to 256 bytes is needed");
    if (bytes < need) return bad("linear: the workspace is too small");
    return JORGE_OK;
}

jorge_status run_forward(const jorge_linear_shape& s, int mats, const void* x, const void* weight, const void* up,
                         const void* bias, const void* residual, void* y, void* workspace, int64_t bytes, void* stream) {
    const int64_t e = dtype_bytes(s.dtype);
    if (s.tokens == 0) return JORGE_OK;
    if (!x || !weight || !y || (mats == 2 && !up)) return bad("linear: x, the weights and y are needed");
    if (!aligned(x, e) || !aligned(weight, e) || !aligned(up, e) || !aligned(y, e) || !aligned(residual, e) ||
        !aligned(bias, dtype_bytes(s.bias_dtype)))
        return bad("linear: a pointer is not aligned to its element");
    if (residual && (s.ldr < s.outs)) return bad("linear: a row stride is below its columns");
    const Wanted want{false, false, false, false};
    const Plan p = plan_of(s, want, nullptr, x, weight, up);
    const jorge_status st = check_workspace(carve(nullptr, s, p, want).bytes, workspace, bytes);
    if (st != JORGE_OK) return st;
    const Work w = carve(workspace, s, p, want);
    const hipStream_t q = reinterpret_cast<hipStream_t>(stream);
    const Bias b{bias, s.bias_dtype == JORGE_BF16};
    if (s.dtype == JORGE_F32) {
        const Finish<float> f{b, (const float*)residual, (float*)y, s.ldr, s.ldy, s.activation};
        return mats == 2 ? forward<float, true>(s, p, w, x, weight, up, f, q)
                         : forward<float, false>(s, p, w, x, weight, up, f, q);
    }
    const Finish<bf16> f{b, (const bf16*)residual, (bf16*)y, s.ldr, s.ldy, s.activation};
    return mats == 2 ? forward<bf16, true>(s, p, w, x, weight, up, f, q)
                     : forward<bf16, false>(s, p, w, x, weight, up, f, q);
}

template <typename T>
void zero(void* p, int64_t rows, int64_t ld, int64_t cols, hipStream_t q) {
    if (p) dense_zero_kernel<T><<<dim3((unsigned)rows), dim3(256), 0, q>>>((T*)p, ld, cols);
}

jorge_status run_backward(const jorge_linear_shape& s, int mats, const void* dy, const void* x, const void* weight,
                          const void* up, const void* bias, const Gradients& g, void* workspace, int64_t bytes,
                          void* stream) {
    const int64_t e = dtype_bytes(s.dtype);
    if (!aligned(g.dx, e) || !aligned(g.dweight, e) || !aligned(g.dup, e) ||
        !aligned(g.dbias, dtype_bytes(s.bias_dtype)) || !aligned(bias, dtype_bytes(s.bias_dtype)))
        return bad("linear: a pointer is not aligned to its element");
    if (mats == 2 && !g.dweight != !g.dup) return bad("gated linear: dgate and dup go together");
    if ((g.dx && g.lddx < s.cols) || (g.dweight && g.lddw < s.cols))
        return bad("linear: a row stride is below its columns");
    const hipStream_t q = reinterpret_cast<hipStream_t>(stream);
    if (s.tokens == 0) {
        if (s.dtype == JORGE_F32) {
            zero<float>(g.dweight, s.outs, g.lddw, s.cols, q);
            zero<float>(g.dup, s.outs, g.lddw, s.cols, q);
        } else {
            zero<bf16>(g.dweight, s.outs, g.lddw, s.cols, q);
            zero<bf16>(g.dup, s.outs, g.lddw, s.cols, q);
        }
        if (s.bias_dtype == JORGE_F32) zero<float>(g.dbias, 1, s.outs, s.outs, q);
        else zero<bf16>(g.dbias, 1, s.outs, s.outs, q);
        return launched("dense product");
    }
    if (!dy || !x || !weight || (mats == 2 && !up)) return bad("linear: dy, x and the weights are needed");
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(weight, e) || !aligned(up, e))
        return bad("linear: a pointer is not aligned to its element");
    const Wanted want{true, g.dx != nullptr, g.dweight != nullptr, g.dbias != nullptr};
    if (!want.dx && !want.dw && !want.db) return JORGE_OK;
    const Plan p = plan_of(s, want, dy, x, weight, up);
    const jorge_status st = check_workspace(carve(nullptr, s, p, want).bytes, workspace, bytes);
    if (st != JORGE_OK) return st;
    const Work w = carve(workspace, s, p, want);
    const Bias b{bias, s.bias_dtype == JORGE_BF16};
    if (s.dtype == JORGE_F32)
        return mats == 2 ? backward<float, true>(s, p, w, dy, x, weight, up, b, g, q)
                         : backward<float, false>(s, p, w, dy, x, weight, up, b, g, q);
    return mats == 2 ? backward<bf16, true>(s, p, w, dy, x, weight, up, b, g, q)
                     : backward<bf16, false>(s, p, w, dy, x, weight, up, b, g, q);
}

}  // namespace
}  // namespace jorge_lm

using namespace jorge_lm;

extern "C" {

jorge_status jorge_linear_workspace(const jorge_linear_shape* shape, int32_t gated, int32_t backward, int64_t* bytes) {
    if (!bytes) return bad("linear: bytes is needed");
    const jorge_status st = check(shape, gated != 0);
    if (st != JORGE_OK) return st;
    *bytes = shape->tokens ? workspace_of(*shape, gated ? 2 : 1, backward != 0) : 0;
    return JORGE_OK;
}

jorge_status jorge_linear_call_workspace(const jorge_linear_shape* shape, const void* dy, const void* x,
                                         const void* weight, const void* up, int32_t wanted, int64_t* bytes) {
    if (!bytes) return bad("linear: bytes is needed");
    const jorge_status st = check(shape, up != nullptr);
    if (st != JORGE_OK) return st;
    const Wanted want{dy != nullptr, dy && (wanted & JORGE_LINEAR_DX), dy && (wanted & JORGE_LINEAR_DWEIGHT),
                      dy && !up && (wanted & JORGE_LINEAR_DBIAS)};
    const bool any = !dy || want.dx || want.dw || want.db;
    *bytes = shape->tokens && any ? carve(nullptr, *shape, plan_of(*shape, want, dy, x, weight, up), want).bytes : 0;
    return JORGE_OK;
}

jorge_status jorge_linear_forward(const jorge_linear_shape* shape, const void* x, const void* weight, const void* bias,
                                  const void* residual, void* y, void* workspace, int64_t workspace_bytes,
                                  void* hip_stream) {
    const jorge_status st = check(shape, false);
    if (st != JORGE_OK) return st;
    return run_forward(*shape, 1, x, weight, nullptr, bias, residual, y, workspace, workspace_bytes, hip_stream);
}

jorge_status jorge_linear_backward(const jorge_linear_shape* shape, const void* dy, const void* x, const void* weight,
                                   const void* bias, void* dx, int64_t lddx, void* dweight, int64_t lddw, void* dbias,
                                   void* workspace, int64_t workspace_bytes, void* hip_stream) {
    const jorge_status st = check(shape, false);
    if (st != JORGE_OK) return st;
    return run_backward(*shape, 1, dy, x, weight, nullptr, bias, {dx, dweight, nullptr, dbias, lddx, lddw}, workspace,
                        workspace_bytes, hip_stream);
}

jorge_status jorge_gated_linear_forward(const jorge_linear_shape* shape, const void* x, const void* gate,
                                        const void* up, void* y, void* workspace, int64_t workspace_bytes,
                                        void* hip_stream) {
    const jorge_status st = check(shape, true);
    if (st != JORGE_OK) return st;
    return run_forward(*shape, 2, x, gate, up, nullptr, nullptr, y, workspace, workspace_bytes, hip_stream);
}

jorge_status jorge_gated_linear_backward(const jorge_linear_shape* shape, const void* dy, const void* x,
                                         const void* gate, const void* up, void* dx, int64_t lddx, void* dgate,
                                         void* dup, int64_t lddw, void* workspace, int64_t workspace_bytes,
                                         void* hip_stream) {
    const jorge_status st = check(shape, true);
    if (st != JORGE_OK) return st;
    return run_backward(*shape, 2, dy, x, gate, up, nullptr, {dx, dgate, dup, nullptr, lddx, lddw}, workspace,
                        workspace_bytes, hip_stream);
}

}  // extern "C"
