// Softmax attention, forward and backward, for gfx950: o = softmax(scale q k^T) v over the keys that a query sees, and
// its gradients with the probabilities formed again from the row's log sum exp.
//
// One side of each product is a wave's own and stays in registers: 32 rows of q (forward, dq) or 32 keys (dk, dv),
// one to a lane of 32. The other side is streamed through LDS, a tile of rows at a time. With the own rows as the
// columns of every product, two products do everything:
//   rows:  S[i][n] = sum_d tile[i][d] own[n][d]       (scores, do v^T)
//   cols:  C[d][n] += sum_i tile[i][d] P[i][n]        (o, dq, dk, dv)
// The MFMA leaves S with lane l holding column l % 32 and rows 8 g + 4 (l / 32) + r of 32; cols takes its right operand
// from just those registers, as the order of a sum over i is free: no probability ever moves between lanes. Softmax
// needs one exchange per tile and row, of the maximum.
//
//   forward:  S = rows(k, q), P = exp(S - m), o += cols(v, P), with the running maximum m and sum of the row
//   dq:       S = rows(k, q), dP = rows(v, do), dS = P (dP - delta), dq += cols(k, dS)
//   dk, dv:   S = rows(q, k), dP = rows(do, v), dv += cols(do, P), dk += cols(q, dS)
// with delta = do . o of a row, which dq forms at its start and leaves for dk and dv. Both backward kernels form S and
// dP: seven products where one kernel would do with five, but that one has to add dq up by atomics, whose order would
// change results.
//
// Bound by the matrix cores and the exponentials between their products in training. 4 sequences of 4096, 16 heads of
// 128, causal, bfloat16: forward 375 us (734 TFLOP/s over what is not masked; matrix cores busy 46%), dq 477 us (864;
// 56%), dk and dv 778 us (706; 39%: one wave to a SIMD has nothing to cover its own softmax with). No bank conflicts in
// any of them. A single token over 32 caches is bound by reading k and v: 158 us for 0.8 GB, 5.1 TB/s. Times that are
// set against each other below are of one session; sessions differ by up to 10%.
//
// Queries whose heads share a key head are rows of one sequence of own rows, (token, head) by (token, head), so that a
// tile of k and v is read once for all of them.
//
// A tile in LDS holds its rows one after the other, their 16-byte chunks permuted by the row's number, so that both
// reads meet no bank twice: `rows` reads 16 bytes of 32 rows, `cols` 4 rows of 32 elements across (transposed by
// ds_read_tr16 for bfloat16). Rows past the end, and elements past dim, come as zeros from the bounds check of the
// loads.
//
// bfloat16: P and dS are rounded to bfloat16 for `cols`, as the matrix instructions take them; scores, statistics and
// sums are fp32. fp32 runs on the fp32 MFMAs throughout, and sums a tile before the long sum. exp2 gives no subnormal
// numbers: a probability below 2^-126 of the row's reference (forward) or of 1 (backward) is 0.
#include "lm_common.hpp"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace jorge_lm {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_any;

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr int kOwn = 32;           // own rows of a wave
constexpr unsigned kNowhere = 0x80000000u;  // an offset that the bounds check turns into zeros

// ---------------------------------------------------------------- arguments
struct Heads {
    char* p;
    int64_t batch, token, head;    // strides in bytes
};

// What the kernels know of the call.
struct Call {
    const int64_t *q_lengths, *kv_lengths;
    int batch, q_tokens, kv_tokens, heads, kv_heads, group, dim;
    int causal, window;            // window: 0 for none
    float scale, scale2, scale2_low;  // scale; scale log2(e), and what its rounding left out
};

// A sequence's own lengths and where its queries stand.
struct Sequence {
    int nq, nk, off;               // query t stands at position off + t
    __device__ __forceinline__ Sequence(const Call& c, int b) {
        const auto of = [&](const int64_t* p, int most) {
            const int64_t n = p ? p[b] : most;
            return (int)(n < 0 ? 0 : n > most ? most : n);
        };
        nq = of(c.q_lengths, c.q_tokens);
        nk = of(c.kv_lengths, c.kv_tokens);
        off = nk - nq;
    }
    // The keys that query t sees: [lo, hi).
    __device__ __forceinline__ int lo(const Call& c, int t) const {
        return c.window ? max(0, off + t - c.window + 1) : 0;
    }
    __device__ __forceinline__ int hi(const Call& c, int t) const {
        return t < 0 || t >= nq ? 0 : c.causal ? max(0, min(nk, off + t + 1)) : nk;
    }
    // The queries that see key k: [first, last).
    __device__ __forceinline__ int first(const Call& c, int k) const { return c.causal ? max(0, k - off) : 0; }
    __device__ __forceinline__ int last(const Call& c, int k) const {
        return k >= nk ? 0 : c.window ? (int)min((int64_t)nq, (int64_t)k - off + c.window) : nq;
    }
};

// Workgroup g's place: the key head (of all sequences), and the tile of its own rows. Workgroup g runs on XCD g mod 8:
// tiles that read the same keys are put on one, so that they do so from one L2, and key heads are dealt out in turn, so
// that a batch of unequal sequences loads all XCDs alike (5 sequences of up to 2011 with a window of 512: 47 us forward
// and 210 us backward, where an equal run of key heads for each XCD took 50 and 221); the last ones, if they are no
// multiple of eight, are spread tile by tile. Where the last tiles have the most to do they come first.
struct Work {
    int bh, tile;
    __device__ __forceinline__ Work(int g, int total, int tiles, int heaviest_last) {
        const int heads = total / tiles, whole = heads / 8, n = g / 8, x = g % 8;
        if (n < whole * tiles) {
            bh = n / tiles * 8 + x;
            tile = n % tiles;
        } else {
            const int rest = (n - whole * tiles) * 8 + x;
            bh = whole * 8 + rest / tiles;
            tile = rest % tiles;
        }
        if (heaviest_last) tile = tiles - 1 - tile;
    }
};

// ---------------------------------------------------------------- tiles
// 4 rows of 16 elements, 8 bytes from each of 16 lanes, to lane i's column i of each row. In a function with a
// restricted pointer: without what that says of aliases the compiler waits here for every direct-to-LDS load in flight.
__device__ __forceinline__ s16x4 read_turned4(const lds_s16x4* __restrict__ p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<lds_s16x4*>(p));
}

template <int N>
__device__ __forceinline__ void clear(f32x16 (&acc)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] = 0.0f;
}

// Rows of D elements (32, 64, 96 or 128).
template <typename T, int D>
struct Tile {
    static constexpr int kRow = (D <= 64 ? 64 : 128) * (int)sizeof(T);  // bytes of a row in LDS
    static constexpr int kChunks = kRow / 16;
    static constexpr int kRows = sizeof(T) == 2 ? 64 : 32;
    static constexpr int kBlocks = kRows / 32;
    static constexpr int kBytes = kRows * kRow;
    static constexpr int kLoads = kBytes / 1024;          // wave-wide loads of 16 bytes a lane
    static constexpr int kSteps = D * (int)sizeof(T) / 32;  // of rows(): 16 bytes of either half of a wave
    static constexpr int kDims = D / 32;                  // blocks of 32 elements of a row

    // What a row's chunk numbers are exclusive-ored with.
    static __device__ __forceinline__ int swizzle(int row) {
        if constexpr (sizeof(T) == 4) return ((row >> 2 & 1) << 3) | ((row >> 3 & 1) << 2) | (row & 3);
        else if constexpr (kRow == 256) return ((row & 3) << 2) | (row >> 2 & 3);
        else return ((row >> 1 & 1) << 2) | (row >> 2 & 3);
    }

    // The loads of a tile by WAVES waves, this one the w-th: byte offsets from the tile's first row.
    template <int WAVES>
    struct Loader {
        static constexpr int kEach = kLoads / WAVES;
        const char* base;
        int64_t stride;
        unsigned off[kEach];
        int row0;
        __device__ __forceinline__ Loader(const char* p, int64_t token, int dim, int w) : base(p), stride(token) {
            const int lane = threadIdx.x & 63;
            row0 = w * kEach * (64 / kChunks) + lane / kChunks;
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                const int row = row0 + v * (64 / kChunks), chunk = (lane % kChunks) ^ swizzle(row);
                off[v] = chunk * 16 < dim * (int)sizeof(T) ? (unsigned)row * (unsigned)token + chunk * 16u : kNowhere;
            }
        }
        // Rows [first, ..) of the operand to a tile in LDS; zeros in the place of rows outside [begin, end).
        __device__ __forceinline__ void load(int first, int begin, int end, char* tile, int w) const {
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<char*>(base + first * stride), 0, 0x7fffffff, 0x00020000);
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                const int row = first + row0 + v * (64 / kChunks);
                const bool there = row >= begin && row < end;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_any*)(tile + (w * kEach + v) * 1024), 16,
                                                         there ? off[v] : kNowhere, 0, 0, 0);
            }
        }
    };

    // A lane's own row: its halves of every 32 bytes.
    typedef typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type Frag;
    struct Own {
        Frag f[kSteps];
        __device__ __forceinline__ void load(const char* row, bool there, int dim) {
            const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int at = k * 32 + half * 16;
                if (there && at < dim * (int)sizeof(T)) f[k] = *reinterpret_cast<const Frag*>(row + at);
                else
#pragma unroll
                    for (int e = 0; e < (int)(16 / sizeof(T)); ++e) f[k][e] = (T)0.0f;
            }
        }
    };

    // Where this lane's reads of a tile start.
    int at_rows, at_cols;
    __device__ __forceinline__ Tile() {
        const int lane = threadIdx.x & 63, row = lane & 31, half = lane >> 5;
        at_rows = row * kRow + ((half ^ swizzle(row)) * 16);
        if constexpr (sizeof(T) == 2) {
            const int i = lane & 15, key = 4 * half + i / 4, chunk = (lane >> 4 & 1) * 2 + (i & 3) / 2;
            at_cols = key * kRow + ((chunk ^ swizzle(key)) * 16) + (i & 1) * 8;
        } else {
            at_cols = 4 * half * kRow + (((row / 4) ^ (half << 3)) * 16) + (row & 3) * 4;
        }
    }

    // S of block kb (32 rows of the tile).
    __device__ __forceinline__ f32x16 rows(const char* tile, int kb, const Own& own) const {
        f32x16 s;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const Frag a = *reinterpret_cast<const Frag*>(tile + (at_rows ^ (k * 32)) + kb * 32 * kRow);
            if constexpr (sizeof(T) == 2) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, own.f[k], s, 0, 0, 0);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], own.f[k][e], s, 0, 0, 0);
        }
        return s;
    }

    // S of every block of the tile. The reads run ahead of the products by one block's (327 us for a forward pass of 338
    // where each waits for its own: 4 sequences of 4096, 16 heads of 128, causal).
    __device__ __forceinline__ void all_rows(const char* tile, const Own& own, f32x16 (&s)[kBlocks]) const {
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) s[kb] = rows(tile, kb, own);
        if constexpr (sizeof(T) == 2) {
            __builtin_amdgcn_sched_group_barrier(0x100, kSteps, 0);
#pragma unroll
            for (int i = 0; i < (kBlocks - 1) * kSteps; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, kSteps, 0);
        } else order_rows(kBlocks);
    }
    // fp32: four products to a read; the reads run four ahead.
    static __device__ __forceinline__ void order_rows(int products) {
        constexpr int kAhead = 4;
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int i = 0; i < products * kSteps - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4 * kAhead, 0);
    }

    // The order of a backward kernel's two products by rows: the reads of one run while the one before it does.
    static __device__ __forceinline__ void order() {
        if constexpr (sizeof(T) == 2) {
            __builtin_amdgcn_sched_group_barrier(0x100, kSteps, 0);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, kSteps, 0);
        } else order_rows(2);
    }

    // acc[db] += the tile's rows of block kb, elements 32 db .., times p.
    __device__ __forceinline__ void cols(const char* tile, int kb, const f32x16& p, f32x16 (&acc)[kDims]) const {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                bf16x8 b;
#pragma unroll
                for (int e = 0; e < 8; ++e) b[e] = (bf16)p[8 * t + e];
#pragma unroll
                for (int db = 0; db < kDims; ++db) {
                    s16x4 v[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const char* const at =
                            tile + ((at_cols ^ (db * 64) ^ (u * 32)) + (kb * 32 + t * 16 + u * 8) * kRow);
                        v[u] = read_turned4((const lds_s16x4*)at);
                    }
                    typedef short s16x8 __attribute__((ext_vector_type(8)));
                    const s16x8 a = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), b, acc[db], 0, 0,
                                                                      0);
                }
            }
            // The reads run 4 products ahead.
            constexpr int kAhead = 4;
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 0);
#pragma unroll
            for (int i = 0; i < 2 * kDims - kAhead; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
        } else {
            // The tile's own sum first: added one by one to the long sum, the products would take sixteen times the
            // roundings of it (o of 16384 keys erred by 2.4e-6 of its size, and so by 5.7e-7; forward of 2 sequences of
            // 4096, 16 heads of 128, causal, takes 1434 us instead of 1390 and backward 5112 instead of 4959). Where the
            // reads alone may pass from one block of elements to the next, there is one such sum at a time: two would
            // spill.
            constexpr int kAhead = 8;
#pragma unroll
            for (int db = 0; db < kDims; ++db) {
                f32x16 part;
#pragma unroll
                for (int r = 0; r < 16; ++r) part[r] = 0.0f;
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float a = *reinterpret_cast<const float*>(
                            tile + ((at_cols ^ (db * 128) ^ ((g & 1) * 64) ^ (r * 16)) + (kb * 32 + g * 8 + r) * kRow));
                        part = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[4 * g + r], part, 0, 0, 0);
                    }
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] += part[r];
                __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
                for (int i = 0; i < 16 - kAhead; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
                __builtin_amdgcn_sched_barrier(0x100);
            }
        }
    }

    // Whether a lane's column holds a NaN (both lanes of it know).
    static __device__ __forceinline__ bool spoilt(const f32x16 (&acc)[kDims]) {
        bool found = false;
#pragma unroll
        for (int db = 0; db < kDims; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) found |= acc[db][r] != acc[db][r];
        return found | (bool)__shfl_xor((int)found, 32);
    }
    // A sum that cols() forms, formed again without the rows that a lane does not see: acc = sum of weight(i) times row i
    // of x over the lane's own i of [first, last), element by element. 0 times an infinity or a NaN is a NaN, so a row
    // with one among those of a tile at a mask's edge spoils the sums of the columns that do not see it. Called after all
    // tiles, for columns with a NaN in their sum that nothing of their own explains. `again`: acc is added to.
    template <typename W>
    static __device__ __forceinline__ void add_seen(f32x16 (&acc)[kDims], bool again, const char* x, int64_t stride,
                                                    int first, int last, int dim, W&& weight) {
        typedef T V __attribute__((ext_vector_type(4)));
        const int half = (threadIdx.x & 63) >> 5;
        if (!again) clear(acc);
#pragma unroll 1
        for (int i = first; i < last; ++i) {
            const float w = weight(i);
            const T* const row = reinterpret_cast<const T*>(x + i * stride);
#pragma unroll
            for (int db = 0; db < kDims; ++db)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int at = db * 32 + g * 8 + half * 4;
                    if (at >= dim) continue;
                    const V v = *reinterpret_cast<const V*>(row + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[db][4 * g + e] = __builtin_fmaf(w, (float)v[e], acc[db][4 * g + e]);
                }
        }
    }
    // The product of two rows, by the two lanes that share a column.
    static __device__ __forceinline__ float dot(const char* a, const char* b, int dim) {
        typedef T V __attribute__((ext_vector_type(4)));
        float s = 0.0f;
#pragma unroll 1
        for (int at = ((threadIdx.x & 63) >> 5) * 4; at < dim; at += 8) {
            const V x = reinterpret_cast<const V*>(a)[at / 4], y = reinterpret_cast<const V*>(b)[at / 4];
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_fmaf((float)x[e], (float)y[e], s);
        }
        return s + __shfl_xor(s, 32);
    }

    // Row n's elements of acc times f, to a row of T or of floats; zeros for a row that has no part in anything, whose
    // sums are zeros times what the other rows meet.
    template <typename O>
    static __device__ __forceinline__ void store(const f32x16 (&acc)[kDims], O* row, int dim, float f, bool live) {
        typedef O V __attribute__((ext_vector_type(4), aligned(sizeof(O))));
        const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
        for (int db = 0; db < kDims; ++db)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int at = db * 32 + g * 8 + half * 4;
                if (at + 4 <= dim) {
                    V v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (O)(live ? acc[db][4 * g + e] * f : 0.0f);
                    *reinterpret_cast<V*>(row + at) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (at + e < dim) row[at + e] = (O)(live ? acc[db][4 * g + e] * f : 0.0f);
                }
            }
    }
};

// The tile row that register r of a lane's block holds.
__device__ __forceinline__ int row_of(int r) { return 8 * (r / 4) + 4 * ((threadIdx.x & 63) >> 5) + (r & 3); }

template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Tiles [t0, t1) of a range of streamed rows [lo, hi) cut into `of` parts, the y-th.
struct Span {
    int lo, hi, t0, t1;
    __device__ __forceinline__ Span(int lo, int hi, int rows, int y, int of) : lo(lo), hi(hi) {
        const int a = lo / rows, n = hi > lo ? (hi + rows - 1) / rows - a : 0;
        t0 = a + (int)((int64_t)n * y / of);
        t1 = a + (int)((int64_t)n * (y + 1) / of);
    }
    // The part's rows of a lane's [first, last).
    __device__ __forceinline__ int from(int first, int rows) const { return max(first, t0 * rows); }
    __device__ __forceinline__ int to(int last, int rows) const { return min(last, t1 * rows); }
};

__device__ __forceinline__ void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Streamed tiles through a ring of two stages of BYTES: fetch(tile, stage) starts a tile's loads, body(tile, stage) uses
// it. All waves have to call it; the barrier says that a stage has landed for all and that the one before it is free.
template <int BYTES, typename G, typename F>
__device__ __forceinline__ void stream(const Span& span, char* lds, G&& fetch, F&& body) {
    if (span.t0 >= span.t1) return;
    wait_lds();
    barrier();
    fetch(span.t0, lds + (span.t0 & 1) * BYTES);
    for (int t = span.t0; t < span.t1; ++t) {
        wait_lds();
        wait_loads<0>();
        barrier();
        if (t + 1 < span.t1) fetch(t + 1, lds + ((t + 1) & 1) * BYTES);
        body(t, lds + (t & 1) * BYTES);
    }
}

// What stream() fetches: a tile of two operands, one after the other.
template <typename TILE>
struct Two {
    typename TILE::template Loader<4> one, two;
    int begin, end, wave;
    __device__ __forceinline__ void operator()(int t, char* to) const {
        one.load(t * TILE::kRows, begin, end, to, wave);
        two.load(t * TILE::kRows, begin, end, to + TILE::kBytes, wave);
    }
};

// Both, and behind them the rows' log2 sum exp and delta: 256 bytes each, waves 0 and 1 bring one each.
template <typename TILE>
struct TwoAndRows {
    Two<TILE> tiles;
    const float* of_rows;          // the wave's
    __device__ __forceinline__ void operator()(int t, char* to) const {
        tiles(t, to);
        if (tiles.wave > 1) return;
        const int lane = threadIdx.x & 63;
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<float*>(of_rows + t * TILE::kRows), 0, 256, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_any*)(to + 2 * TILE::kBytes + tiles.wave * 256), 4,
                                                 t * TILE::kRows + lane < tiles.end ? lane * 4 : kNowhere, 0, 0, 0);
    }
};

// exp(scale s - lse) from a score and the row's log2 sum exp.
template <typename T>
__device__ __forceinline__ float probability(const Call& c, float s, float lse2) {
    float z = __builtin_fmaf(s, c.scale2, -lse2);
    if constexpr (sizeof(T) == 4) z = __builtin_fmaf(s, c.scale2_low, z);
    return __builtin_amdgcn_exp2f(z);
}

// ---------------------------------------------------------------- forward
// A row's running softmax: the reference `base` (log2) that its sum and output are relative to, and the sum over the
// lane's own keys.
template <typename TILE>
struct Softmax {
    // How far (log2) a score may stand above the reference before everything is scaled down to it: sums of 2^8 and
    // products with them are as exact, and most tiles need no scaling.
    static constexpr float kRoom = 8.0f;
    float base, sum;
    f32x16 acc[TILE::kDims];
    __device__ __forceinline__ Softmax() : base(-INFINITY), sum(0.0f) { clear(acc); }

    // Scores (before scaling) to probabilities relative to `base`. A lane sees rows [lo, hi) from k0 on.
    template <typename T>
    __device__ __forceinline__ void tile(const Call& c, f32x16 (&s)[TILE::kBlocks], int k0, int lo, int hi) {
        if (__any(k0 < lo || k0 + TILE::kRows > hi))
#pragma unroll
            for (int kb = 0; kb < TILE::kBlocks; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int k = k0 + kb * 32 + row_of(r);
                    s[kb][r] = k >= lo && k < hi ? s[kb][r] : -INFINITY;
                }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < TILE::kBlocks; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
        top = fmaxf(top, __shfl_xor(top, 32)) * c.scale2;
        const bool higher = top > base + kRoom || (base == -INFINITY && top > base);
        if (__any(higher)) {
            // For the columns that need it alone: a row's result does not depend on the others of its wave.
            const float f = higher ? __builtin_amdgcn_exp2f(base - top) : 1.0f;
            base = higher ? top : base;
            sum *= f;
#pragma unroll
            for (int db = 0; db < TILE::kDims; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= f;
        }
        float add = 0.0f;
#pragma unroll
        for (int kb = 0; kb < TILE::kBlocks; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = weight<T>(c, s[kb][r]);
                add += s[kb][r];
            }
        sum += add;
    }
    // A score's exponential, relative to the reference.
    template <typename T>
    __device__ __forceinline__ float weight(const Call& c, float s) const {
        float z = __builtin_fmaf(s, c.scale2, base == -INFINITY ? 0.0f : -base);
        // A masked score stays at minus infinity, whatever the low part's sign.
        if constexpr (sizeof(T) == 4) z = s == -INFINITY ? z : __builtin_fmaf(s, c.scale2_low, z);
        return __builtin_amdgcn_exp2f(z);
    }
};

// A row's place: its query's token and head.
struct Row {
    int token, head;
    bool there;                    // a row of the matrix (its token may be past the sequence's end)
    __device__ __forceinline__ Row(const Call& c, int bh, int r) {
        token = r / c.group;
        head = bh % c.kv_heads * c.group + r - token * c.group;
        there = token < c.q_tokens;
    }
};

// Where a forward pass leaves its results: o and lse, or, where the keys are cut into ranges, o of a range's keys alone
// [range][key head][row][D], and its log2 sum exp.
struct Output {
    Heads o;
    float* lse;
    float *part, *part_lse;
};

// Four waves of 32 rows, all keys of the range; or (SPLIT) 32 rows for which every wave takes every fourth tile of keys.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attention_forward_kernel(Call c, Heads q, Heads k, Heads v, Output out,
                                                                   int tiles) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using L = Tile<T, D>;
    const Work at(blockIdx.x, gridDim.x, tiles, c.causal);
    const int b = at.bh / c.kv_heads, hk = at.bh % c.kv_heads;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const Sequence s(c, b);
    const int row0 = at.tile * 4 * kOwn, r = row0 + wave * kOwn + (lane & 31);
    const Row row(c, at.bh, r);
    const int lo = s.lo(c, row.token), hi = s.hi(c, row.token);
    const int first = row0 / c.group, last = min((row0 + 4 * kOwn - 1) / c.group, s.nq - 1);
    const Span span(s.lo(c, first), first < s.nq ? s.hi(c, last) : 0, L::kRows, blockIdx.y, gridDim.y);
    const L tile;
    typename L::Own own;
    const char* const qp = q.p + b * q.batch + row.token * q.token + row.head * q.head;
    own.load(qp, row.there, c.dim);
    const Two<L> fetch{{k.p + b * k.batch + hk * k.head, k.token, c.dim, wave},
                       {v.p + b * v.batch + hk * v.head, v.token, c.dim, wave}, span.lo, span.hi, wave};
    Softmax<L> soft;
    stream<2 * L::kBytes>(span, lds, fetch, [&](int t, const char* kt) {
        const int k0 = t * L::kRows;
        const char* const vt = kt + L::kBytes;
        if (!__any(k0 < hi && k0 + L::kRows > lo)) return;
        f32x16 z[L::kBlocks];
        tile.all_rows(kt, own, z);
        soft.template tile<T>(c, z, k0, lo, hi);
#pragma unroll
        for (int kb = 0; kb < L::kBlocks; ++kb) tile.cols(vt, kb, z[kb], soft.acc);
    });
    if (!row.there) return;
    if (L::spoilt(soft.acc) && soft.sum == soft.sum) {
        const char* const kp = k.p + b * k.batch + hk * k.head;
        L::add_seen(soft.acc, false, v.p + b * v.batch + hk * v.head, v.token, span.from(lo, L::kRows),
                    span.to(hi, L::kRows), c.dim, [&](int i) {
                        return soft.template weight<T>(c, L::dot(qp, kp + i * k.token, c.dim));
                    });
    }
    const float sum = soft.sum + __shfl_xor(soft.sum, 32);
    // A row that sees nothing is zero, its log sum exp minus infinity.
    const float f = hi > lo && soft.base != -INFINITY ? 1.0f / sum : hi > lo && sum != sum ? sum : 0.0f;
    const float lse2 = hi > lo ? (soft.base == -INFINITY ? log2f(sum) : soft.base + log2f(sum)) : -INFINITY;
    if (out.part) {
        const int64_t rows = (int64_t)c.q_tokens * c.group;
        const int64_t to = ((int64_t)blockIdx.y * c.batch * c.kv_heads + at.bh) * rows + r;
        L::store(soft.acc, out.part + to * D, D, f, hi > lo);
        if (lane < 32) out.part_lse[to] = lse2;
        return;
    }
    L::store(soft.acc, reinterpret_cast<T*>(out.o.p + b * out.o.batch + row.token * out.o.token +
                                            row.head * out.o.head), c.dim, f, hi > lo);
    if (lane < 32) out.lse[((int64_t)b * c.heads + row.head) * c.q_tokens + row.token] = lse2 * kLn2;
}

// Few rows (at most 32 to a key head): every wave takes every fourth tile of the range's keys with a stage of its own,
// of which k is loaded again as soon as the scores are formed, and v as soon as they are used; the waves' results are
// joined in LDS. Bound by reading k and v.
template <typename T, int D>
__global__ __launch_bounds__(256, 1) void attention_few_kernel(Call c, Heads q, Heads k, Heads v, Output out) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using L = Tile<T, D>;
    const Work at(blockIdx.x, gridDim.x, 1, 0);
    const int b = at.bh / c.kv_heads, hk = at.bh % c.kv_heads;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const Sequence s(c, b);
    const Row row(c, at.bh, lane & 31);
    const int lo = s.lo(c, row.token), hi = s.hi(c, row.token);
    const Span span(s.lo(c, 0), s.hi(c, min((kOwn - 1) / c.group, s.nq - 1)), L::kRows, blockIdx.y, gridDim.y);
    const L tile;
    typename L::Own own;
    const char* const qp = q.p + b * q.batch + row.token * q.token + row.head * q.head;
    own.load(qp, row.there, c.dim);
    const typename L::template Loader<1> lk(k.p + b * k.batch + hk * k.head, k.token, c.dim, 0);
    const typename L::template Loader<1> lv(v.p + b * v.batch + hk * v.head, v.token, c.dim, 0);
    char *const kt = lds + wave * 2 * L::kBytes, *const vt = kt + L::kBytes;
    Softmax<L> soft;
    int t = span.t0 + wave;
    if (t < span.t1) {
        lk.load(t * L::kRows, span.lo, span.hi, kt, 0);
        lv.load(t * L::kRows, span.lo, span.hi, vt, 0);
    }
    for (; t < span.t1; t += 4) {
        // Where no tile is left the loads bring zeros, and are not used: the numbers in flight stay the same.
        const int next = t + 4 < span.t1 ? (t + 4) * L::kRows : span.hi;
        wait_loads<L::kLoads>();
        f32x16 z[L::kBlocks];
#pragma unroll
        for (int kb = 0; kb < L::kBlocks; ++kb) z[kb] = tile.rows(kt, kb, own);
        wait_lds();
        lk.load(next, span.lo, span.hi, kt, 0);
        const int k0 = t * L::kRows;
        soft.template tile<T>(c, z, k0, lo, hi);
        wait_loads<L::kLoads>();
#pragma unroll
        for (int kb = 0; kb < L::kBlocks; ++kb) tile.cols(vt, kb, z[kb], soft.acc);
        wait_lds();
        lv.load(next, span.lo, span.hi, vt, 0);
    }
    wait_loads<0>();
    if (L::spoilt(soft.acc) && soft.sum == soft.sum && row.there) {
        const char* const kp = k.p + b * k.batch + hk * k.head;
        clear(soft.acc);
        for (int n = span.t0 + wave; n < span.t1; n += 4)
            L::add_seen(soft.acc, true, v.p + b * v.batch + hk * v.head, v.token, max(lo, n * L::kRows),
                        min(hi, (n + 1) * L::kRows), c.dim, [&](int i) {
                            return soft.template weight<T>(c, L::dot(qp, kp + i * k.token, c.dim));
                        });
    }
    __syncthreads();
    // The waves' references, sums and outputs: [wave][row], [wave][row][D + 4].
    float* const refs = reinterpret_cast<float*>(lds);
    float* const sums = refs + 4 * kOwn;
    float* const outs = sums + 4 * kOwn;
    const float sum = soft.sum + __shfl_xor(soft.sum, 32);
    if (lane < 32) {
        refs[wave * kOwn + lane] = soft.base;
        sums[wave * kOwn + lane] = sum;
    }
    L::store(soft.acc, outs + (wave * kOwn + (lane & 31)) * (D + 4), D, 1.0f, true);
    __syncthreads();
    const int64_t rows = (int64_t)c.q_tokens * c.group;
    for (int i = threadIdx.x; i < kOwn * D / 4; i += 256) {
        const int n = i / (D / 4), d = i % (D / 4) * 4;
        if (n >= rows) break;
        const Row to(c, at.bh, n);
        float top = -INFINITY, total = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, refs[w * kOwn + n]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(refs[w * kOwn + n] - base);
            // A wave without a key above minus infinity has a sum of 0, or of NaN.
            total += refs[w * kOwn + n] == -INFINITY ? sums[w * kOwn + n] : sums[w * kOwn + n] * f;
            const f32x4 x = *reinterpret_cast<const f32x4*>(outs + (w * kOwn + n) * (D + 4) + d);
            o += x * f;
        }
        const bool seen = s.hi(c, to.token) > s.lo(c, to.token) && (top != -INFINITY || total != total);
        const float f = seen ? 1.0f / total : 0.0f, lse2 = seen ? base + log2f(total) : -INFINITY;
        float e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = seen ? o[j] * f : 0.0f;
        if (out.part) {
            const int64_t p = ((int64_t)blockIdx.y * c.batch * c.kv_heads + at.bh) * rows + n;
#pragma unroll
            for (int j = 0; j < 4; ++j) out.part[p * D + d + j] = e[j];
            if (d == 0) out.part_lse[p] = lse2;
            continue;
        }
        T* const o_row = reinterpret_cast<T*>(out.o.p + b * out.o.batch + to.token * out.o.token + to.head * out.o.head);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < c.dim) o_row[d + j] = (T)e[j];
        if (d == 0) out.lse[((int64_t)b * c.heads + to.head) * c.q_tokens + to.token] = lse2 * kLn2;
    }
}

// Joins the ranges' outputs of a row, 32 lanes to it, in order.
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(Call c, Output out, int ranges) {
    const int64_t rows = (int64_t)c.q_tokens * c.group, all = rows * c.batch * c.kv_heads;
    const int64_t id = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (id >= all) return;
    const int bh = (int)(id / rows), b = bh / c.kv_heads, d = (threadIdx.x & 31) * 4;
    const Row to(c, bh, (int)(id - bh * rows));
    float top = -INFINITY;
    for (int k = 0; k < ranges; ++k) top = fmaxf(top, out.part_lse[k * all + id]);
    const float base = top == -INFINITY ? 0.0f : top;
    float total = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < ranges; ++k) {
        const float f = __builtin_amdgcn_exp2f(out.part_lse[k * all + id] - base);
        total += f;
        if (d < D) o += *reinterpret_cast<const f32x4*>(out.part + (k * all + id) * D + d) * f;
    }
    const bool none = total == 0.0f;
    T* const row = reinterpret_cast<T*>(out.o.p + b * out.o.batch + to.token * out.o.token + to.head * out.o.head);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (d + e < c.dim) row[d + e] = (T)(none ? 0.0f : o[e] / total);
    if (d == 0)
        out.lse[((int64_t)b * c.heads + to.head) * c.q_tokens + to.token] = none ? -INFINITY
                                                                                 : (base + log2f(total)) * kLn2;
}

// ---------------------------------------------------------------- backward
// A row's log2 sum exp for dk and dv. A row whose q or gradient is not finite has a lse or a delta that is not: it counts
// as a NaN, which attention_dkv_kernel goes by.
__device__ __forceinline__ float stat_of(float lse, float delta) {
    const float x = lse * kLog2e;
    return __builtin_fabsf(x) < INFINITY && __builtin_fabsf(delta) < INFINITY ? x : __builtin_nanf("");
}

// delta = do . o, [batch][head][token], where o cannot be read in whole pieces of 16 bytes. Two lanes to a row, which add
// it up as attention_dq_kernel does where that reads o: the results are the same to the bit.
template <typename T>
__global__ __launch_bounds__(256) void attention_delta_kernel(Call c, Heads o, Heads g, float* __restrict__ delta) {
    const int64_t id = (int64_t)blockIdx.x * 128 + (threadIdx.x >> 1);
    if (id >= (int64_t)c.batch * c.heads * c.q_tokens) return;
    // Neighbouring rows are heads of a token, as they lie in memory.
    const int h = (int)(id % c.heads);
    const int64_t bt = id / c.heads;
    const int t = (int)(bt % c.q_tokens), b = (int)(bt / c.q_tokens);
    const Sequence s(c, b);
    const T* const po = reinterpret_cast<const T*>(o.p + b * o.batch + t * o.token + h * o.head);
    const T* const pg = reinterpret_cast<const T*>(g.p + b * g.batch + t * g.token + h * g.head);
    const int64_t at = ((int64_t)b * c.heads + h) * c.q_tokens + t;
    const bool seen = s.hi(c, t) > s.lo(c, t);
    constexpr int N = 16 / sizeof(T);
    float sum = 0.0f;
    if (seen)
        for (int d = (threadIdx.x & 1) * N; d < c.dim; d += 2 * N) {
            typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
            if (d + N <= c.dim) {
                const V x = *reinterpret_cast<const V*>(po + d), y = *reinterpret_cast<const V*>(pg + d);
#pragma unroll
                for (int e = 0; e < N; ++e) sum = __builtin_fmaf((float)x[e], (float)y[e], sum);
            } else {
                for (int e = d; e < c.dim; ++e) sum = __builtin_fmaf((float)po[e], (float)pg[e], sum);
            }
        }
    sum += __shfl_xor(sum, 1);
    if (!(threadIdx.x & 1)) delta[at] = seen ? sum : 0.0f;
}

// Gradients of rows of one matrix: to it, or, where the streamed side is cut into ranges, the range's sums
// [range][head of it, of all sequences][row][D].
struct Gradient {
    Heads g;
    float* part;
};

// A row's log2 sum exp (plus infinity where it sees nothing, so that every probability is 0) and delta, [batch][head]
// [token], which attention_dq_kernel leaves for attention_dkv_kernel. delta is formed from the row's o and gradient, which
// saves reading the gradient twice, or (no o) is there from attention_delta_kernel. o's rounding to bfloat16 puts an
// error into delta that is an average over the keys that a row sees; where a workgroup's rows see few (kFewTiles), delta
// is the sum of p dp instead, formed in a pass of its own: without it dq errs by 3.8e-3 of its size where rows see 2
// keys and by 2.6e-3 at 96, with it by 2.3e-3 to 2.4e-3, as it does with more keys.
constexpr int kFewTiles = 4;
struct RowStats {
    Heads o;
    const float* lse;
    float *lse2, *delta;
};

// dq absent: only the rows' statistics.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(Call c, Heads q, Heads k, Heads v, Heads g,
                                                              RowStats stats, Gradient dq, int tiles) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using L = Tile<T, D>;
    const Work at(blockIdx.x, gridDim.x, tiles, c.causal);
    const int b = at.bh / c.kv_heads, hk = at.bh % c.kv_heads;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const Sequence s(c, b);
    const int row0 = at.tile * 4 * kOwn, r = row0 + wave * kOwn + (lane & 31);
    const Row row(c, at.bh, r);
    const int lo = s.lo(c, row.token), hi = s.hi(c, row.token);
    const int first = row0 / c.group, last = min((row0 + 4 * kOwn - 1) / c.group, s.nq - 1);
    const Span span(s.lo(c, first), first < s.nq ? s.hi(c, last) : 0, L::kRows, blockIdx.y, gridDim.y);
    const L tile;
    typename L::Own own, grad;
    const char* const qp = q.p + b * q.batch + row.token * q.token + row.head * q.head;
    const char* const gp = g.p + b * g.batch + row.token * g.token + row.head * g.head;
    own.load(qp, row.there, c.dim);
    // A row that sees nothing has no part in anything, whatever its gradient is.
    grad.load(gp, row.there && hi > lo, c.dim);
    const Two<L> fetch{{k.p + b * k.batch + hk * k.head, k.token, c.dim, wave},
                       {v.p + b * v.batch + hk * v.head, v.token, c.dim, wave}, span.lo, span.hi, wave};
    const int64_t stat = ((int64_t)b * c.heads + row.head) * c.q_tokens + row.token;
    float l2 = INFINITY, de = 0.0f;
    const Span all(span.lo, span.hi, L::kRows, 0, 1);
    const bool few = sizeof(T) == 2 && all.t1 - all.t0 <= kFewTiles;
    if (stats.o.p) {
        typename L::Own o;
        o.load(stats.o.p + b * stats.o.batch + row.token * stats.o.token + row.head * stats.o.head,
               row.there && hi > lo, c.dim);
#pragma unroll
        for (int n = 0; n < L::kSteps; ++n)
#pragma unroll
            for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
                de = __builtin_fmaf((float)o.f[n][e], (float)grad.f[n][e], de);
        de += __shfl_xor(de, 32);
        if (row.there && hi > lo) l2 = stats.lse[stat] * kLog2e;
    } else if (row.there) {
        l2 = hi > lo ? stats.lse[stat] * kLog2e : INFINITY;
        de = stats.delta[stat];
    }
    if constexpr (sizeof(T) == 2) {
        if (few) {
            de = 0.0f;
            stream<2 * L::kBytes>(all, lds, fetch, [&](int t, const char* kt) {
                const int k0 = t * L::kRows;
                if (!__any(k0 < hi && k0 + L::kRows > lo)) return;
#pragma unroll
                for (int kb = 0; kb < L::kBlocks; ++kb) {
                    const f32x16 z = tile.rows(kt, kb, own), dp = tile.rows(kt + L::kBytes, kb, grad);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int key = k0 + kb * 32 + row_of(i);
                        de += key >= lo && key < hi ? probability<T>(c, z[i], l2) * dp[i] : 0.0f;
                    }
                }
            });
            de += __shfl_xor(de, 32);
        }
    }
    if (row.there && lane < 32 && blockIdx.y == 0) {
        stats.lse2[stat] = hi > lo ? stat_of(stats.lse[stat], de) : INFINITY;
        stats.delta[stat] = de;
    }
    if (!dq.g.p) return;
    f32x16 acc[L::kDims];
    clear(acc);
    stream<2 * L::kBytes>(span, lds, fetch, [&](int t, const char* kt) {
        const int k0 = t * L::kRows;
        const char* const vt = kt + L::kBytes;
        if (!__any(k0 < hi && k0 + L::kRows > lo)) return;
        const bool edge = __any(k0 < lo || k0 + L::kRows > hi);
#pragma unroll
        for (int kb = 0; kb < L::kBlocks; ++kb) {
            f32x16 z = tile.rows(kt, kb, own);
            const f32x16 dp = tile.rows(vt, kb, grad);
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = probability<T>(c, z[i], l2) * (dp[i] - de);
            L::order();
            if (edge) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = k0 + kb * 32 + row_of(i);
                    z[i] = key >= lo && key < hi ? z[i] : 0.0f;
                }
            }
            tile.cols(kt, kb, z, acc);
        }
    });
    if (!row.there) return;
    if (L::spoilt(acc) && l2 == l2 && de == de) {
        const char *const kp = k.p + b * k.batch + hk * k.head, *const vp = v.p + b * v.batch + hk * v.head;
        L::add_seen(acc, false, kp, k.token, span.from(lo, L::kRows), span.to(hi, L::kRows), c.dim, [&](int i) {
            const float p = probability<T>(c, L::dot(qp, kp + i * k.token, c.dim), l2);
            return p * (L::dot(gp, vp + i * v.token, c.dim) - de);
        });
    }
    if (dq.part) {
        const int64_t rows = (int64_t)c.q_tokens * c.group;
        L::store(acc, dq.part + (((int64_t)blockIdx.y * c.batch * c.kv_heads + at.bh) * rows + r) * D, D, c.scale,
                 hi > lo);
        return;
    }
    L::store(acc, reinterpret_cast<T*>(dq.g.p + b * dq.g.batch + row.token * dq.g.token + row.head * dq.g.head), c.dim,
             c.scale, hi > lo);
}

// Zeros in the place of the rows of a stage whose log2 sum exp is a NaN, in q's and the gradient's tile: 0 times an
// infinity or a NaN is a NaN, which must not reach a key that does not see the row; p of one that does is a NaN by
// itself. Every wave that uses the stage at a mask's edge writes the same zeros before it reads.
template <typename TILE>
__device__ __forceinline__ void without_spoilt_rows(char* stage) {
    const int lane = threadIdx.x & 63;
    const float* const stats = reinterpret_cast<const float*>(stage + 2 * TILE::kBytes);
    const float mine = lane < TILE::kRows ? stats[lane] : 0.0f;
    uint64_t bad = __ballot(mine != mine);
    while (bad) {
        const int row = __builtin_ctzll(bad);
        bad &= bad - 1;
        for (int at = lane * 4; at < 2 * TILE::kRow; at += 256) {
            const int tile = at >= TILE::kRow;
            *reinterpret_cast<float*>(stage + tile * TILE::kBytes + row * TILE::kRow + at - tile * TILE::kRow) = 0.0f;
        }
    }
}

// Two waves to a SIMD where their registers allow it (a wave's k, v and sums of dk and dv take D of them for every four
// bytes of T): with D = 96 in bfloat16 that takes 111 us where one wave takes 128 (5 sequences of up to 2011, 12 heads
// of 80, window 512). At D = 128 two would spill in the loop (1.7 times the time); eight waves to a workgroup that keep
// v in LDS instead took as long as four with one to a SIMD, and the exponentials of one block put between the products of
// the next took 738 us for 687 (4 sequences of 4096, 16 heads, causal).
template <typename T, int D>
__global__ __launch_bounds__(256, D <= (sizeof(T) == 2 ? 96 : 64) ? 2 : 1) void attention_dkv_kernel(
    Call c, Heads q, Heads k, Heads v, Heads g, const float* __restrict__ lse2, const float* __restrict__ delta,
    Gradient dk, Gradient dv, int tiles) {
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    using L = Tile<T, D>;
    const Work at(blockIdx.x, gridDim.x, tiles, 0);
    const int b = at.bh / c.kv_heads, hk = at.bh % c.kv_heads;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const Sequence s(c, b);
    const int key0 = at.tile * 4 * kOwn, key = key0 + wave * kOwn + (lane & 31);
    const bool there = key < c.kv_tokens;
    const int lo = s.first(c, key), hi = s.last(c, key);
    const Span span(s.first(c, key0), key0 < s.nk ? s.last(c, min(key0 + 4 * kOwn, s.nk) - 1) : 0, L::kRows, blockIdx.y,
                    gridDim.y);
    const L tile;
    typename L::Own own, val;
    // Keys past the sequence's end may hold anything.
    own.load(k.p + b * k.batch + key * k.token + hk * k.head, key < s.nk, c.dim);
    val.load(v.p + b * v.batch + key * v.token + hk * v.head, key < s.nk, c.dim);
    f32x16 ak[L::kDims], av[L::kDims];
    clear(ak);
    clear(av);
    for (int h = hk * c.group; h < (hk + 1) * c.group; ++h) {
        const TwoAndRows<L> fetch{{{q.p + b * q.batch + h * q.head, q.token, c.dim, wave},
                                   {g.p + b * g.batch + h * g.head, g.token, c.dim, wave}, span.lo, span.hi, wave},
                                  (wave ? delta : lse2) + ((int64_t)b * c.heads + h) * c.q_tokens};
        stream<2 * L::kBytes + 512>(span, lds, fetch, [&](int t, const char* qt) {
            const int t0 = t * L::kRows;
            const char *const gt = qt + L::kBytes, *const st = gt + L::kBytes;
            if (!__any(t0 < hi && t0 + L::kRows > lo)) return;
            const bool edge = __any(t0 < lo || t0 + L::kRows > hi);
            if (edge) without_spoilt_rows<L>(const_cast<char*>(qt));
#pragma unroll
            for (int kb = 0; kb < L::kBlocks; ++kb) {
                f32x16 z = tile.rows(qt, kb, own), dp = tile.rows(gt, kb, val);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const f32x4* const at = reinterpret_cast<const f32x4*>(st + (kb * 32 + row_of(4 * n)) * 4);
                    const f32x4 l2 = at[0], de = at[16];
#pragma unroll
                    for (int i = 4 * n; i < 4 * n + 4; ++i) {
                        z[i] = probability<T>(c, z[i], l2[i & 3]);
                        dp[i] = z[i] * (dp[i] - de[i & 3]);
                    }
                }
                L::order();
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int row = t0 + kb * 32 + row_of(i);
                        const bool seen = row >= lo && row < hi;
                        z[i] = seen ? z[i] : 0.0f;
                        dp[i] = seen ? dp[i] : 0.0f;
                    }
                }
                tile.cols(gt, kb, z, av);
                tile.cols(qt, kb, dp, ak);
            }
        });
    }
    if (!there) return;
    const int64_t to = (((int64_t)blockIdx.y * c.batch * c.kv_heads + at.bh) * c.kv_tokens + key) * D;
    const auto write = [&](const f32x16(&acc)[L::kDims], const Gradient& out, float f) {
        if (out.part) L::store(acc, out.part + to, D, f, key < s.nk);
        else if (out.g.p)
            L::store(acc, reinterpret_cast<T*>(out.g.p + b * out.g.batch + key * out.g.token + hk * out.g.head), c.dim, f,
                     key < s.nk);
    };
    write(ak, dk, c.scale);
    write(av, dv, 1.0f);
}

// The sum of the ranges' gradients of a row, 32 lanes to it, in order; of two matrices (blockIdx.y), of which one may be
// none. group: rows of a token.
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_sum_kernel(Gradient one, Gradient two, int ranges, int64_t rows,
                                                            int64_t all, int kv_heads, int group, int dim) {
    const Gradient& out = blockIdx.y ? two : one;
    const int64_t id = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (id >= all || !out.part) return;
    const int bh = (int)(id / rows), b = bh / kv_heads, r = (int)(id - bh * rows), d = (threadIdx.x & 31) * 4;
    if (d >= D) return;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < ranges; ++k) s += *reinterpret_cast<const f32x4*>(out.part + (k * all + id) * D + d);
    const int token = r / group, head = bh % kv_heads * group + r % group;
    T* const row = reinterpret_cast<T*>(out.g.p + b * out.g.batch + token * out.g.token + head * out.g.head);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (d + e < dim) row[d + e] = (T)s[e];
}

// A copy of a matrix of heads with rows of `width` elements (a multiple of 16 bytes, zeros past dim), as the kernels
// read them: 16 bytes a lane.
template <typename T>
__global__ __launch_bounds__(256) void attention_copy_kernel(Heads in, T* __restrict__ out, int64_t tokens, int heads,
                                                             int dim, int width, int64_t pieces) {
    constexpr int N = 16 / sizeof(T);
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= pieces) return;
    const int per = width / N, d = (int)(id % per) * N;
    const int64_t row = id / per, h = row % heads, bt = row / heads;
    const T* const p = reinterpret_cast<const T*>(in.p + bt / tokens * in.batch + bt % tokens * in.token + h * in.head);
    T f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = d + e < dim ? p[d + e] : (T)0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) out[id * N + e] = f[e];
}

// ---------------------------------------------------------------- host
constexpr int kCus = 256;

Heads in_bytes(const jorge_heads& h, int64_t e) { return {(char*)h.data, h.batch * e, h.token * e, h.head * e}; }

// Whether a matrix can be read as it lies: whole pieces of 16 bytes.
bool readable(const jorge_attention_shape& s, const jorge_heads& h) {
    const int64_t n = 16 / dtype_bytes(s.dtype);
    return s.dim % n == 0 && h.batch % n == 0 && h.token % n == 0 && h.head % n == 0 && aligned(h.data, 16);
}
int64_t copy_width(const jorge_attention_shape& s) { return round_up(s.dim, 16 / dtype_bytes(s.dtype)); }

struct Plan {
    bool few;                      // forward: the kernel for few rows
    int tiles, tiles_k;            // of own rows, of own keys
    int ranges, ranges_q, ranges_k;  // forward; dq (over keys); dk, dv (over queries)
    int wide;                      // elements of a row as the kernels take it: 32, 64, 96 or 128
};
// Into how many ranges a launch of `groups` workgroups cuts `tiles` streamed tiles: enough that each CU has two
// workgroups, of at least `least` tiles.
int cut(int64_t groups, int64_t tiles, int64_t least) {
    return (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(2 * kCus, std::max<int64_t>(1, groups)), tiles / least,
                                                        64}));
}
Plan plan_of(const jorge_attention_shape& s) {
    Plan p{};
    const int64_t group = s.heads / s.kv_heads, rows = s.q_tokens * group, bh = s.batch * s.kv_heads;
    const int tile = s.dtype == JORGE_F32 ? 32 : 64;
    p.wide = (int)round_up(s.dim, 32);
    p.few = rows <= kOwn;
    p.tiles = (int)ceil_div(rows, 4 * kOwn);
    p.tiles_k = (int)ceil_div(s.kv_tokens, 4 * kOwn);
    // What a query sees at most, in tiles.
    const int64_t window = std::min(s.window, s.kv_tokens);
    const int64_t keys = window ? std::min(s.kv_tokens, window + 4 * kOwn / group + 1) : s.kv_tokens;
    const int64_t key_tiles = ceil_div(keys, tile), row_tiles = ceil_div(s.q_tokens, tile);
    p.ranges = p.few ? cut(bh, key_tiles, 8) : cut(bh * p.tiles, key_tiles, 2);
    p.ranges_q = cut(bh * p.tiles, key_tiles, 2);
    p.ranges_k = cut(bh * p.tiles_k, row_tiles, 2);
    return p;
}

struct Space {
    char *q, *k, *v, *g;           // copies
    float *part, *part_lse;
    float *lse2, *delta, *part_k, *part_v;
    int64_t bytes;
};
Space carve(void* base, const jorge_attention_shape& s, const Plan& p, const jorge_heads* dout) {
    Carve c{(char*)base};
    Space w{};
    const int64_t e = dtype_bytes(s.dtype), width = copy_width(s);
    const auto copy = [&](const jorge_heads& h, int64_t tokens, int64_t heads) {
        return readable(s, h) ? nullptr : c.take<char>(s.batch * tokens * heads * width * e);
    };
    w.q = copy(s.q, s.q_tokens, s.heads);
    w.k = copy(s.k, s.kv_tokens, s.kv_heads);
    w.v = copy(s.v, s.kv_tokens, s.kv_heads);
    const int64_t rows = s.batch * s.heads * s.q_tokens, keys = s.batch * s.kv_heads * s.kv_tokens;
    if (!dout) {
        if (p.ranges > 1) {
            w.part = c.take<float>(p.ranges * rows * p.wide);
            w.part_lse = c.take<float>(p.ranges * rows);
        }
    } else {
        w.g = copy(*dout, s.q_tokens, s.heads);
        w.lse2 = c.take<float>(rows);
        w.delta = c.take<float>(rows);
        if (p.ranges_q > 1) w.part = c.take<float>(p.ranges_q * rows * p.wide);
        if (p.ranges_k > 1) {
            w.part_k = c.take<float>(p.ranges_k * keys * p.wide);
            w.part_v = c.take<float>(p.ranges_k * keys * p.wide);
        }
    }
    w.bytes = c.used;
    return w;
}

Call call_of(const jorge_attention_shape& s) {
    Call c{};
    c.q_lengths = s.q_lengths;
    c.kv_lengths = s.kv_lengths;
    c.batch = (int)s.batch;
    c.q_tokens = (int)s.q_tokens;
    c.kv_tokens = (int)s.kv_tokens;
    c.heads = s.heads;
    c.kv_heads = s.kv_heads;
    c.group = s.heads / s.kv_heads;
    c.dim = s.dim;
    c.causal = s.causal;
    c.window = (int)std::min<int64_t>(s.window, 1 << 30);
    c.scale = (float)s.scale;
    const double scale2 = (double)c.scale * 1.4426950408889634;
    c.scale2 = (float)scale2;
    c.scale2_low = (float)(scale2 - (double)c.scale2);
    return c;
}

template <typename T>
Heads operand(const jorge_attention_shape& s, const jorge_heads& h, int64_t tokens, int heads, char* copy,
              hipStream_t st) {
    if (!copy) return in_bytes(h, sizeof(T));
    const int64_t width = copy_width(s), pieces = s.batch * tokens * heads * width / (16 / (int64_t)sizeof(T));
    if (pieces)
        attention_copy_kernel<T><<<dim3((unsigned)ceil_div(pieces, 256)), dim3(256), 0, st>>>(
            in_bytes(h, sizeof(T)), (T*)copy, tokens, heads, s.dim, (int)width, pieces);
    const int64_t row = width * (int64_t)sizeof(T);
    return {copy, tokens * heads * row, heads * row, row};
}

template <typename K>
jorge_status allow_lds(K* kernel, int bytes) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) !=
        hipSuccess) {
        (void)hipGetLastError();
        return refuse(JORGE_ERR_HIP, "attention: no LDS for its tiles");
    }
    return JORGE_OK;
}

template <typename T, int D>
jorge_status forward(const jorge_attention_shape& s, const Plan& p, const Space& w, const jorge_heads& out, float* lse,
                     hipStream_t st) {
    using L = Tile<T, D>;
    const Call c = call_of(s);
    const Heads q = operand<T>(s, s.q, s.q_tokens, s.heads, w.q, st);
    const Heads k = operand<T>(s, s.k, s.kv_tokens, s.kv_heads, w.k, st);
    const Heads v = operand<T>(s, s.v, s.kv_tokens, s.kv_heads, w.v, st);
    const Output o{in_bytes(out, sizeof(T)), lse, w.part, w.part_lse};
    const int bh = c.batch * c.kv_heads;
    jorge_status err;
    if (p.few) {
        constexpr int joined = 4 * kOwn * (D + 4 + 2) * 4, ring = 8 * L::kBytes, bytes = joined > ring ? joined : ring;
        const auto f = attention_few_kernel<T, D>;
        if ((err = allow_lds(f, bytes)) != JORGE_OK) return err;
        f<<<dim3(bh, p.ranges), dim3(256), bytes, st>>>(c, q, k, v, o);
    } else {
        const auto f = attention_forward_kernel<T, D>;
        if ((err = allow_lds(f, 4 * L::kBytes)) != JORGE_OK) return err;
        f<<<dim3(bh * p.tiles, p.ranges), dim3(256), 4 * L::kBytes, st>>>(c, q, k, v, o, p.tiles);
    }
    if (w.part)
        attention_join_kernel<T, D><<<dim3((unsigned)ceil_div(s.batch * s.heads * s.q_tokens, 8)), dim3(256), 0, st>>>(
            c, o, p.ranges);
    return launched("attention");
}

template <typename T, int D>
jorge_status backward(const jorge_attention_shape& s, const Plan& p, const Space& w, const jorge_heads& dout,
                      const jorge_heads& out, const float* lse, const jorge_heads& dq, const jorge_heads& dk,
                      const jorge_heads& dv, hipStream_t st) {
    using L = Tile<T, D>;
    const Call c = call_of(s);
    const Heads q = operand<T>(s, s.q, s.q_tokens, s.heads, w.q, st);
    const Heads k = operand<T>(s, s.k, s.kv_tokens, s.kv_heads, w.k, st);
    const Heads v = operand<T>(s, s.v, s.kv_tokens, s.kv_heads, w.v, st);
    const Heads g = operand<T>(s, dout, s.q_tokens, s.heads, w.g, st);
    const int64_t rows = s.batch * s.heads * s.q_tokens, keys = s.batch * s.kv_heads * s.kv_tokens;
    const int bh = c.batch * c.kv_heads;
    // dq's kernel comes first and forms what dk's and dv's reads of a row too, also without dq.
    const bool fused = readable(s, out);
    if (rows && !fused)
        attention_delta_kernel<T><<<dim3((unsigned)ceil_div(rows, 128)), dim3(256), 0, st>>>(
            c, in_bytes(out, sizeof(T)), in_bytes(dout, sizeof(T)), w.delta);
    jorge_status err;
    if (rows) {
        if ((err = allow_lds(attention_dq_kernel<T, D>, 4 * L::kBytes)) != JORGE_OK) return err;
        const Gradient to{in_bytes(dq, sizeof(T)), dq.data ? w.part : nullptr};
        attention_dq_kernel<T, D><<<dim3(bh * p.tiles, dq.data ? p.ranges_q : 1), dim3(256), 4 * L::kBytes, st>>>(
            c, q, k, v, g, {fused ? in_bytes(out, sizeof(T)) : Heads{}, lse, w.lse2, w.delta}, to, p.tiles);
        if (to.part)
            attention_sum_kernel<T, D><<<dim3((unsigned)ceil_div(rows, 8)), dim3(256), 0, st>>>(
                to, {}, p.ranges_q, s.q_tokens * c.group, rows, c.kv_heads, c.group, c.dim);
    }
    if ((dk.data || dv.data) && keys) {
        constexpr int bytes = 4 * L::kBytes + 1024;
        if ((err = allow_lds(attention_dkv_kernel<T, D>, bytes)) != JORGE_OK) return err;
        const Gradient tk{in_bytes(dk, sizeof(T)), dk.data ? w.part_k : nullptr};
        const Gradient tv{in_bytes(dv, sizeof(T)), dv.data ? w.part_v : nullptr};
        attention_dkv_kernel<T, D><<<dim3(bh * p.tiles_k, p.ranges_k), dim3(256), bytes, st>>>(
            c, q, k, v, g, w.lse2, w.delta, tk, tv, p.tiles_k);
        if (tk.part || tv.part)
            attention_sum_kernel<T, D><<<dim3((unsigned)ceil_div(keys, 8), 2), dim3(256), 0, st>>>(
                tk, tv, p.ranges_k, s.kv_tokens, keys, c.kv_heads, 1, c.dim);
    }
    return launched("attention");
}

// f(an element, the row's width as a constant).
template <typename F>
jorge_status with_kernels(const jorge_attention_shape& s, const Plan& p, F&& f) {
    const auto wide = [&](auto t) {
        switch (p.wide) {
            case 32: return f(t, std::integral_constant<int, 32>());
            case 64: return f(t, std::integral_constant<int, 64>());
            case 96: return f(t, std::integral_constant<int, 96>());
            default: return f(t, std::integral_constant<int, 128>());
        }
    };
    return s.dtype == JORGE_F32 ? wide(0.0f) : wide((bf16)0.0f);
}

// Strides that the kernels' offsets can hold: a tile's rows within 2^31 bytes.
jorge_status check_heads(const jorge_attention_shape& s, const jorge_heads& h, const char* why) {
    if (!h.data) return bad(why);
    if (!aligned(h.data, dtype_bytes(s.dtype))) return bad("attention: a pointer is not aligned to its element");
    if (h.batch < 0 || h.token < 0 || h.head < 0) return bad("attention: a stride is negative");
    if (h.token > JORGE_ATTENTION_MAX_STRIDE)
        return refuse(JORGE_ERR_UNSUPPORTED, "attention: a token stride above JORGE_ATTENTION_MAX_STRIDE (2^22)");
    return JORGE_OK;
}
jorge_status check(const jorge_attention_shape* shape) {
    if (!shape) return bad("attention: a shape is needed");
    const jorge_attention_shape& s = *shape;
    if (!known_dtype(s.dtype)) return bad("attention: unknown element type");
    if (s.batch < 0 || s.q_tokens < 0 || s.kv_tokens < 0) return bad("attention: batch and tokens >= 0 are needed");
    if (s.heads < 1 || s.kv_heads < 1 || s.heads % s.kv_heads)
        return bad("attention: heads must be a positive multiple of kv_heads");
    if (s.dim < 1) return bad("attention: dim >= 1 is needed");
    if (s.dim > JORGE_ATTENTION_MAX_DIM)
        return refuse(JORGE_ERR_UNSUPPORTED, "attention: dim above JORGE_ATTENTION_MAX_DIM");
    if (!(s.scale > 0.0) || !(s.scale < 1e30)) return bad("attention: scale must be positive and below 1e30");
    if (s.causal != 0 && s.causal != 1) return bad("attention: causal must be 0 or 1");
    if (s.window < 0) return bad("attention: window >= 0 is needed");
    if (s.window && !s.causal) return bad("attention: a window needs causal");
    if (s.q_tokens > JORGE_ATTENTION_MAX_TOKENS || s.kv_tokens > JORGE_ATTENTION_MAX_TOKENS)
        return refuse(JORGE_ERR_UNSUPPORTED, "attention: tokens above JORGE_ATTENTION_MAX_TOKENS");
    // Lengths of launches: tiles of 128 rows, rows by the eight, copies' pieces by the 256; k and v have kv_heads.
    if (s.batch > 1 << 20 || s.heads > 1 << 20 || s.batch * s.heads > 1 << 22 ||
        s.batch * s.heads * s.q_tokens > JORGE_ATTENTION_MAX_ROWS)
        return refuse(JORGE_ERR_UNSUPPORTED, "attention: batch * heads * q_tokens above JORGE_ATTENTION_MAX_ROWS (2^26)");
    if (s.batch * s.kv_heads * s.kv_tokens > JORGE_ATTENTION_MAX_ROWS)
        return refuse(JORGE_ERR_UNSUPPORTED,
                      "attention: batch * kv_heads * kv_tokens above JORGE_ATTENTION_MAX_ROWS (2^26)");
    return JORGE_OK;
}
jorge_status check_inputs(const jorge_attention_shape& s) {
    jorge_status st;
    if (s.q_tokens && (st = check_heads(s, s.q, "attention: q is needed")) != JORGE_OK) return st;
    if (s.kv_tokens && (st = check_heads(s, s.k, "attention: k is needed")) != JORGE_OK) return st;
    if (s.kv_tokens && (st = check_heads(s, s.v, "attention: v is needed")) != JORGE_OK) return st;
    if (!aligned(s.q_lengths, 8) || !aligned(s.kv_lengths, 8))
        return bad("attention: a pointer is not aligned to its element");
    return JORGE_OK;
}
jorge_status check_workspace(int64_t need, const void* workspace, int64_t bytes) {
    if (need == 0) return JORGE_OK;
    if (!workspace || !aligned(workspace, kAlign)) return bad("attention: a workspace aligned to 256 bytes is needed");
    if (bytes < need) return bad("attention: the workspace is too small");
    return JORGE_OK;
}

}  // namespace
}  // namespace jorge_lm

using namespace jorge_lm;

extern "C" {

jorge_status jorge_attention_workspace(const jorge_attention_shape* shape, const jorge_heads* dout, int64_t* bytes) {
    if (!bytes) return bad("attention: bytes is needed");
    const jorge_status st = check(shape);
    if (st != JORGE_OK) return st;
    *bytes = shape->batch ? carve(nullptr, *shape, plan_of(*shape), dout).bytes : 0;
    return JORGE_OK;
}

jorge_status jorge_attention_forward(const jorge_attention_shape* shape, const jorge_heads* out, float* lse,
                                     void* workspace, int64_t workspace_bytes, void* hip_stream) {
    jorge_status st = check(shape);
    if (st != JORGE_OK) return st;
    const jorge_attention_shape& s = *shape;
    if (s.batch == 0 || s.q_tokens == 0) return JORGE_OK;
    if (!out || !lse) return bad("attention: out and lse are needed");
    if (!aligned(lse, 4)) return bad("attention: a pointer is not aligned to its element");
    if ((st = check_inputs(s)) != JORGE_OK || (st = check_heads(s, *out, "attention: out is needed")) != JORGE_OK)
        return st;
    const Plan p = plan_of(s);
    if ((st = check_workspace(carve(nullptr, s, p, nullptr).bytes, workspace, workspace_bytes)) != JORGE_OK) return st;
    const Space w = carve(workspace, s, p, nullptr);
    const hipStream_t q = reinterpret_cast<hipStream_t>(hip_stream);
    return with_kernels(s, p, [&](auto t, auto D) {
        return forward<decltype(t), decltype(D)::value>(s, p, w, *out, lse, q);
    });
}

jorge_status jorge_attention_backward(const jorge_attention_shape* shape, const jorge_heads* dout,
                                      const jorge_heads* out, const float* lse, const jorge_heads* dq,
                                      const jorge_heads* dk, const jorge_heads* dv, void* workspace,
                                      int64_t workspace_bytes, void* hip_stream) {
    jorge_status st = check(shape);
    if (st != JORGE_OK) return st;
    const jorge_attention_shape& s = *shape;
    const jorge_heads none{};
    const jorge_heads &gq = dq ? *dq : none, &gk = dk ? *dk : none, &gv = dv ? *dv : none;
    if (s.batch == 0 || (!gq.data && !gk.data && !gv.data)) return JORGE_OK;
    if ((st = check_inputs(s)) != JORGE_OK) return st;
    if (s.q_tokens) {
        if (!dout || !out || !lse) return bad("attention: dout, out and lse are needed");
        if (!aligned(lse, 4)) return bad("attention: a pointer is not aligned to its element");
        if ((st = check_heads(s, *dout, "attention: dout is needed")) != JORGE_OK ||
            (st = check_heads(s, *out, "attention: out is needed")) != JORGE_OK)
            return st;
    }
    for (const jorge_heads* g : {&gq, &gk, &gv})
        if (g->data && (st = check_heads(s, *g, "")) != JORGE_OK) return st;
    const Plan p = plan_of(s);
    const jorge_heads& d = dout ? *dout : none;
    if ((st = check_workspace(carve(nullptr, s, p, &d).bytes, workspace, workspace_bytes)) != JORGE_OK) return st;
    const Space w = carve(workspace, s, p, &d);
    const hipStream_t q = reinterpret_cast<hipStream_t>(hip_stream);
    const jorge_heads& o = out ? *out : none;
    return with_kernels(s, p, [&](auto t, auto D) {
        return backward<decltype(t), decltype(D)::value>(s, p, w, d, o, lse, gq, gk, gv, q);
    });
}

}  // extern "C"
