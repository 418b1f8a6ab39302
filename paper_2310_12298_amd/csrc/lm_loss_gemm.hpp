// The bfloat16 matrix product that cross entropy and the linear layers are made of, for gfx950:
//   C[a][b] = sum_k A[a][k] B[b][k],  both operands K-contiguous, fp32 accumulators,
// as a device function that leaves a tile of C in registers for the caller's epilogue.
//
// A workgroup of four waves (2 x 2) computes a tile of 32 WA x 32 WB: each wave 16 WA x 16 WB, as
// WA x WB accumulators of v_mfma_f32_16x16x32_bf16. With WA = WB = 8 that is a 256 x 256 tile, one
// wave per SIMD: 256 accumulator registers per lane and two sets of fragments. A wave's 128 x 128
// takes 16 KB from LDS per 64 MFMAs, the least per flop that the registers allow: LDS would bound
// waves of 128 x 64 (two per SIMD) at 9/8 of the MFMAs' time, these at 3/4.
//
// K goes by stages through a ring of buffers in LDS. Each stage is written by direct-to-LDS loads, started as soon as
// its buffer is free; nothing passes through registers. A wave reads the next fragments while the MFMAs of the current
// ones run.
//
// Which row of the tile goes where. An MFMA leaves lane l with rows 4 (l / 16) + r (r = 0 .. 3) and
// column l % 16 of its 16 x 16 block. The rows that feed block i and the columns that feed block j
// are chosen so that a lane ends up with WA * 4 consecutive a and WB consecutive b:
//   a = 4 WA (l / 16) + 4 i + r,  b = WB (l % 16) + j  of the wave's part,
// so that both C and its transpose are written in whole pieces from registers. The choice costs
// nothing: it is the row that each direct-to-LDS load fetches.
//
// A load brings 1 KB to consecutive LDS, 16 bytes per lane. For one product (plain) a stage is 64 k: a load fetches 8
// rows of 128 bytes, whole cache lines (4096 x 4096 x 8192: 1200-1250 TFLOP/s, against 1140 with stages of 32 k and
// half lines). For products of terms it is 32 k: 16 rows of 64 bytes. Within a row the 16-byte chunks are permuted by
// the row's number so that a fragment read (lane l: row l % 16, chunk l / 16) meets no bank twice: the LDS serves lanes
// 0-3, 12-15 and 20-27 together, then the others of the first 32, and the same of the last 32 (shown by the counter of
// bank conflicts: 0, where a permutation made for 16 consecutive lanes doubled the reads' time).
#pragma once

#include "lm_common.hpp"

#include <type_traits>

namespace jorge_lm {

constexpr int kStageK = 32;

// One operand of a product: `rows` rows of K elements at a stride of ld elements. Rows past the end are
// not read: the last one is, in their place. `plane`: elements between a row's terms, of a split operand.
//
// A turned operand (Tile's TA, TB) lies the other way round: K lines of `rows` elements (a multiple of 8, 16-byte
// aligned) at a stride of ld. `depth` of the lines exist; the others count as zeros. It may be two such matrices, one
// after the other along K: the second one, p2, begins at line `part` (a multiple of 64).
struct Operand {
    const bf16* p;
    int64_t ld, plane;
    int64_t rows;
    const bf16* p2 = nullptr;
    int64_t depth = 0, part = 0;
};
constexpr unsigned kNowhere = 0x80000000u;  // an offset past every resource's end: a load brings zeros

constexpr int kTerms = 3;  // of a split operand

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

// 4 lines of 16 elements, 8 bytes from each of 16 lanes, to lane i's column i of each line. In a function with a
// restricted pointer: without what that says of aliases the compiler waits here for every direct-to-LDS load in flight,
// the next stages' too, which the callers' own waits keep apart (2.5 times the time of a product).
__device__ __forceinline__ s16x4 read_turned4(const lds_s16x4* __restrict__ p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<lds_s16x4*>(p));
}

// What chunk numbers are exclusive-ored with in row rho of 16, for rows of 64 and of 128 bytes.
__device__ __forceinline__ int swizzle64(int rho) { return -(rho >> 2) & 3; }
__device__ __forceinline__ int swizzle128(int rho) { return rho >> 1; }

// PAIR: A is two matrices of the same shape and plane, and a tile half as many rows of each: a wave's blocks i < WA / 2
// are of the first, the others of the second, so that a lane holds the same 2 WA rows of both:
//   a = 2 WA (l / 16) + 4 i + r  of 8 WA rows, in blocks i and i + WA / 2.
// The loads of waves 0 and 2 are then all of the first matrix, those of 1 and 3 of the second.
//
// TA, TB: the operand is turned. A stage then holds 64 lines of the tile's 32 WA elements, and a fragment is read by
// ds_read_tr16, which gives lane l % 16 of 16 the elements in column l % 16 of 4 lines of 16. The columns of a block are
// 4 times 4 consecutive ones, so B's block j has those that A's rule gives: b = 4 WB (n / 4) + 4 j + n % 4 for column n
// of the block. The 16-byte chunks of a line are permuted by its number so that the 4 x 4 pieces of 8 bytes that 16
// lanes read meet 16 chunks.
template <int WA, int WB, int RING, bool SPLIT, bool PAIR = false, bool TA = false, bool TB = false>
struct Tile {
    static_assert(!SPLIT || (!TA && !TB), "terms are K-contiguous");
    static constexpr int kA = 32 * WA, kB = 32 * WB;
    static constexpr int kRowsA = PAIR ? 16 * WA : kA;             // of A (of each of two)
    static constexpr int kLaneA = PAIR ? 2 * WA : 4 * WA;          // consecutive ones that a lane ends up with
    static constexpr int kBytes = RING * (kA + kB) * kStageK * 2;  // of LDS: RING stages of 32 k
    // Direct-to-LDS loads per wave and stage of the ring.
    static constexpr int kLoadsA = SPLIT ? WA / 2 : WA, kLoadsB = SPLIT ? WB / 2 : WB, kLoads = kLoadsA + kLoadsB;

    f32x4 acc[WA][WB];

    // First a and first b of the calling lane's part of the tile.
    static __device__ __forceinline__ int lane_a() {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        return (wave >> 1) * (kRowsA / 2) + (lane >> 4) * kLaneA;
    }
    static __device__ __forceinline__ int lane_b() {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        return (wave & 1) * 16 * WB + (lane & 15) * WB;
    }

    // Which b of the wave's part column n of block j is.
    static __device__ __forceinline__ int part_b(int n, int j) {
        return TB ? (n >> 2) * 4 * WB + 4 * j + (n & 3) : n * WB + j;
    }

    // What a line's chunk numbers are exclusive-ored with, of a turned operand with W blocks to a wave.
    template <int W>
    static __device__ __forceinline__ int swizzle_line(int k) {
        return W == 8 ? k & 3 : W == 4 ? (k & 1) | (k >> 1 & 1) << 3 : (k >> 1 & 1) << 2;
    }

    // Stages [s0, s1) of the product of rows a0 .. of A and b0 .. of B, of which each row has `stages` (32 k each).
    // s0 and s1 are even, s1 > s0. lds: kBytes.
    __device__ __forceinline__ void multiply(const Operand& A, const Operand& B, int64_t a0, int64_t b0, int s0, int s1,
                                             int stages, char* lds) {
        multiply(A, A, B, a0, b0, s0, s1, stages, lds);
    }
    // PAIR: of A1 and A2.
    __device__ __forceinline__ void multiply(const Operand& A1, const Operand& A2, const Operand& B, int64_t a0,
                                             int64_t b0, int s0, int s1, int stages, char* lds) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const Operand& A = PAIR && (wave & 1) ? A2 : A1;
        Loads load;
        if constexpr (TA) load.la = Lines(A, a0);
        if constexpr (TB) load.lb = Lines(B, b0);
        load.line = s0 * kStageK;
        // Where this lane's loads start: load n of the operand (n = wave * kLoads + v) takes rows rho of block i of a
        // half of the tile. Bytes from the tile's first row to the end of its last one are what a load may reach.
        const int limA = (int)(A.rows - a0 < kRowsA ? A.rows - a0 : kRowsA) - 1;
        const int limB = (int)(B.rows - b0 < kB ? B.rows - b0 : kB) - 1;
        const unsigned K = (unsigned)(stages * kStageK), more = SPLIT ? kTerms - 1 : 0;
        const auto place = [&](int n, int& block, int& rho) {
            block = SPLIT ? n : n / 2;
            rho = SPLIT ? lane >> 2 : (n & 1) * 8 + (lane >> 3);
            return (unsigned)(SPLIT ? (lane & 3) ^ swizzle64(rho) : (lane & 7) ^ swizzle128(rho)) * 16u;
        };
        // Of a turned operand: 1 KB is 16 / W lines of 32 W elements.
        const auto line = [&](int n, auto W, int64_t there, unsigned ld) {
            constexpr int w = decltype(W)::value, chunks = 4 * w;
            const int k = n * (64 / chunks) + lane / chunks, chunk = (lane % chunks) ^ swizzle_line<w>(k);
            return chunk * 8 < there ? (unsigned)k * ld * 2u + chunk * 16u : kNowhere;
        };
#pragma unroll
        for (int v = 0; v < kLoadsA; ++v) {
            if constexpr (TA) {
                load.offA[v] = line(wave * kLoadsA + v, std::integral_constant<int, WA>(), A.rows - a0, (unsigned)A.ld);
                continue;
            }
            int block, rho;
            const unsigned chunk = place(wave * kLoadsA + v, block, rho);
            const int row = block / WA * (kRowsA / 2) + (rho >> 2) * kLaneA + 4 * (block % (kLaneA / 4)) + (rho & 3);
            load.offA[v] = (unsigned)(row < limA ? row : limA) * (unsigned)A.ld * 2u + chunk;
        }
#pragma unroll
        for (int v = 0; v < kLoadsB; ++v) {
            if constexpr (TB) {
                load.offB[v] = line(wave * kLoadsB + v, std::integral_constant<int, WB>(), B.rows - b0, (unsigned)B.ld);
                continue;
            }
            int block, rho;
            const unsigned chunk = place(wave * kLoadsB + v, block, rho);
            const int row = block / WB * 16 * WB + rho * WB + block % WB;
            load.offB[v] = (unsigned)(row < limB ? row : limB) * (unsigned)B.ld * 2u + chunk;
        }
        if constexpr (!TA)
            load.ra = resource(A.p + a0 * A.ld, ((unsigned)limA * (unsigned)A.ld + more * (unsigned)A.plane + K) * 2u);
        if constexpr (!TB)
            load.rb = resource(B.p + b0 * B.ld, ((unsigned)limB * (unsigned)B.ld + more * (unsigned)B.plane + K) * 2u);
        load.lines();
        load.k = s0 * (kStageK * 2);
        load.left = SPLIT ? s1 - s0 : (s1 - s0) / 2;
#pragma unroll
        for (int i = 0; i < WA; ++i)
#pragma unroll
            for (int j = 0; j < WB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (SPLIT) terms(load, (int)A.plane * 2, (int)B.plane * 2, s0, s1, wave, lds);
        else plain(load, s0, s1, wave, lds);
        wait_loads<0>();
        __builtin_amdgcn_s_barrier();  // the ring is free for the epilogue
    }

private:
    // A turned operand from element `first` of its lines on: the 64 lines of a stage, of which those past `depth` are past
    // the resource's end. Without branches: the loop's body stays one block.
    struct Lines {
        const bf16 *p, *p2;
        int ld, depth, part, last;  // last: elements of a line from `first` on, in whole chunks
        Lines() = default;
        __device__ __forceinline__ Lines(const Operand& o, int64_t first)
            : p(o.p + first), p2(o.p2 ? o.p2 + first : nullptr), ld((int)o.ld), depth((int)o.depth), part(o.p2 ? (int)o.part : 1 << 30),
              last((int)((o.rows + 7) / 8 * 8 - first)) {}
        __device__ __forceinline__ __amdgpu_buffer_rsrc_t stage(int line) const {
            const bool two = line >= part;
            const int at = two ? line - part : line, left = depth - at, n = left < 64 ? left : 64;
            const unsigned bytes = (unsigned)((n - 1) * ld + last) * 2u;
            return resource((two ? p2 : p) + (int64_t)at * ld, n > 0 ? bytes : 0u);
        }
    };

    // The loads of one stage after the other.
    struct Loads {
        unsigned offA[kLoadsA], offB[kLoadsB];
        __amdgpu_buffer_rsrc_t ra, rb;
        int k, left;  // bytes into the rows, and stages left
        Lines la, lb; // turned operands
        int line;     // of the stage's first one
        __device__ __forceinline__ void a(int v, char* to, int at) const {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)to, 16, offA[v], TA ? 0 : at, 0, 0);
        }
        __device__ __forceinline__ void b(int v, char* to, int at) const {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void*)to, 16, offB[v], TB ? 0 : at, 0, 0);
        }
        __device__ __forceinline__ void lines() {
            if constexpr (TA) ra = la.stage(line);
            if constexpr (TB) rb = lb.stage(line);
        }
        // Where no stage is left the last one is loaded again and not used: every wave always has the same number of
        // loads in flight, and the loop's body stays one block.
        __device__ __forceinline__ void next() {
            --left;
            k += left > 0 ? kStageK * (SPLIT ? 2 : 4) : 0;
            if constexpr (TA || TB) {
                line += left > 0 ? 2 * kStageK : 0;
                lines();
            }
        }
    };

    // After the last MFMA of all, the wait states that reading its result takes. They stand inside the loop, ahead of
    // any place where the compiler, which does not see MFMAs in the asm, may copy an accumulator.
    static __device__ __forceinline__ void settle(int s, int s1) {
        asm volatile("s_cmp_lt_i32 %0, %1\n\ts_cbranch_scc1 1f\n\ts_nop 15\n\ts_nop 15\n1:" ::"s"(s), "s"(s1) : "scc");
    }

    // One product, in stages of 64 k. A stage in the ring is A's blocks of 16 rows (2 KB), then B's.
    __device__ __forceinline__ void plain(Loads& load, int s0, int s1, int wave, char* lds) {
        constexpr int kRing = RING / 2, kStageBytes = (kA + kB) * kStageK * 4;
        static_assert(kRing >= 2 && (kRing & (kRing - 1)) == 0, "a power of two");
        const int rho = threadIdx.x & 15, frag = rho * 128 + ((((threadIdx.x & 63) >> 4) ^ swizzle128(rho)) * 16);
        const int fragA = frag + (wave >> 1) * WA * 2048, fragB = frag + (2 * WA + (wave & 1) * WB) * 2048;
        // Of turned operands: line 8 (l / 16) + l % 16 / 4 of 32, elements 4 W (l % 4) .. + 3 of the wave's part; the next
        // four lines are 4 further, whose chunks are permuted alike.
        const int lane = threadIdx.x & 63, line = (lane >> 4) * 8 + (lane & 15) / 4;
        const auto turned = [&](auto W, int part) {
            constexpr int w = decltype(W)::value;
            return line * (64 * w) + (((part * 2 * w + (lane & 3) * (w / 2)) ^ swizzle_line<w>(line)) * 16);
        };
        const int turnA = turned(std::integral_constant<int, WA>(), wave >> 1);
        const int turnB = turned(std::integral_constant<int, WB>(), wave & 1) + kA * kStageK * 4;
        bf16x8 fa[2][WA], fb[2][WB];
        // Block i of half h: chunk i / 2 of the lane's, its half i % 2.
        const auto read_turned = [](const char* p, int at, auto W, int h, int i) {
            constexpr int w = decltype(W)::value;
            s16x4 v[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                v[u] = read_turned4((const lds_s16x4*)(p + (at ^ (i / 2 * 16)) + (h * 32 + u * 4) * (64 * w) + (i & 1) * 8));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        };
        const auto one = [&](int v, int slot) {
            char* const to = lds + slot * kStageBytes;
            if (v < kLoadsA) load.a(v, to + (wave * kLoadsA + v) * 1024, load.k);
            else load.b(v - kLoadsA, to + (4 * WA + wave * kLoadsB + v - kLoadsA) * 1024, load.k);
        };
        // Fragment f of half h of a stage: first B's, which the first row of MFMAs needs together, then A's.
        const auto read = [&](int slot, int h, int f) {
            const char* const p = lds + slot * kStageBytes;
            if (f < WB) {
                if constexpr (TB) fb[h][f] = read_turned(p, turnB, std::integral_constant<int, WB>(), h, f);
                else fb[h][f] = *reinterpret_cast<const bf16x8*>(p + (fragB ^ (h * 64)) + f * 2048);
            } else {
                if constexpr (TA) fa[h][f - WB] = read_turned(p, turnA, std::integral_constant<int, WA>(), h, f - WB);
                else fa[h][f - WB] = *reinterpret_cast<const bf16x8*>(p + (fragA ^ (h * 64)) + (f - WB) * 2048);
            }
        };
#pragma unroll
        for (int r = 0; r < kRing; ++r) {
#pragma unroll
            for (int v = 0; v < kLoads; ++v) one(v, r);
            load.next();
        }
        wait_loads<(kRing - 1) * kLoads>();
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int f = 0; f < WA + WB; ++f) read(0, 0, f);
        int slot = 0;
        // The MFMAs of half h, and among them, in this order: the fragment reads of the next half by twos in the first
        // half of the groups, so that it need not wait for them; a load in every group (h = 1), and after the last one
        // the way to the next stage (the scalar unit runs beside the MFMAs).
        const auto half = [&](auto H, int from) {
            constexpr int h = decltype(H)::value, G = WA + WB, PER = WA * WB / G;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                __builtin_amdgcn_sched_barrier(0);
                if (g < G / 2) {
                    read(from, h ^ 1, 2 * g);
                    read(from, h ^ 1, 2 * g + 1);
                }
                if constexpr (h == 1) {
                    one(g, slot);
                    if (g == G - 1) load.next();
                }
#pragma unroll
                for (int m = g * PER; m < (g + 1) * PER; ++m)
                    mfma(acc[m / WB][m % WB], fa[h][m / WB], fb[h][m % WB]);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int s = s0; s < s1; s += 2) {
            const int ahead = (slot + 1) & (kRing - 1);
            half(std::integral_constant<int, 0>(), slot);
            // All waves have read this stage whole, so its buffer is free; and the next one has landed for all.
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            wait_loads<(kRing - 2) * kLoads>();
            __builtin_amdgcn_s_barrier();
            half(std::integral_constant<int, 1>(), ahead);
            slot = ahead;
            settle(s + 2, s1);
        }
    }

    // Six products of the operands' terms, those down to 2^-16 of the whole, stage by stage in the order
    //   A2 B0, A1 B0, A1 B1, A0 B1, A0 B2, A0 B0,
    // in which each step exchanges one of the two factors. The ring holds planes of one term of one operand, in the
    // order A2 B0 A1 B1 A0 B2, in which the steps come to need them: each step loads one plane and reads one plane's
    // fragments, half of what six products of their own would.
    __device__ __forceinline__ void terms(Loads& load, int planeA, int planeB, int s0, int s1, int wave, char* lds) {
        static_assert(WA == WB, "planes of one size");
        constexpr int kPlanes = 2 * RING, kPlaneBytes = kA * kStageK * 2;
        const int rho = threadIdx.x & 15, frag = rho * 64 + ((((threadIdx.x & 63) >> 4) ^ swizzle64(rho)) * 16);
        static_assert((kPlanes & (kPlanes - 1)) == 0, "a power of two");
        const int fragA = frag + (wave >> 1) * WA * 1024, fragB = frag + (wave & 1) * WB * 1024;
        bf16x8 fa[2][WA], fb[3][WB];
        // Load v of the plane that plays role r, to a slot.
        const auto one = [&](int r, int v, int slot) {
            char* const to = lds + slot * kPlaneBytes + (wave * kLoadsA + v) * 1024;
            if (r % 2 == 0) load.a(v, to, load.k + (2 - r / 2) * planeA);
            else load.b(v, to, load.k + r / 2 * planeB);
        };
        const auto read = [&](bool a, int set, int f, int slot) {
            const char* const p = lds + slot * kPlaneBytes + f * 1024;
            if (a) fa[set][f] = *reinterpret_cast<const bf16x8*>(p + fragA);
            else fb[set][f] = *reinterpret_cast<const bf16x8*>(p + fragB);
        };
#pragma unroll
        for (int n = 0; n < kPlanes; ++n) {
#pragma unroll
            for (int v = 0; v < kLoadsA; ++v) one(n % 6, v, n);
            if (n % 6 == 5) load.next();
        }
        wait_loads<(kPlanes - 2) * kLoadsA>();
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int f = 0; f < WA; ++f) {
            read(true, 0, f, 0);
            read(false, 0, f, 1);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // plane 0's slot is written from step 0 on
        int slot = 0;  // of plane n, n the number of the step
        const auto step = [&](auto S) {
            constexpr int k = decltype(S)::value % 6, P = decltype(S)::value / 6;
            constexpr int useA = k == 1 || k == 2 ? P ^ 1 : P, useB = k == 4 ? 2 : k == 2 || k == 3 ? P ^ 1 : P;
            // What the next step needs anew: plane n + 2. Its set's last use was before this step.
            constexpr bool readA = k % 2 == 0;
            constexpr int set = k == 2 ? P : k == 3 ? 2 : P ^ 1;
            constexpr int role = (k + kPlanes) % 6;  // of plane n + kPlanes, which is loaded
            // Plane n + 2 has landed for every wave once all have passed the barrier; plane n's fragments were read two
            // steps ago, so its slot is free.
            wait_loads<(kPlanes - 3) * kLoadsA>();
            __builtin_amdgcn_s_barrier();
            const int ahead = (slot + 2) & (kPlanes - 1);
            constexpr int G = 2 * WA, PER = WA * WB / G;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                __builtin_amdgcn_sched_barrier(0);
                if (g < WA) read(readA, set, g, ahead);
                else if ((g - WA) % 2 == 1) one(role, (g - WA) / 2, slot);
                if (g == G - 1 && role == 5) load.next();
#pragma unroll
                for (int m = g * PER; m < (g + 1) * PER; ++m)
                    mfma(acc[m / WB][m % WB], fa[useA][m / WB], fb[useB][m % WB]);
            }
            __builtin_amdgcn_sched_barrier(0);
            slot = (slot + 1) & (kPlanes - 1);
        };
        const auto chunk = [&](auto P) {
            constexpr int b = decltype(P)::value * 6;
            step(std::integral_constant<int, b>());
            step(std::integral_constant<int, b + 1>());
            step(std::integral_constant<int, b + 2>());
            step(std::integral_constant<int, b + 3>());
            step(std::integral_constant<int, b + 4>());
            step(std::integral_constant<int, b + 5>());
        };
        for (int s = s0; s < s1; s += 2) {
            chunk(std::integral_constant<int, 0>());
            chunk(std::integral_constant<int, 1>());
            settle(s + 2, s1);
        }
    }

    // In place, in accumulator registers: left to the compiler the 64 accumulators wander between the two halves
    // of the register file, 3.5 moves for every MFMA.
    static __device__ __forceinline__ void mfma(f32x4& c, const bf16x8& a, const bf16x8& b) {
        asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    }

    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const bf16* p, unsigned bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16*>(p), 0, bytes, 0x00020000);
    }

    template <int N>
    static __device__ __forceinline__ void wait_loads() {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    }
};

}  // namespace jorge_lm
