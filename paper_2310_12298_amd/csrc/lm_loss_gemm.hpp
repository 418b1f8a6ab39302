// The bfloat16 matrix product that cross entropy is made of, for gfx950:
//   C[a][b] = sum_k A[a][k] B[b][k],  both operands K-contiguous, fp32 accumulators,
// as a device function that leaves a tile of C in registers for the caller's epilogue.
//
// A workgroup of four waves (2 x 2) computes a tile of 32 WA x 32 WB: each wave 16 WA x 16 WB, as
// WA x WB accumulators of v_mfma_f32_16x16x32_bf16. With WA = WB = 8 that is a 256 x 256 tile, one
// wave per SIMD: 256 accumulator registers per lane and two sets of fragments. A wave's 128 x 128
// takes 16 KB from LDS per 64 MFMAs, the least per flop that the registers allow: LDS would bound
// waves of 128 x 64 (two per SIMD) at 9/8 of the MFMAs' time, these at 3/4.
//
// K goes by stages of 32 through a ring of RING buffers in LDS. Each stage is written by
// direct-to-LDS loads, started RING - 1 stages ahead; nothing passes through registers. A wave
// reads the next stage's fragments while the MFMAs of the current one run.
//
// Which row of the tile goes where. An MFMA leaves lane l with rows 4 (l / 16) + r (r = 0 .. 3) and
// column l % 16 of its 16 x 16 block. The rows that feed block i and the columns that feed block j
// are chosen so that a lane ends up with WA * 4 consecutive a and WB consecutive b:
//   a = 4 WA (l / 16) + 4 i + r,  b = WB (l % 16) + j  of the wave's part,
// so that both C and its transpose are written in whole pieces from registers. The choice costs
// nothing: it is the row that each direct-to-LDS load fetches.
//
// A block of 16 rows by 32 k is 1 KB of LDS: row rho at 64 rho, its 16-byte chunk c (k = 8 c ..) at
// 16 (c ^ swizzle(rho)). Four neighbouring lanes fetch one row's 64 bytes; a fragment read (lane l:
// row l % 16, chunk l / 16) takes the whole block, and the swizzle spreads any 8 or 16 lanes of it
// over all banks.
#pragma once

#include "lm_common.hpp"

namespace jorge_lm {

constexpr int kStageK = 32;

// One operand of a product: `rows` rows of K elements at a stride of ld elements. Rows past the end are
// not read: the last one is, in their place. `plane`: elements between a row's terms, of a split operand.
struct Operand {
    const bf16* p;
    int64_t ld, plane;
    int64_t rows;
};

// The order in which the terms of split operands are multiplied: the six products down to 2^-16 of the
// whole, smallest first (term t of A with term u of B).
constexpr int kTerms = 3, kSegments = 6;
__device__ __forceinline__ int term_a(int seg) { return (0x001012 >> (4 * seg)) & 3; }
__device__ __forceinline__ int term_b(int seg) { return (0x010210 >> (4 * seg)) & 3; }

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void global_void;

__device__ __forceinline__ int swizzle(int rho) { return -(rho >> 2) & 3; }

template <int WA, int WB, int RING, bool SPLIT>
struct Tile {
    static constexpr int kRing = RING;
    static constexpr int kA = 32 * WA, kB = 32 * WB;
    static constexpr int kStageBytes = (kA + kB) * kStageK * 2;
    static constexpr int kBytes = kRing * kStageBytes;
    // Direct-to-LDS loads per wave and stage: half of each operand's WA (WB) * 2 blocks over the four waves.
    static constexpr int kLoadsA = WA / 2, kLoadsB = WB / 2, kLoads = kLoadsA + kLoadsB;

    f32x4 acc[WA][WB];

    // First a and first b of the calling lane's part of the tile.
    static __device__ __forceinline__ int lane_a() {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        return (wave >> 1) * 16 * WA + (lane >> 4) * 4 * WA;
    }
    static __device__ __forceinline__ int lane_b() {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        return (wave & 1) * 16 * WB + (lane & 15) * WB;
    }

    // Stages [s0, s1) of the product of rows a0 .. of A and b0 .. of B; each segment (pair of terms) has
    // `per` stages. s0, s1 and per are even, s1 > s0. lds: kBytes.
    __device__ __forceinline__ void multiply(const Operand& A, const Operand& B, int64_t a0, int64_t b0, int s0, int s1,
                                             int per, char* lds) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // Where this lane's loads start: block n of the operand (n = wave * kLoads + v), row rho of it.
        const int rho = lane >> 2, chunk = (lane & 3) ^ swizzle(rho);
        unsigned offA[kLoadsA], offB[kLoadsB];
        const int limA = (int)(A.rows - a0 < kA ? A.rows - a0 : kA) - 1, limB = (int)(B.rows - b0 < kB ? B.rows - b0 : kB) - 1;
#pragma unroll
        for (int v = 0; v < kLoadsA; ++v) {
            const int n = wave * kLoadsA + v, half = n / WA, i = n % WA;
            const int row = half * 16 * WA + (rho >> 2) * 4 * WA + 4 * i + (rho & 3);
            offA[v] = (unsigned)(row < limA ? row : limA) * (unsigned)A.ld * 2u + chunk * 16u;
        }
#pragma unroll
        for (int v = 0; v < kLoadsB; ++v) {
            const int n = wave * kLoadsB + v, half = n / WB, j = n % WB;
            const int row = half * 16 * WB + rho * WB + j;
            offB[v] = (unsigned)(row < limB ? row : limB) * (unsigned)B.ld * 2u + chunk * 16u;
        }
        // Bytes from the tile's first row to the end of its last one: what a load may reach.
        const unsigned K = (unsigned)(per * kStageK), terms = SPLIT ? kTerms - 1 : 0;
        const unsigned lenA = ((unsigned)limA * (unsigned)A.ld + terms * (unsigned)A.plane + K) * 2u;
        const unsigned lenB = ((unsigned)limB * (unsigned)B.ld + terms * (unsigned)B.plane + K) * 2u;
        // The loads of one stage after the other. What it takes to go on to the next stage is spread over the MFMAs
        // of a step (the scalar unit runs beside them, but not beside a wait).
        struct Loader {
            const unsigned *offA, *offB;
            __amdgpu_buffer_rsrc_t ra, rb;
            int planeA, planeB;      // bytes
            int per, seg, in, left, kA, kB, wave;  // in: bytes into the segment
            char *lds, *to;
            __device__ __forceinline__ void one(int v) {
                if (v < kLoadsA)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(to + v * 1024), 16, offA[v], kA, 0, 0);
                else
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        rb, (lds_void*)(to + (2 * WA - wave * (kLoadsA - kLoadsB) + v - kLoadsA) * 1024), 16,
                        offB[v - kLoadsA], kB, 0, 0);
            }
            __device__ __forceinline__ void slot(int n) { to = lds + n * kStageBytes + wave * kLoadsA * 1024; }
            // Where no stage is left the last one is loaded again and not used: every wave always has the same
            // number of loads in flight. Arithmetic, so that the loop's body stays one block.
            __device__ __forceinline__ void next() {
                --left;
                const int on = left > 0 ? kStageK * 2 : 0;
                if constexpr (SPLIT) {
                    // Uniform, which the compiler does not see by itself.
                    const int k = __builtin_amdgcn_readfirstlane(in + on), wrap = k == per * (kStageK * 2) ? 1 : 0;
                    in = k - wrap * k;
                    seg = __builtin_amdgcn_readfirstlane(seg + wrap);
                    kA = term_a(seg) * planeA + in;
                    kB = term_b(seg) * planeB + in;
                } else {
                    kA += on;
                    kB = kA;
                }
            }
        };
        const int seg0 = SPLIT ? s0 / per : 0, in0 = (s0 - seg0 * per) * (kStageK * 2), pA = SPLIT ? (int)A.plane * 2 : 0,
                  pB = SPLIT ? (int)B.plane * 2 : 0;
        Loader load{offA, offB, resource(A.p + a0 * A.ld, lenA), resource(B.p + b0 * B.ld, lenB), pA, pB, per, seg0, in0, s1 - s0,
                    term_a(seg0) * pA + in0, term_b(seg0) * pB + in0, wave, lds, lds};
        const int frag = (lane & 15) * 64 + (((lane >> 4) ^ swizzle(lane & 15)) * 16);
        const int fragA = frag + (wave >> 1) * WA * 1024, fragB = frag + (2 * WA + (wave & 1) * WB) * 1024;
        bf16x8 fa[2][WA], fb[2][WB];
        // Fragment f of a stage: first B's, which the first row of MFMAs needs together, then A's.
        const auto read = [&](int slot, int set, int f) {
            const char* const p = lds + slot * kStageBytes;
            if (f < WB) fb[set][f] = *reinterpret_cast<const bf16x8*>(p + fragB + f * 1024);
            else fa[set][f - WB] = *reinterpret_cast<const bf16x8*>(p + fragA + (f - WB) * 1024);
        };
#pragma unroll
        for (int i = 0; i < WA; ++i)
#pragma unroll
            for (int j = 0; j < WB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < kRing - 1; ++r) {
            load.slot(r);
#pragma unroll
            for (int v = 0; v < kLoads; ++v) load.one(v);
            load.next();
        }
        wait_loads<(kRing - 2) * kLoads>();
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int f = 0; f < WA + WB; ++f) read(0, 0, f);
        int slot = 0;
        const auto step = [&](int set) {
            // The next stage has landed for every wave once all have passed the barrier, and the buffer that the
            // new loads write was read by all before their last barrier but one.
            wait_loads<(kRing - 3) * kLoads>();
            __builtin_amdgcn_s_barrier();
            const int ahead = slot + 1 == kRing ? 0 : slot + 1;
            load.slot(slot == 0 ? kRing - 1 : slot - 1);
            // In this order: the fragment reads by twos in the first half, so that the next step need not wait for
            // them, a load in every second group, and after the last load the way to the next stage.
            constexpr int G = WA + WB, PER = WA * WB / G;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                __builtin_amdgcn_sched_barrier(0);
                if (g < G / 2) {
                    read(ahead, set ^ 1, 2 * g);
                    read(ahead, set ^ 1, 2 * g + 1);
                }
                if (g % 2 == 0) load.one(g / 2);
                if (g == G - 1) load.next();
#pragma unroll
                for (int m = g * PER; m < (g + 1) * PER; ++m) mfma(acc[m / WB][m % WB], fa[set][m / WB], fb[set][m % WB]);
            }
            __builtin_amdgcn_sched_barrier(0);
            slot = ahead;
        };
        for (int s = s0; s < s1; s += 2) {
            step(0);
            step(1);
            // After the last MFMA of all, the wait states that reading its result takes. They stand inside the loop,
            // ahead of any place where the compiler, which does not see MFMAs in the asm, may copy an accumulator.
            asm volatile("s_cmp_lt_i32 %0, %1\n\ts_cbranch_scc1 1f\n\ts_nop 15\n\ts_nop 15\n1:" ::"s"(s + 2), "s"(s1) : "scc");
        }
        wait_loads<0>();
        __builtin_amdgcn_s_barrier();  // the ring is free for the epilogue
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
