// What the operators of jorge_lm.h share: element types, vector loads and
// stores, sums over a wave and a workgroup, argument checks and errors.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "jorge_lm.h"

namespace jorge_lm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16;
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWave = 64;

// 16 bytes of T as floats. The types are aligned like their element, so that rows of odd widths
// keep the wide loads: global memory takes them at any address.
template <typename T>
struct Wide;
template <>
struct Wide<float> {
    static constexpr int N = 4;
    typedef float V __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Wide<bf16> {
    static constexpr int N = 8;
    typedef __bf16 V __attribute__((ext_vector_type(8), aligned(2)));
};

// A lane's ITEMS wide pieces of a row of `cols` elements that LANES lanes share; elements past the
// row's end are 0. Every load is started before anything waits for one: a piece that does not lie
// whole in the row is loaded from the last place where it does, and put right afterwards.
template <int LANES, int ITEMS, typename T>
__device__ __forceinline__ void load_row(const T* p, int cols, int lane, typename Wide<T>::V (&v)[ITEMS]) {
    constexpr int N = Wide<T>::N;
    if (cols >= N) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int c = (i * LANES + lane) * N;
            v[i] = *reinterpret_cast<const typename Wide<T>::V*>(p + (c < cols - N ? c : cols - N));
        }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int c = (i * LANES + lane) * N, left = cols - c;
        if (left < N) {
#pragma unroll
            for (int e = 0; e < N; ++e) v[i][e] = e < left ? p[c + e] : (T)0.0f;
        }
    }
}
template <typename T>
__device__ __forceinline__ void store_wide(T* p, int left, const float (&f)[Wide<T>::N]) {
    constexpr int N = Wide<T>::N;
    if (left >= N) {
        typename Wide<T>::V v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (T)f[i];
        *reinterpret_cast<typename Wide<T>::V*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = (T)f[i];
    }
}
// N elements of a parameter vector (weight, bias) of either type, as floats.
template <int N, typename P>
__device__ __forceinline__ void load_param(const P* p, int left, float (&f)[N]) {
    typedef P V __attribute__((ext_vector_type(N), aligned(sizeof(P))));
    if (left >= N) {
        const V v = *reinterpret_cast<const V*>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = (float)v[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = i < left ? (float)p[i] : 0.0f;
    }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// ---------------------------------------------------------------- host
constexpr int64_t kAlign = 256;
// A grid holds fewer than 2^32 threads: rows of one launch, and workgroups of up to 512 threads.
constexpr int64_t kRowsPerLaunch = 1 << 22;
constexpr int64_t kMaxGroups = (1ll << 32) / 512 - 1;
inline int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Records why a call is refused or failed (for jorge_lm_last_error) and returns st.
jorge_status refuse(jorge_status st, const char* why);
inline jorge_status bad(const char* why) { return refuse(JORGE_ERR_INVALID_ARGUMENT, why); }
// The status of the launches queued so far.
jorge_status launched(const char* what);

inline bool known_dtype(int32_t d) { return d == JORGE_F32 || d == JORGE_BF16; }
inline int64_t dtype_bytes(int32_t d) { return d == JORGE_BF16 ? 2 : 4; }
inline bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0; }

// A workspace handed out piece by piece; each piece starts at a multiple of kAlign.
struct Carve {
    char* base;
    int64_t used = 0;
    template <typename T>
    T* take(int64_t count) {
        char* const p = base ? base + used : nullptr;
        used += round_up(count * (int64_t)sizeof(T), kAlign);
        return reinterpret_cast<T*>(p);
    }
};

}  // namespace jorge_lm
