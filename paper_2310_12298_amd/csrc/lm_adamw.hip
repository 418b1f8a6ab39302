// AdamW over many tensors, with moments in 32 or in 8 bits, and the global norm of the gradients, for gfx950.
//
// Both are bound by HBM. A step reads weight, gradient and both moments and writes back all
// but the gradient: 28 bytes per fp32 weight with 32-bit moments, 16 with 8-bit ones. Up to
// kBatch tensors go into a launch; their pointers travel in the kernel's arguments, so
// nothing is uploaded and a call can be captured. A workgroup takes 16 blocks of 256
// elements of one tensor; a wave takes a block at a time, four elements per lane, which
// makes the largest magnitude of an 8-bit block a sum-like exchange within one wave.
//
// Measured: 25.5 M fp32 weights in 54 tensors, 32-bit moments: 110-119 us (6.0-6.5 TB/s; a large copy reaches
// 5.0-5.15, but part of these 408 MB stays in the 256 MB cache behind L2); the norm of their gradients 25.5 us
// (4.0 TB/s, as torch's sum of 1 GiB; their bytes at a copy's rate would take 20) and 4 us to finish. 168 M weights,
// 8-bit moments: 544 us (4.9 TB/s);
// reading both moments back 2 x 85 us (5.9 TB/s).
//
// The step's arithmetic rounds every operation once (no contraction), so that the same
// formula written out elsewhere in 32 bits gives the same moments to the bit: a code of
// four mantissa bits would turn a last bit into six percent.
#include "lm_common.hpp"

#include <math.h>

namespace jorge_lm {
namespace {

constexpr int kBlock = JORGE_ADAMW_BLOCK;
constexpr int kWaveBlocks = 4;               // blocks per wave
constexpr int kGroupBlocks = 4 * kWaveBlocks;  // per workgroup of four waves
static_assert(kBlock == 64 * 4, "a block is a wave of four elements per lane");

struct TensorArg {
    void* param;
    const void* grad;
    int64_t numel;
    uint32_t block;  // first block in the moments
    uint32_t group;  // first workgroup of the launch
};
constexpr int kBatch = 112;  // 3.5 KB of a kernel's 4 KB of arguments
struct TensorBatch {
    TensorArg t[kBatch];
    int n;
};

// The tensor that a workgroup belongs to.
__device__ __forceinline__ int find_tensor(const TensorBatch& b, uint32_t group) {
    int low = 0, high = b.n - 1;
    while (low < high) {
        const int mid = (low + high + 1) >> 1;
        if (b.t[mid].group <= group) low = mid;
        else high = mid - 1;
    }
    return low;
}

// Four elements at p + c of a tensor of n elements as floats (0 past its end), and back.
template <typename T>
__device__ __forceinline__ void load4(const T* p, int64_t c, int64_t n, float (&f)[4]) {
    typedef T V __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (c + 4 <= n) {
        const V v = *reinterpret_cast<const V*>(p + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = (float)v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = c + e < n ? (float)p[c + e] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, int64_t c, int64_t n, const float (&f)[4]) {
    typedef T V __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (c + 4 <= n) {
        V v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (T)f[e];
        *reinterpret_cast<V*>(p + c) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < n) p[c + e] = (T)f[e];
    }
}

// ---------------------------------------------------------------- 8-bit moments
__device__ __forceinline__ float pow2(int e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

// First: sign, 3 exponent bits, 4 mantissa bits. Second: 4 exponent bits, 4 mantissa bits.
template <bool SIGNED>
struct Code {
    static constexpr int kBias = SIGNED ? 7 : 15;
    static constexpr uint32_t kMax = SIGNED ? 127 : 255;

    // The value of a code times 2^(k - 127): the code's exponent and mantissa bits are the upper bits
    // of a float whose exponent is off by 127 - bias (E = 0 gives a subnormal of the right value), and
    // products with powers of two are exact.
    static __device__ __forceinline__ float value(uint32_t code, uint32_t k) {
        const float y = __builtin_bit_cast(float, (code & kMax) << 19) * pow2(127 - kBias);
        const float x = y * __builtin_bit_cast(float, k << 23);
        return SIGNED && (code & 128) ? -x : x;
    }
    // The block's scale from its largest magnitude: the least k in 1 .. 253 with top <= 31/16 2^(k - 127).
    static __device__ __forceinline__ uint32_t scale(float top) {
        const uint32_t k = (__builtin_bit_cast(uint32_t, top) + 0x7ffffu) >> 23;
        return k < 1 ? 1u : k > 253 ? 253u : k;
    }
    // The code of x in a block of scale k; random: 16 bits, added below the mantissa's last one. NaN and
    // infinities: the largest code.
    static __device__ __forceinline__ uint32_t round(float x, uint32_t k, uint32_t random) {
        const float size = fabsf(x);
        const uint32_t b = __builtin_bit_cast(uint32_t, size * __builtin_bit_cast(float, (254 - k) << 23));
        const int e = (int)(b >> 23), least = 128 - kBias;   // of the float; of the smallest normal code
        // 4 mantissa bits and 16 below them, in units of the exponent, or of the smallest normal code's.
        const uint32_t man = e > 0 ? (b & 0x7fffffu) | 0x800000u : 0u;
        const int down = least - e;
        const uint32_t fixed = down <= 0 ? man >> 3 : (down > 28 ? 0u : man >> (3 + down));
        uint32_t code = ((uint32_t)(down <= 0 ? -down : 0) << 4) + ((fixed + random) >> 16);
        if (!SIGNED && x > 0.0f && code == 0) code = 1;
        if (code > kMax || !(size < INFINITY)) code = kMax;
        return SIGNED && x < 0.0f ? code | 128u : code;
    }
    // The nearest code, ties to the even one.
    static __device__ __forceinline__ uint32_t nearest(float x, uint32_t k) {
        const uint32_t low = round(x, k, 0x7fff), high = round(x, k, 0x8000);
        return low == high ? low : ((low & 1) ? high : low);
    }
};

// 32 random bits for the element at `index` of the moments: a counter's hash, sums and products modulo 2^32.
__device__ __forceinline__ uint32_t random32(uint64_t index, uint32_t key) {
    uint32_t h = (uint32_t)index * 0x9E3779B1u + (uint32_t)(index >> 32) * 0x632BE5ABu + key;
    h = (h ^ (h >> 16)) * 0x7C2E1B35u;
    h = (h ^ (h >> 15)) * 0x46D8C6A9u;
    return h ^ (h >> 16);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}
__device__ __forceinline__ float finite_size(float x) {
    const float s = fabsf(x);
    return s < INFINITY ? s : 0.0f;
}

// ---------------------------------------------------------------- the step
struct StepArgs {
    void *m, *v;
    uint8_t *ms, *vs;
    const float* clip;
    float w1, w2;    // 1 - beta1, 1 - beta2
    float decay;     // lr weight_decay
    float rate;      // lr / (1 - beta1^t)
    float root;      // 1 / sqrt(1 - beta2^t)
    float eps;
    uint32_t key;    // of the random bits: seed and t
};

template <typename T, int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(TensorBatch batch, StepArgs a) {
#pragma clang fp contract(off)
    const TensorArg& t = batch.t[find_tensor(batch, blockIdx.x)];
    T* const param = (T*)t.param;
    const T* const grad = (const T*)t.grad;
    const int64_t n = t.numel;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b0 = (int64_t)(blockIdx.x - t.group) * kGroupBlocks + wave * kWaveBlocks;
    const float clip = a.clip ? *a.clip : 1.0f;
    const bool scaled = a.clip != nullptr;
    float p[kWaveBlocks][4], g[kWaveBlocks][4], m[kWaveBlocks][4], v[kWaveBlocks][4];
    uint32_t mc[kWaveBlocks], vc[kWaveBlocks], mk[kWaveBlocks], vk[kWaveBlocks];
#pragma unroll
    for (int u = 0; u < kWaveBlocks; ++u) {
        const int64_t c = (b0 + u) * kBlock + lane * 4;
        if ((b0 + u) * kBlock >= n) break;
        load4(param, c, n, p[u]);
        load4(grad, c, n, g[u]);
        const int64_t at = ((int64_t)t.block + b0 + u) * kBlock + lane * 4;
        if constexpr (BITS == 32) {
            const f32x4 x = *reinterpret_cast<const f32x4*>((const float*)a.m + at);
            const f32x4 y = *reinterpret_cast<const f32x4*>((const float*)a.v + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[u][e] = x[e];
                v[u][e] = y[e];
            }
        } else {
            mc[u] = *reinterpret_cast<const uint32_t*>((const uint8_t*)a.m + at);
            vc[u] = *reinterpret_cast<const uint32_t*>((const uint8_t*)a.v + at);
            mk[u] = a.ms[t.block + b0 + u];
            vk[u] = a.vs[t.block + b0 + u];
        }
    }
#pragma unroll
    for (int u = 0; u < kWaveBlocks; ++u) {
        const int64_t c = (b0 + u) * kBlock + lane * 4;
        if ((b0 + u) * kBlock >= n) break;
        if constexpr (BITS == 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[u][e] = Code<true>::value((mc[u] >> (8 * e)) & 255, mk[u]);
                v[u][e] = Code<false>::value((vc[u] >> (8 * e)) & 255, vk[u]);
            }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float gr = scaled ? g[u][e] * clip : g[u][e];
            m[u][e] = m[u][e] + (gr - m[u][e]) * a.w1;
            v[u][e] = v[u][e] + (gr * gr - v[u][e]) * a.w2;
            const float d = sqrtf(v[u][e]) * a.root + a.eps;
            p[u][e] = p[u][e] - (p[u][e] * a.decay + (m[u][e] * a.rate) / d);
            if (c + e >= n) m[u][e] = v[u][e] = 0.0f;  // what pads the last block stays zero
        }
        store4(param, c, n, p[u]);
        const int64_t at = ((int64_t)t.block + b0 + u) * kBlock + lane * 4;
        if constexpr (BITS == 32) {
            *reinterpret_cast<f32x4*>((float*)a.m + at) = f32x4{m[u][0], m[u][1], m[u][2], m[u][3]};
            *reinterpret_cast<f32x4*>((float*)a.v + at) = f32x4{v[u][0], v[u][1], v[u][2], v[u][3]};
        } else {
            float mt = 0.0f, vt = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mt = fmaxf(mt, finite_size(m[u][e]));
                vt = fmaxf(vt, finite_size(v[u][e]));
            }
            const uint32_t km = Code<true>::scale(wave_max(mt)), kv = Code<false>::scale(wave_max(vt));
            uint32_t mo = 0, vo = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t r = random32((uint64_t)(at + e), a.key);
                mo |= Code<true>::round(m[u][e], km, r & 0xffff) << (8 * e);
                vo |= Code<false>::round(v[u][e], kv, r >> 16) << (8 * e);
            }
            *reinterpret_cast<uint32_t*>((uint8_t*)a.m + at) = mo;
            *reinterpret_cast<uint32_t*>((uint8_t*)a.v + at) = vo;
            if (lane == 0) {
                a.ms[t.block + b0 + u] = (uint8_t)km;
                a.vs[t.block + b0 + u] = (uint8_t)kv;
            }
        }
    }
}

// ---------------------------------------------------------------- reading and writing 8-bit moments
template <bool SIGNED, typename T>
__global__ __launch_bounds__(256) void moments_read_kernel(const uint8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scales, int64_t count,
                                                           T* __restrict__ out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, at = i * 16;  // 16 elements, all of one block
    if (at >= count * kBlock) return;
    const uint32_t k = scales[at / kBlock];
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 c = *reinterpret_cast<const u32x4*>(codes + at);
    float f[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = Code<SIGNED>::value((c[e / 4] >> (8 * (e & 3))) & 255, k);
#pragma unroll
    for (int e = 0; e < 16; e += Wide<T>::N) {
        float o[Wide<T>::N];
#pragma unroll
        for (int j = 0; j < Wide<T>::N; ++j) o[j] = f[e + j];
        store_wide(out + at + e, Wide<T>::N, o);
    }
}

template <bool SIGNED>
__global__ __launch_bounds__(256) void moments_write_kernel(uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                            int64_t count, const float* __restrict__ values) {
    const int64_t b = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= count) return;
    const int lane = threadIdx.x & 63;
    const int64_t at = b * kBlock + lane * 4;
    float x[4], top = 0.0f;
    load4(values, at, count * kBlock, x);
#pragma unroll
    for (int e = 0; e < 4; ++e) top = fmaxf(top, finite_size(x[e]));
    const uint32_t k = Code<SIGNED>::scale(wave_max(top));
    uint32_t o = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) o |= Code<SIGNED>::nearest(x[e], k) << (8 * e);
    *reinterpret_cast<uint32_t*>(codes + at) = o;
    if (lane == 0) scales[b] = (uint8_t)k;
}

// ---------------------------------------------------------------- the norm
constexpr int kNormGroup = 16384;  // elements per workgroup
template <typename T>
__global__ __launch_bounds__(256) void norm_partials_kernel(TensorBatch batch, double* __restrict__ partial) {
    __shared__ double red[4];
    const TensorArg& t = batch.t[find_tensor(batch, blockIdx.x)];
    const T* const g = (const T*)t.grad;
    constexpr int N = Wide<T>::N;
    const int64_t c0 = (int64_t)(blockIdx.x - t.group) * kNormGroup;
    const int cols = (int)(t.numel - c0 < kNormGroup ? t.numel - c0 : kNormGroup);
    constexpr int ROUND = 4 * 256 * N;  // elements per round of four pieces per lane
    float s[4] = {};
    for (int c = 0; c < cols; c += ROUND) {
        typename Wide<T>::V v[4];
        load_row<256>(g + c0 + c, cols - c, threadIdx.x, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) s[i] += (float)v[i][e] * (float)v[i][e];
    }
    const double sum = wave_sum(((double)s[0] + (double)s[1]) + ((double)s[2] + (double)s[3]));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(1024) void norm_finish_kernel(const double* __restrict__ partial, int64_t n,
                                                           float max_norm, float* __restrict__ out) {
    __shared__ double red[16];
    double s[4] = {};
    int64_t i = threadIdx.x;
    for (; i + 3 * 1024 < n; i += 4 * 1024)
#pragma unroll
        for (int u = 0; u < 4; ++u) s[u] += partial[i + u * 1024];
    for (; i < n; i += 1024) s[0] += partial[i];
    const double sum = wave_sum((s[0] + s[1]) + (s[2] + s[3]));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int w = 0; w < 16; ++w) t += red[w];
        const float norm = (float)sqrt(t);
        out[0] = norm;
        float f = 1.0f;
        if (max_norm > 0.0f) {
            f = max_norm / norm;
            f = f > 1.0f ? 1.0f : f;  // a NaN stays
        }
        out[1] = f;
    }
}

// ---------------------------------------------------------------- host
constexpr int64_t kMostElements = (int64_t)1 << 38;  // of a tensor

jorge_status check_tensors(const jorge_adamw_tensor* t, int32_t n, bool step) {
    if (n < 0 || (n > 0 && !t)) return bad("adamw: n >= 0 tensors are needed");
    for (int32_t i = 0; i < n; ++i) {
        if (!known_dtype(t[i].dtype)) return bad("adamw: unknown element type");
        if (t[i].numel < 0) return bad("adamw: numel >= 0 is needed");
        if (t[i].numel > kMostElements)
            return refuse(JORGE_ERR_UNSUPPORTED, "adamw: a tensor of more than 2^38 elements");
        if (t[i].numel == 0) continue;
        if (!t[i].grad || (step && !t[i].param)) return bad("adamw: a tensor's pointer is null");
        const int64_t e = dtype_bytes(t[i].dtype);
        if (!aligned(t[i].grad, e) || (step && !aligned(t[i].param, e)))
            return bad("adamw: a pointer is not aligned to its element");
    }
    return JORGE_OK;
}

jorge_status check_moments(const jorge_adamw_moments* m) {
    if (!m) return bad("adamw: moments are needed");
    if (m->bits != 32 && m->bits != 8) return bad("adamw: bits must be 32 or 8");
    if (m->blocks < 0 || m->blocks > (int64_t)UINT32_MAX) return bad("adamw: blocks must be in [0, 2^32)");
    if (m->blocks == 0) return JORGE_OK;
    if (!m->exp_avg || !m->exp_avg_sq) return bad("adamw: the moments' buffers are needed");
    if (!aligned(m->exp_avg, 16) || !aligned(m->exp_avg_sq, 16))
        return bad("adamw: the moments must be aligned to 16 bytes");
    if (m->bits == 8 && (!m->exp_avg_scale || !m->exp_avg_sq_scale))
        return bad("adamw: 8-bit moments need their scales");
    return JORGE_OK;
}

// Calls launch(batch, groups) over the tensors of one element type, in batches.
template <typename F>
jorge_status batches(const jorge_adamw_tensor* t, int32_t n, int32_t dtype, int64_t per_group, F&& launch) {
    TensorBatch b;
    b.n = 0;
    int64_t groups = 0;
    const auto flush = [&]() -> jorge_status {
        if (b.n == 0) return JORGE_OK;
        launch(b, groups);
        b.n = 0;
        groups = 0;
        return launched("adamw");
    };
    for (int32_t i = 0; i < n; ++i) {
        if (t[i].dtype != dtype || t[i].numel == 0) continue;
        // A tensor with more workgroups than a grid holds goes in pieces of whole groups.
        for (int64_t at = 0; at < t[i].numel;) {
            if (b.n == kBatch || groups == kMaxGroups) {
                const jorge_status st = flush();
                if (st != JORGE_OK) return st;
            }
            const int64_t room = (kMaxGroups - groups) * per_group, left = t[i].numel - at;
            const int64_t take = left < room ? left : room;
            TensorArg& a = b.t[b.n++];
            const int64_t e = dtype_bytes(dtype);
            a.param = (char*)t[i].param + at * e;
            a.grad = (const char*)t[i].grad + at * e;
            a.numel = take;
            a.block = (uint32_t)(t[i].block + at / kBlock);
            a.group = (uint32_t)groups;
            groups += ceil_div(take, per_group);
            at += take;
        }
    }
    return flush();
}

int64_t norm_groups(const jorge_adamw_tensor* t, int32_t n) {
    int64_t g = 0;
    for (int32_t i = 0; i < n; ++i) g += ceil_div(t[i].numel, kNormGroup);
    return g;
}

// Blocks of moments that one launch reads or writes: a wave or less each, and a grid holds fewer than 2^32 threads.
constexpr int64_t kBlocksPerLaunch = 1 << 24;

jorge_status check_range(const jorge_adamw_moments* m, int32_t second, int64_t first, int64_t count, const void* p) {
    const jorge_status st = check_moments(m);
    if (st != JORGE_OK) return st;
    if (m->bits != 8) return bad("adamw: 32-bit moments are read and written in place");
    if (second != 0 && second != 1) return bad("adamw: second must be 0 or 1");
    if (first < 0 || count < 0 || first > m->blocks || count > m->blocks - first)
        return bad("adamw: blocks outside the moments");
    if (count > 0 && !p) return bad("adamw: a buffer is needed");
    return JORGE_OK;
}

}  // namespace
}  // namespace jorge_lm

using namespace jorge_lm;

extern "C" {

jorge_status jorge_gradient_norm_workspace(const jorge_adamw_tensor* tensors, int32_t n, int64_t* bytes) {
    if (!bytes) return bad("gradient norm: bytes is needed");
    if (n < 0 || (n > 0 && !tensors)) return bad("gradient norm: n >= 0 tensors are needed");
    for (int32_t i = 0; i < n; ++i) {
        if (tensors[i].numel < 0) return bad("gradient norm: numel >= 0 is needed");
        if (tensors[i].numel > kMostElements)
            return refuse(JORGE_ERR_UNSUPPORTED, "gradient norm: a tensor of more than 2^38 elements");
    }
    *bytes = round_up((norm_groups(tensors, n) + 1) * (int64_t)sizeof(double), kAlign);
    return JORGE_OK;
}

jorge_status jorge_gradient_norm(const jorge_adamw_tensor* tensors, int32_t n, double max_norm, float* out,
                                 void* workspace, int64_t workspace_bytes, void* hip_stream) {
    jorge_status st = check_tensors(tensors, n, false);
    if (st != JORGE_OK) return st;
    if (!(max_norm >= 0.0) || !(max_norm - max_norm == 0.0))
        return bad("gradient norm: max_norm must be finite and not negative");
    if (!out || !aligned(out, 4)) return bad("gradient norm: out is needed");
    const int64_t groups = norm_groups(tensors, n);
    if (!workspace || !aligned(workspace, kAlign))
        return bad("gradient norm: a workspace aligned to 256 bytes is needed");
    if (workspace_bytes < round_up((groups + 1) * (int64_t)sizeof(double), kAlign))
        return bad("gradient norm: the workspace is too small");
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    double* partial = (double*)workspace;
    double* at = partial;
    for (const int32_t dtype : {JORGE_F32, JORGE_BF16}) {
        st = batches(tensors, n, dtype, kNormGroup, [&](const TensorBatch& b, int64_t g) {
            if (dtype == JORGE_F32) norm_partials_kernel<float><<<dim3((unsigned)g), dim3(256), 0, s>>>(b, at);
            else norm_partials_kernel<bf16><<<dim3((unsigned)g), dim3(256), 0, s>>>(b, at);
            at += g;
        });
        if (st != JORGE_OK) return st;
    }
    norm_finish_kernel<<<dim3(1), dim3(1024), 0, s>>>(partial, at - partial, (float)max_norm, out);
    return launched("gradient norm");
}

jorge_status jorge_adamw_step(const jorge_adamw_tensor* tensors, int32_t n, const jorge_adamw_moments* moments,
                              int64_t t, double lr, double beta1, double beta2, double eps, double weight_decay,
                              const float* clip, void* hip_stream) {
    jorge_status st = check_tensors(tensors, n, true);
    if (st != JORGE_OK) return st;
    if ((st = check_moments(moments)) != JORGE_OK) return st;
    int64_t end = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (tensors[i].numel == 0) continue;
        if (tensors[i].block < end || tensors[i].block > moments->blocks ||
            ceil_div(tensors[i].numel, kBlock) > moments->blocks - tensors[i].block)
            return bad("adamw: the tensors' blocks must ascend without overlap and lie within the moments");
        end = tensors[i].block + ceil_div(tensors[i].numel, kBlock);
    }
    const auto finite = [](double x) { return x - x == 0.0; };
    if (t < 1) return bad("adamw: t >= 1 is needed");
    if (!(lr >= 0.0) || !(eps >= 0.0) || !(weight_decay >= 0.0) || !finite(lr) || !finite(eps) || !finite(weight_decay))
        return bad("adamw: lr, eps and weight_decay must be finite and not negative");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0))
        return bad("adamw: the betas must be in [0, 1)");
    if (!aligned(clip, 4)) return bad("adamw: clip is not aligned");
    StepArgs a{};
    a.m = moments->exp_avg;
    a.v = moments->exp_avg_sq;
    a.ms = moments->exp_avg_scale;
    a.vs = moments->exp_avg_sq_scale;
    a.clip = clip;
    a.w1 = (float)(1.0 - beta1);
    a.w2 = (float)(1.0 - beta2);
    a.decay = (float)(lr * weight_decay);
    a.rate = (float)(lr / (1.0 - pow(beta1, (double)t)));
    a.root = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)t)));
    a.eps = (float)eps;
    a.key = moments->seed * 0x85157AF5u + (uint32_t)t * 0x2C9277B5u;
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    for (const int32_t dtype : {JORGE_F32, JORGE_BF16}) {
        st = batches(tensors, n, dtype, kGroupBlocks * kBlock, [&](const TensorBatch& b, int64_t g) {
            const dim3 grid((unsigned)g), block(256);
            if (dtype == JORGE_F32) {
                if (moments->bits == 32) adamw_kernel<float, 32><<<grid, block, 0, s>>>(b, a);
                else adamw_kernel<float, 8><<<grid, block, 0, s>>>(b, a);
            } else {
                if (moments->bits == 32) adamw_kernel<bf16, 32><<<grid, block, 0, s>>>(b, a);
                else adamw_kernel<bf16, 8><<<grid, block, 0, s>>>(b, a);
            }
        });
        if (st != JORGE_OK) return st;
    }
    return JORGE_OK;
}

jorge_status jorge_adamw_read(const jorge_adamw_moments* moments, int32_t second, int64_t first, int64_t count,
                              void* out, int32_t dtype, void* hip_stream) {
    const jorge_status st = check_range(moments, second, first, count, out);
    if (st != JORGE_OK) return st;
    if (!known_dtype(dtype)) return bad("adamw: unknown element type");
    if (!aligned(out, dtype_bytes(dtype))) return bad("adamw: out is not aligned to its element");
    if (count == 0) return JORGE_OK;
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    const uint8_t* codes = (const uint8_t*)(second ? moments->exp_avg_sq : moments->exp_avg) + first * kBlock;
    const uint8_t* scales = (second ? moments->exp_avg_sq_scale : moments->exp_avg_scale) + first;
    for (int64_t left = count; left > 0;) {
        const int64_t n = left < kBlocksPerLaunch ? left : kBlocksPerLaunch;
        const dim3 grid((unsigned)ceil_div(n * kBlock, 256 * 16)), block(256);
        if (dtype == JORGE_F32) {
            if (second) moments_read_kernel<false, float><<<grid, block, 0, s>>>(codes, scales, n, (float*)out);
            else moments_read_kernel<true, float><<<grid, block, 0, s>>>(codes, scales, n, (float*)out);
        } else {
            if (second) moments_read_kernel<false, bf16><<<grid, block, 0, s>>>(codes, scales, n, (bf16*)out);
            else moments_read_kernel<true, bf16><<<grid, block, 0, s>>>(codes, scales, n, (bf16*)out);
        }
        left -= n;
        codes += n * kBlock;
        scales += n;
        out = (char*)out + n * kBlock * dtype_bytes(dtype);
    }
    return launched("adamw");
}

jorge_status jorge_adamw_write(const jorge_adamw_moments* moments, int32_t second, int64_t first, int64_t count,
                               const float* values, void* hip_stream) {
    const jorge_status st = check_range(moments, second, first, count, values);
    if (st != JORGE_OK) return st;
    if (!aligned(values, 4)) return bad("adamw: values is not aligned to its element");
    if (count == 0) return JORGE_OK;
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    uint8_t* codes = (uint8_t*)(second ? moments->exp_avg_sq : moments->exp_avg) + first * kBlock;
    uint8_t* scales = (second ? moments->exp_avg_sq_scale : moments->exp_avg_scale) + first;
    for (int64_t left = count; left > 0;) {
        const int64_t n = left < kBlocksPerLaunch ? left : kBlocksPerLaunch;
        const dim3 grid((unsigned)ceil_div(n, 4)), block(256);
        if (second) moments_write_kernel<false><<<grid, block, 0, s>>>(codes, scales, n, values);
        else moments_write_kernel<true><<<grid, block, 0, s>>>(codes, scales, n, values);
        left -= n;
        codes += n * kBlock;
        scales += n;
        values += n * kBlock;
    }
    return launched("adamw");
}

}  // extern "C"
