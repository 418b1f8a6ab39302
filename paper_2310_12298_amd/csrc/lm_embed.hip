// Embedding lookup with scaling, and its gradient, for gfx950.
//
// Forward: a gather of rows, bound by HBM (each distinct row read, each output row written).
//
// Backward: dtable[v] is the sum of the rows of dout whose token is v, and every row of
// dtable is written. Bound by HBM too: dout read once, dtable written once. Float atomics
// would make the sum's order, and so its last bits, a matter of timing, and serialise on
// the tokens that make up most of a text. So the tokens are sorted:
//   1. tiles of 4096 tokens, each by one workgroup in LDS: a stable radix sort, so equal
//      tokens keep their order of position. (One tile of 16384 takes 37 us, bound by the one
//      CU's LDS.);
//   2. where there are several tiles, up to 16 sorted runs are merged per launch: an
//      element's place is its place in its own run plus, in each of the others, the number
//      of elements before it, by binary searches that go on side by side;
//   3. the sorted list is cut into chunks of equal length, whatever the tokens: a wave sums
//      the runs of equal tokens of one chunk, in order, eight rows in flight. A run within
//      the chunk is a finished row of dtable. The first and the last run of a chunk may
//      go on in its neighbours: their sums go to the workspace. Other waves of the same
//      launch write zeros to the rows that no token takes;
//   4. the runs that cross chunks: their chunks' sums are added by a workgroup per run.
// A token that half of all positions hold is thus spread over as many waves as any others; what it adds is the join of
// its chunks (all tokens equal against a Zipf distribution: 16384 of 2048 columns 54 against 49 us, 65536 of 512 76
// against 68).
//
// Measured: 16384 tokens, 50000 x 2048 bf16: forward 21 us (134 MB to move at most, 6.3 TB/s: repeated rows
// come from the cache), sorting 12, merging 8.5, sums and zeros 53-62 (272 MB, 4.4-5.1 TB/s), joining 7.
// 65536 tokens, half of them one token, 8192 x 512 fp32: 28-33, 11.5, 21.5, 33 (151 MB, 4.6 TB/s) and 16 us.
#include "lm_common.hpp"

#include <utility>

namespace jorge_lm {
namespace {

// ---------------------------------------------------------------- forward
constexpr int kFwdItems = 4;
// LANES lanes share kFwdItems * LANES wide pieces of one row; blockIdx.y counts such slabs.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void embed_forward_kernel(const int64_t* __restrict__ tokens, int64_t count,
                                                            const T* __restrict__ table, int64_t ldt, int64_t vocab,
                                                            int cols, float scale, T* __restrict__ out, int64_t ldo) {
    constexpr int N = Wide<T>::N;
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= count) return;
    const int64_t tok = tokens[row];
    const int c0 = blockIdx.y * (kFwdItems * LANES * N);
    const bool live = tok >= 0 && tok < vocab;
    typename Wide<T>::V v[kFwdItems];
    load_row<LANES>(table + (live ? tok : 0) * ldt + c0, cols - c0, lane, v);
#pragma unroll
    for (int i = 0; i < kFwdItems; ++i) {
        const int c = c0 + (i * LANES + lane) * N;
        if (c >= cols) break;
        float f[N];
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = live ? (float)v[i][e] * scale : 0.0f;
        store_wide(out + row * ldo + c, cols - c, f);
    }
}

// ---------------------------------------------------------------- sorting
// A sorted element: the token (vocab for one that stands for none: behind all others) and its position.
struct Entry {
    uint32_t key, pos;
};

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 4;
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kDigitBits = 8;
constexpr int kDigits = 1 << kDigitBits;

// Element (wave, item, lane) of a tile is at wave * 64 ITEMS + item * 64 + lane, in this order.
// Each pass ranks the elements of one digit value in that order: within 64 elements by the lanes
// that share the digit (found with one ballot per bit), then by a wave's own counters, then by a
// prefix sum over (digit, wave).
template <int ITEMS>
__global__ __launch_bounds__(kSortThreads) void sort_tiles_kernel(const int64_t* __restrict__ tokens, int64_t count,
                                                                  int64_t vocab, int64_t padding, int bits,
                                                                  Entry* __restrict__ out) {
    __shared__ Entry held[kSortThreads * ITEMS];
    __shared__ uint32_t counts[kDigits][kSortWaves];
    __shared__ uint32_t totals[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t base = (int64_t)blockIdx.x * kSortTile;
    const int n = (int)(count - base < kSortThreads * ITEMS ? count - base : kSortThreads * ITEMS);
    Entry e[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int k = wave * 64 * ITEMS + i * 64 + lane;
        uint32_t key = 0xffffffffu;  // past the end: behind everything
        if (k < n) {
            const int64_t t = tokens[base + k];
            key = t >= 0 && t < vocab && t != padding ? (uint32_t)t : (uint32_t)vocab;
        }
        e[i] = {key, (uint32_t)(base + k)};
    }
    for (int shift = 0; shift < bits; shift += kDigitBits) {
        for (int k = tid; k < kDigits * kSortWaves; k += kSortThreads) (&counts[0][0])[k] = 0;
        __syncthreads();
        uint32_t rank[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const uint32_t d = (e[i].key >> shift) & (kDigits - 1);
            uint64_t same = ~0ull;
#pragma unroll
            for (int b = 0; b < kDigitBits; ++b) {
                const bool set = (d >> b) & 1;
                const uint64_t with = __ballot(set);
                same &= set ? with : ~with;
            }
            const int first = __ffsll((unsigned long long)same) - 1;
            uint32_t before = 0;
            if (lane == first) before = atomicAdd(&counts[d][wave], (uint32_t)__popcll(same));
            rank[i] = __shfl(before, first) + __popcll(same & ((1ull << lane) - 1));
        }
        __syncthreads();
        // Exclusive prefix sum over the counts, digit by digit and in each the waves in order: four per thread.
        static_assert(kDigits * kSortWaves == 4 * kSortThreads, "four counts per thread");
        uint32_t* const mine = &counts[0][0] + 4 * tid;
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            c[u] = sum;
            sum += mine[u];
        }
        uint32_t upto = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t o = __shfl_up(upto, off);
            if (lane >= off) upto += o;
        }
        if (lane == 63) totals[wave] = upto;
        __syncthreads();
        uint32_t start = upto - sum;
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) start += w < wave ? totals[w] : 0u;
#pragma unroll
        for (int u = 0; u < 4; ++u) mine[u] = start + c[u];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) held[counts[(e[i].key >> shift) & (kDigits - 1)][wave] + rank[i]] = e[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) e[i] = held[wave * 64 * ITEMS + i * 64 + lane];
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int k = wave * 64 * ITEMS + i * 64 + lane;
        if (k < n) out[base + k] = e[i];
    }
}

// Elements of the sorted list a[0 .. n) that come before `key`: below it, or equal to it too (`equal`).
__device__ __forceinline__ int64_t before(const Entry* __restrict__ a, int64_t n, uint32_t key, bool equal) {
    int64_t low = 0, high = n;
    while (low < high) {
        const int64_t mid = (low + high) >> 1;
        const uint32_t k = a[mid].key;
        if (equal ? k <= key : k < key) low = mid + 1;
        else high = mid;
    }
    return low;
}

constexpr int kMergeRuns = 16;
// Merges groups of up to RUNS sorted runs of length `run` (the last may be shorter). steps: halvings until a run's
// length is 0.
template <int RUNS>
__global__ __launch_bounds__(256) void merge_kernel(const Entry* __restrict__ in, int count, int run, int steps,
                                                    Entry* __restrict__ out) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    const Entry e = in[i];
    const int mine = i / run, g = mine / RUNS * RUNS;
    int low[RUNS], high[RUNS];
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
        const int s = (g + r) * run;
        low[r] = s < count ? s : count - 1;
        high[r] = s >= count ? low[r] : count - s < run ? count : s + run;
        if (g + r == mine) low[r] = high[r] = i;  // its place among its own run is known
    }
    for (int k = 0; k < steps; ++k) {
        uint32_t key[RUNS];
#pragma unroll
        for (int r = 0; r < RUNS; ++r) {
            const int mid = (low[r] + high[r]) >> 1;
            key[r] = in[mid < count ? mid : count - 1].key;
        }
#pragma unroll
        for (int r = 0; r < RUNS; ++r) {
            // Equal tokens of an earlier run come first.
            const int mid = (low[r] + high[r]) >> 1;
            const bool first = g + r < mine ? key[r] <= e.key : key[r] < e.key;
            if (low[r] < high[r]) {
                if (first) low[r] = mid + 1;
                else high[r] = mid;
            }
        }
    }
    int at = g * run;
#pragma unroll
    for (int r = 0; r < RUNS; ++r) {
        const int s = (g + r) * run;
        if (s < count) at += low[r] - s;
    }
    out[at] = e;
}

// ---------------------------------------------------------------- sums
constexpr int kSumItems = 8;  // rows in flight
constexpr int kZeroRows = 64;

struct SumArgs {
    const Entry* sorted;
    int64_t count, vocab, lddo, lddt;
    float* partial;  // [2][chunks][ldp]: sums of a chunk's first run and of its last, where they cross its ends
    int64_t chunks;
    int cols, chunk, slabs;
    // cols rounded up to 64, and 64 more: a long run's rows, 2 KB apart for 512 columns, would all lie in the same few
    // channels of the L2.
    int ldp;
    float scale;
};

// blockIdx.x < sum_groups: four waves, a (chunk, slab of 64 wide pieces) each. Beyond: zero rows, a (64 rows, slab)
// each.
template <typename T>
__global__ __launch_bounds__(256) void embed_sums_kernel(SumArgs a, const T* __restrict__ dout, T* __restrict__ dtable,
                                                         int64_t sum_groups) {
    constexpr int N = Wide<T>::N;
    const int lane = threadIdx.x & 63;
    const bool zeros = blockIdx.x >= sum_groups;
    const int64_t unit =
        ((int64_t)blockIdx.x - (zeros ? sum_groups : 0)) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t part = unit / a.slabs;
    const int c = ((int)(unit % a.slabs) * 64 + lane) * N, left = a.cols - c;
    if (zeros) {
        const int64_t v0 = part * kZeroRows;
        if (v0 >= a.vocab) return;
        // Lane l: whether row v0 + l has a token.
        const int64_t v = v0 + lane;
        const int64_t k = before(a.sorted, a.count, (uint32_t)(v < a.vocab ? v : a.vocab - 1), false);
        const bool none = v < a.vocab && !(k < a.count && a.sorted[k].key == (uint32_t)v);
        uint64_t todo = __ballot(none);
        const float zero[N] = {};
        while (todo) {
            const int r = __ffsll((unsigned long long)todo) - 1;
            todo &= todo - 1;
            if (left > 0) store_wide(dtable + (v0 + r) * a.lddt + c, left, zero);
        }
        return;
    }
    if (part >= a.chunks) return;
    const int64_t s0 = part * a.chunk, s1 = s0 + a.chunk < a.count ? s0 + a.chunk : a.count;
    const uint32_t prev = s0 > 0 ? a.sorted[s0 - 1].key : 0xffffffffu;
    const uint32_t next = s1 < a.count ? a.sorted[s1].key : 0xffffffffu;
    const bool whole = left >= N;
    float acc[N] = {};
    int64_t begin = s0;  // of the run being summed
    uint32_t key = a.sorted[s0].key;
    const auto flush = [&](int64_t end) {
        if (key < a.vocab && left > 0) {
            const bool from_left = begin == s0 && key == prev, to_right = end == s1 && key == next;
            if (!from_left && !to_right) {
                float o[N];
#pragma unroll
                for (int e = 0; e < N; ++e) o[e] = acc[e] * a.scale;
                store_wide(dtable + (int64_t)key * a.lddt + c, left, o);
            } else {
                float* const p = a.partial + (part + (begin == s0 ? 0 : a.chunks)) * a.ldp + c;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (e < left) p[e] = acc[e];
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = 0.0f;
        begin = end;
    };
    for (int64_t s = s0; s < s1; s += kSumItems) {
        typename Wide<T>::V v[kSumItems];
        uint32_t keys[kSumItems];
#pragma unroll
        for (int u = 0; u < kSumItems; ++u) {
            // Past the chunk's end: its last row again, which is not added.
            const Entry x = a.sorted[s + u < s1 ? s + u : s1 - 1];
            keys[u] = x.key;
            const T* const row = dout + (int64_t)x.pos * a.lddo;
            if (whole) {
                v[u] = *reinterpret_cast<const typename Wide<T>::V*>(row + c);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[u][e] = e < left ? row[c + e] : (T)0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < kSumItems; ++u) {
            if (s + u >= s1) break;
            if (keys[u] != key) {
                flush(s + u);
                key = keys[u];
            }
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += (float)v[u][e];
        }
    }
    flush(s1);
}

// Adds the sums that the chunks of one run left, where a run starts in a chunk and goes on past its end. A workgroup
// looks at the ends of kJoinWaves neighbouring chunks, a wave at each, for a slab of 4 LANES columns: LANES lanes take
// a chunk's sums, a wave 64 / LANES chunks at a time. A wave adds a short run's sums by itself; a long run is shared by
// all waves of the workgroup. Slabs of 64 columns serve narrow tables, where a long run would have too few CUs to
// itself (one gets some 50 GB/s): 1024 chunks of 512 columns take 17 us, in slabs of 256 columns 27. Wide tables have
// enough slabs of 256, and four times as many workgroups would cost more: 16384 tokens, 2048 columns 7 us against 13.
// The whole gradient of 4000 bf16 rows, 65536 tokens, with either, Zipf-distributed and all equal: 512 columns 65 and
// 71 us in narrow slabs, 62 and 93 in wide ones; 1024 columns 82 and 85 against 73 and 102; 1536 columns 100 and 108
// against 86 and 117; 2048 columns 142 and 141 against 121 and 140.
constexpr int kJoinWaves = 8;
constexpr int kJoinAlone = 16;  // chunks after the first that a wave adds alone

__device__ __forceinline__ f32x4 add_up(const float* p, int64_t stride, int64_t k, int64_t last, int step) {
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (; k + 15 * step <= last; k += 16 * step) {
        f32x4 v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = *reinterpret_cast<const f32x4*>(p + (k + u * step) * stride);
#pragma unroll
        for (int half = 8; half > 0; half >>= 1)
#pragma unroll
            for (int u = 0; u < half; ++u) v[u] += v[u + half];
        sum += v[0];
    }
    for (; k <= last; k += step) sum += *reinterpret_cast<const f32x4*>(p + k * stride);
    return sum;
}

template <typename T, int LANES>
__global__ __launch_bounds__(kJoinWaves * 64) void embed_join_kernel(SumArgs a, T* __restrict__ dtable) {
    __shared__ f32x4 lds[kJoinWaves][LANES];
    constexpr int ROWS = 64 / LANES;
    __shared__ int64_t run_part[kJoinWaves], run_last[kJoinWaves];  // long runs
    __shared__ uint32_t run_key[kJoinWaves];
    __shared__ int64_t run_first[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / LANES;
    const int c = (blockIdx.y * LANES + lane % LANES) * 4;
    const int64_t stride = a.ldp, tails = a.chunks * stride;
    const auto write = [&](uint32_t key, const f32x4& t) {
        T* const out = dtable + (int64_t)key * a.lddt + c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.cols) out[e] = (T)(t[e] * a.scale);
    };
    const int64_t part = (int64_t)blockIdx.x * kJoinWaves + wave, s0 = part * a.chunk, s1 = s0 + a.chunk;
    bool run = s1 < a.count;
    uint32_t key = 0;
    bool fills = false;  // the run takes the whole chunk
    if (run) {
        key = a.sorted[s1].key;
        fills = a.sorted[s0].key == key;
        run = key < a.vocab && a.sorted[s1 - 1].key == key && !(fills && s0 > 0 && a.sorted[s0 - 1].key == key);
    }
    // The run's last chunk: the first whose end it does not cross. 64 ends are looked at at a time: every end, every
    // 64th, then every one again.
    int64_t last = part + 1;
    if (run)
        for (int step = 1;; step = 65 - step) {
            const int64_t next = (last + (int64_t)lane * step + step) * a.chunk;
            const uint64_t on = __ballot(next < a.count && a.sorted[next < a.count ? next : 0].key == key);
            const int crossed = ~on ? __ffsll((unsigned long long)~on) - 1 : 64;
            last += (int64_t)crossed * step;
            if (step == 1 && crossed < 64) break;
        }
    const bool alone = last - part <= kJoinAlone;
    if (lane == 0) {
        run_part[wave] = run && !alone ? part : -1;
        run_last[wave] = last;
        run_key[wave] = key;
        run_first[wave] = fills ? 0 : tails;
    }
    // The run is the last of its first chunk (its only one, if it fills it) and the first of each later one.
    // Columns past the last one, as far as a row of sums reaches, are added up and not written.
    const float* const p = a.partial + (c < a.ldp ? c : 0);
    const auto over_rows = [&](f32x4 v) {  // of a wave
#pragma unroll
        for (int off = LANES; off < 64; off <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], off);
        return v;
    };
    if (run && alone) {
        f32x4 sum = add_up(p, stride, part + 1 + sub, last, ROWS);
        if (sub == 0) sum += *reinterpret_cast<const f32x4*>(p + part * stride + (fills ? 0 : tails));
        sum = over_rows(sum);
        if (sub == 0) write(key, sum);
    }
    __syncthreads();
    for (int w = 0; w < kJoinWaves; ++w) {
        const int64_t q = run_part[w];
        if (q < 0) continue;  // the same for all waves
        f32x4 sum = add_up(p, stride, q + 1 + ROWS * wave + sub, run_last[w], ROWS * kJoinWaves);
        if (wave == 0 && sub == 0) sum += *reinterpret_cast<const f32x4*>(p + q * stride + run_first[w]);
        sum = over_rows(sum);
        __syncthreads();
        if (sub == 0) lds[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && sub == 0) {
            f32x4 t = lds[0][lane];
#pragma unroll
            for (int u = 1; u < kJoinWaves; ++u) t += lds[u][lane];
            write(run_key[w], t);
        }
    }
}

// ---------------------------------------------------------------- host
// Sorted entries per chunk: 32, and more where that would leave more than 4096 chunks' sums for one run to join. Above
// 32 entries (which are one chunk, with nothing to join) and up to 4096 it is 16: a wave sums a chunk's rows in turn,
// which is much of a short call's time. Gradient of a 4000 x 512 fp32 table in chunks of 32, 16 and 8: 64 tokens 19.3,
// 14.4, 14.4 us; 1651 tokens 24.1, 19.0, 18.5; 4096 tokens 27.8, 22.9, 23.4, and all of them equal 24.4, 24.8, 27.2.
// Over 23 to 8192 columns, 20 to 65536 tokens, Zipf-distributed or all equal, and 8 to 128 entries a chunk (80 cases),
// the rule's length takes at most 15% longer than the best, but for 4096 rows of 8192 fp32 columns that are all equal
// (63 against 48 us in 32), 6000 of 23 (36 against 31 in 16), and 16384 or 65536 equal ones of 2048 columns and more
// (16 to 24%, in 64 or 128).
int chunk_of(int64_t count) {
    int c = count > 32 && count <= 4096 ? 16 : 32;
    while (ceil_div(count, c) > 4096 && c < 4096) c *= 2;
    return c;
}

int64_t partial_row(int64_t cols) { return round_up(cols, 64) + 64; }

struct Work {
    Entry *a, *b;
    float* partial;
    int64_t bytes;
};
Work carve(void* base, int64_t count, int64_t cols) {
    Carve c{(char*)base};
    Work w{};
    w.a = c.take<Entry>(count);
    w.b = count > kSortTile ? c.take<Entry>(count) : nullptr;
    const int64_t chunks = ceil_div(count, chunk_of(count));
    w.partial = chunks > 1 ? c.take<float>(chunks * 2 * partial_row(cols)) : nullptr;
    w.bytes = c.used;
    return w;
}

jorge_status check(int64_t count, int64_t vocab, int64_t cols, int32_t dtype, double scale) {
    if (!known_dtype(dtype)) return bad("embedding: unknown element type");
    if (count < 0 || vocab < 1 || cols < 1) return bad("embedding: count >= 0, vocab >= 1 and cols >= 1 are needed");
    if (count > JORGE_EMBED_MAX_TOKENS)
        return refuse(JORGE_ERR_UNSUPPORTED, "embedding: count above JORGE_EMBED_MAX_TOKENS");
    if (vocab > JORGE_EMBED_MAX_VOCAB)
        return refuse(JORGE_ERR_UNSUPPORTED, "embedding: vocab above JORGE_EMBED_MAX_VOCAB");
    if (cols > JORGE_EMBED_MAX_COLS) return refuse(JORGE_ERR_UNSUPPORTED, "embedding: cols above JORGE_EMBED_MAX_COLS");
    if (!(scale - scale == 0.0)) return bad("embedding: scale must be finite");
    return JORGE_OK;
}

template <typename T>
void forward(const int64_t* tokens, int64_t count, const void* table, int64_t ldt, int64_t vocab, int cols, float scale,
             void* out, int64_t ldo, hipStream_t s) {
    const int64_t pieces = ceil_div(cols, Wide<T>::N);
    const auto go = [&](auto L) {
        constexpr int lanes = decltype(L)::value;
        const dim3 grid((unsigned)ceil_div(count, 256 / lanes), (unsigned)ceil_div(pieces, lanes * kFwdItems));
        embed_forward_kernel<T, lanes>
            <<<grid, dim3(256), 0, s>>>(tokens, count, (const T*)table, ldt, vocab, cols, scale, (T*)out, ldo);
    };
    // Narrow rows share a wave.
    if (pieces <= 4) go(std::integral_constant<int, 4>());
    else if (pieces <= 16) go(std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 64>());
}

template <typename T>
jorge_status backward(const void* dout, int64_t lddo, const int64_t* tokens, int64_t count, int64_t vocab, int64_t cols,
                      double scale, int64_t padding, void* dtable, int64_t lddt, void* workspace, hipStream_t s) {
    Work w = carve(workspace, count, cols);
    if (count > 0) {
        int bits = 0;
        while ((vocab >> bits) != 0) ++bits;  // keys 0 .. vocab
        const dim3 tiles((unsigned)ceil_div(count, kSortTile)), threads(kSortThreads);
        // A single short tile leaves out the elements that it does not have (1651 tokens: 13.3 us with four
        // elements per thread, 10.0 with two).
        if (count <= kSortThreads)
            sort_tiles_kernel<1><<<tiles, threads, 0, s>>>(tokens, count, vocab, padding, bits, w.a);
        else if (count <= 2 * kSortThreads)
            sort_tiles_kernel<2><<<tiles, threads, 0, s>>>(tokens, count, vocab, padding, bits, w.a);
        else
            sort_tiles_kernel<kSortItems><<<tiles, threads, 0, s>>>(tokens, count, vocab, padding, bits, w.a);
        for (int64_t run = kSortTile; run < count; run *= kMergeRuns) {
            const dim3 grid((unsigned)ceil_div(count, 256));
            int steps = 1;
            while (run >> steps) ++steps;
            if (ceil_div(count, run) <= 4)
                merge_kernel<4><<<grid, dim3(256), 0, s>>>(w.a, (int)count, (int)run, steps, w.b);
            else
                merge_kernel<kMergeRuns><<<grid, dim3(256), 0, s>>>(w.a, (int)count, (int)run, steps, w.b);
            std::swap(w.a, w.b);
        }
    }
    SumArgs a{};
    a.sorted = w.a;
    a.count = count;
    a.vocab = vocab;
    a.lddo = lddo;
    a.lddt = lddt;
    a.partial = w.partial;
    a.chunk = chunk_of(count);
    a.chunks = ceil_div(count, a.chunk);
    a.cols = (int)cols;
    a.ldp = (int)partial_row(cols);
    a.slabs = (int)ceil_div(cols, 64 * Wide<T>::N);
    a.scale = (float)scale;
    // The largest of tokens, rows and columns fit in one grid (fewer than 2^32 threads): at most 4096 chunks, and 64
    // rows or a chunk per wave and slab.
    constexpr int64_t kMostSlabs = JORGE_EMBED_MAX_COLS / (64 * 4);
    static_assert((4096 + JORGE_EMBED_MAX_VOCAB / kZeroRows) * kMostSlabs / 4 + 2 < (1ll << 32) / 256, "one launch");
    static_assert(JORGE_EMBED_MAX_TOKENS / 4096 <= 4096, "4096 chunks of up to 4096");
    const int64_t sum_groups = ceil_div(a.chunks * a.slabs, 4);
    const int64_t zero_groups = ceil_div(ceil_div(vocab, kZeroRows) * a.slabs, 4);
    embed_sums_kernel<T><<<dim3((unsigned)(sum_groups + zero_groups)), dim3(256), 0, s>>>(a, (const T*)dout, (T*)dtable,
                                                                                         sum_groups);
    if (a.chunks > 1) {
        const unsigned groups = (unsigned)ceil_div(a.chunks - 1, kJoinWaves);
        if (cols <= 1024)
            embed_join_kernel<T, 16>
                <<<dim3(groups, (unsigned)ceil_div(cols, 64)), dim3(kJoinWaves * 64), 0, s>>>(a, (T*)dtable);
        else
            embed_join_kernel<T, 64>
                <<<dim3(groups, (unsigned)ceil_div(cols, 256)), dim3(kJoinWaves * 64), 0, s>>>(a, (T*)dtable);
    }
    return launched("embedding");
}

}  // namespace
}  // namespace jorge_lm

using namespace jorge_lm;

extern "C" {

jorge_status jorge_embedding_forward(const int64_t* tokens, int64_t count, const void* table, int64_t ldt,
                                     int32_t dtype, int64_t vocab, int64_t cols, double scale, void* out,
                                     int64_t ldo, void* hip_stream) {
    const jorge_status st = check(count, vocab, cols, dtype, scale);
    if (st != JORGE_OK) return st;
    if (ldt < cols || ldo < cols) return bad("embedding: a row stride is below cols");
    if (count == 0) return JORGE_OK;
    if (!tokens || !table || !out) return bad("embedding: tokens, table and out are needed");
    const int64_t e = dtype_bytes(dtype);
    if (!aligned(tokens, 8) || !aligned(table, e) || !aligned(out, e))
        return bad("embedding: a pointer is not aligned to its element");
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    // A grid holds fewer than 2^32 threads.
    for (int64_t r0 = 0; r0 < count; r0 += kRowsPerLaunch) {
        const int64_t n = count - r0 < kRowsPerLaunch ? count - r0 : kRowsPerLaunch;
        if (dtype == JORGE_F32)
            forward<float>(tokens + r0, n, table, ldt, vocab, (int)cols, (float)scale, (float*)out + r0 * ldo, ldo, s);
        else
            forward<bf16>(tokens + r0, n, table, ldt, vocab, (int)cols, (float)scale, (bf16*)out + r0 * ldo, ldo, s);
    }
    return launched("embedding");
}

jorge_status jorge_embedding_workspace(int64_t count, int64_t vocab, int64_t cols, int64_t* bytes) {
    if (!bytes) return bad("embedding: bytes is needed");
    const jorge_status st = check(count, vocab, cols, JORGE_F32, 1.0);
    if (st != JORGE_OK) return st;
    *bytes = carve(nullptr, count, cols).bytes;
    return JORGE_OK;
}

jorge_status jorge_embedding_backward(const void* dout, int64_t lddo, const int64_t* tokens, int64_t count,
                                      int32_t dtype, int64_t vocab, int64_t cols, double scale, int64_t padding,
                                      void* dtable, int64_t lddt, void* workspace, int64_t workspace_bytes,
                                      void* hip_stream) {
    const jorge_status st = check(count, vocab, cols, dtype, scale);
    if (st != JORGE_OK) return st;
    if (lddo < cols || lddt < cols) return bad("embedding: a row stride is below cols");
    if (!dtable || (count > 0 && (!dout || !tokens))) return bad("embedding: dout, tokens and dtable are needed");
    const int64_t e = dtype_bytes(dtype);
    if (!aligned(tokens, 8) || !aligned(dout, e) || !aligned(dtable, e))
        return bad("embedding: a pointer is not aligned to its element");
    const int64_t need = carve(nullptr, count, cols).bytes;
    if (need > 0 && (!workspace || !aligned(workspace, kAlign)))
        return bad("embedding: a workspace aligned to 256 bytes is needed");
    if (workspace_bytes < need) return bad("embedding: the workspace is too small");
    const hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
    if (dtype == JORGE_F32)
        return backward<float>(dout, lddo, tokens, count, vocab, cols, scale, padding, dtable, lddt, workspace, s);
    return backward<bf16>(dout, lddo, tokens, count, vocab, cols, scale, padding, dtable, lddt, workspace, s);
}

}  // extern "C"
