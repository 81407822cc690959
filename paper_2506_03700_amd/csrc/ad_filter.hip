// Distributions that temperature, top-k, top-p and min-p make of rows of logits: draws from them, the accept / resample rule between
// them, and the distributions themselves.
//
// Ids are ordered by logit, largest first, equal ones by id; every step of a filter keeps a first part of that order, so what is kept is the ids whose key (the logit's
// bits made to compare like integers, then the id, smaller ids first) is not below the smallest kept one.  Finding that key is
// all there is to it, and nothing is sorted.  Weights exp((z - max) / T) are formed in 64 bits and held as integers, multiples of 2^-weight_bits: sums of
// integers do not depend on their order, so neither does an outcome, atomics and all, and a boundary falls where
// it falls in exact arithmetic unless it is within some 1e-11 of a border.
//
//   k_filter_top      largest logit of each segment of a row
//   k_filter_buckets  (top-k, top-p) count and weight of 2048 buckets of logits; the last workgroup of the row finds the
//                     buckets that the boundaries lie in
//   k_filter_row      weight of each segment's ids that are kept for certain, and a list of the ids in the boundaries' buckets; the
//                     last workgroup of the row finds the boundaries among those, and draws
//   k_filter_one      all of that for a row of one segment
//   k_filter_few      all of that for a small top-k: the first top_k ids of the row are among the first top_k of its segments
//   k_filter_probs, k_filter_verify: from the rows' outcomes
//
// What bounds them is not the rows (0.5 MB) but the chain of dependent loads, barriers and kernel boundaries: of a draw from 128256 logits with all three steps on,
// 24 us in three kernels (2.9, 9.7, 12.0), the last takes 1.0 for its first loads, 1.0 to 1.3 for the classes, 1.2 to publish, 1.5 for the list, 3.3 for the two
// boundaries, 0.6 to add up, 3.0 to draw.  With every entry of a boundary ranked against all others, and boundaries found through memory, it was 32; ten workgroup-wide steps per boundary in
// place of two barriers cost 2 more.  A small top-k in one kernel: 12.6 (largest 50).  A row of one segment in
// one kernel: 11.3 us for 2048 logits, 29 in four.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ad_device.h"
#include "ad_filter.h"
#include "ad_internal.h"
#include "ad_launch.h"

namespace ad {

namespace {

constexpr int NT = kFilterThreads, NW = NT / 64;
constexpr int kRank = 64;                                // entries that are ranked against each other
constexpr int kKeep = kFilterSegIds / NT;                // logits that a thread keeps (longer segments read the others again)
constexpr uint64_t kUnused = ~0ull, kTooMany = ~0ull - 1; // in places of a list (no listed logit has these bits)
constexpr int kLinear = 1792;                            // buckets of equal width

// ---------------------------------------------------------------------------------------------------
// keys, weights, buckets
// ---------------------------------------------------------------------------------------------------
// -0 counts as 0, which it equals
__device__ __forceinline__ float plain(float z) { return z + 0.0f; }
__device__ __forceinline__ uint64_t key_of(float z, int id) {
    uint32_t u = __float_as_uint(plain(z));
    u ^= (uint32_t)((int32_t)u >> 31) | 0x80000000u;
    return (uint64_t)u << 32 | (0xffffffffu - (uint32_t)id);
}
// weight relative to the largest logit, in 64 bits
__device__ __forceinline__ double weight_of(float z, float top, double inv_t) {
    double x = ((double)z - (double)top) * inv_t;
    asm("" : "+v"(x));                                   // (the same rounding wherever this is inlined)
    return exp(x);
}
__device__ __forceinline__ uint64_t whole(double w, int bits) { return (uint64_t)ldexp(w, bits); }
// 28 times the temperature below the top in steps of 1/64, then 16 steps for each factor of two
__device__ __forceinline__ int bucket_of(float z, float top, float scale) {
    const float x = (top - z) * scale;
    if (x < (float)kLinear) return (int)x;
    const uint32_t b = (__float_as_uint(x) - __float_as_uint((float)kLinear)) >> 19;
    return kLinear + (int)(b < kFilterBuckets - 1 - kLinear ? b : kFilterBuckets - 1 - kLinear);
}
__device__ __forceinline__ bool masked(float z) { return !(z > -INFINITY); }
__device__ __forceinline__ const float *row_of(const FilterArgs &a, int r) {
    return r < a.n_first ? a.z0 + (size_t)r * a.V : a.z1 + (size_t)(r - a.n_first) * a.V;
}

// ---------------------------------------------------------------------------------------------------
// a workgroup's sums and scans
// ---------------------------------------------------------------------------------------------------
struct BlockLds {
    float f[NW];
    uint64_t u[NW], u2[NW];
    int last_wg;
};
// maximum over the workgroup; not a number if one of the values is none
__device__ __forceinline__ float block_top(float v, BlockLds &L) {
    const bool nan = __any(v != v);
    v = max64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) L.f[threadIdx.x >> 6] = nan ? __uint_as_float(0x7fc00000u) : v;
    __syncthreads();
    float r = L.f[0];
    for (int w = 1; w < NW; ++w) r = (r != r || L.f[w] != L.f[w]) ? __uint_as_float(0x7fc00000u) : fmaxf(r, L.f[w]);
    return r;
}
// v of the lane that DPP control CTRL names, 0 where there is none
template <int CTRL>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xf, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xf, 0xf, false);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, int lane) {     // inclusive
    v += dpp_u64<0x111>(v);                              // row_shr 1, 2, 4, 8: within a row of 16 lanes
    v += dpp_u64<0x112>(v);
    v += dpp_u64<0x114>(v);
    v += dpp_u64<0x118>(v);
    const uint64_t r0 = lane_u64(v, 15), r1 = r0 + lane_u64(v, 31), r2 = r1 + lane_u64(v, 47);
    const int row = lane >> 4;
    return v + (row == 0 ? 0 : row == 1 ? r0 : row == 2 ? r1 : r2);
}
// sum over the threads before this one; *total: over all
__device__ __forceinline__ uint64_t block_scan(uint64_t v, BlockLds &L, uint64_t *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t in = wave_scan(v, lane);
    __syncthreads();
    if (lane == 63) L.u[wave] = in;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        before += w < wave ? L.u[w] : 0;
        all += L.u[w];
    }
    *total = all;
    return before + in - v;
}
// of two numbers at once
__device__ __forceinline__ void block_scan2(uint64_t &v, uint64_t &u, BlockLds &L, uint64_t *total_v, uint64_t *total_u) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t in = wave_scan(v, lane), iu = wave_scan(u, lane);
    __syncthreads();
    if (lane == 63) {
        L.u[wave] = in;
        L.u2[wave] = iu;
    }
    __syncthreads();
    uint64_t before = 0, all = 0, before2 = 0, all2 = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        before += w < wave ? L.u[w] : 0;
        all += L.u[w];
        before2 += w < wave ? L.u2[w] : 0;
        all2 += L.u2[w];
    }
    *total_v = all;
    *total_u = all2;
    v = before + in - v;
    u = before2 + iu - u;
}
__device__ __forceinline__ uint64_t block_sum(uint64_t v, BlockLds &L) {
    uint64_t all;
    (void)block_scan(v, L, &all);
    return all;
}
template <bool MAX>
__device__ __forceinline__ uint64_t block_extreme(uint64_t v, BlockLds &L) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, d);
        v = MAX ? (o > v ? o : v) : (o < v ? o : v);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) L.u[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t r = L.u[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) r = MAX ? (L.u[w] > r ? L.u[w] : r) : (L.u[w] < r ? L.u[w] : r);
    return r;
}

__device__ __forceinline__ uint64_t seen(const uint64_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class T>
__device__ __forceinline__ void leave(T *p, T v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// the last workgroup of n on this counter, when everything that any wavefront of any of them has left is in memory
__device__ __forceinline__ bool last_of(uint32_t *counter, int n, BlockLds &L) {
    reported();
    __syncthreads();
    return last_to_arrive(counter, n, &L.last_wg);
}

// A segment's logits: a thread has ids j0 + tid, + NT, ...; the first kKeep of them, all on their way at once, stay in registers.
struct SegLogits {
    const float *z;
    int j0, j1;
    float v[kKeep];
    __device__ __forceinline__ void load(const FilterArgs &a, int r, int seg) {
        z = row_of(a, r);
        j0 = seg * a.seg_ids;
        j1 = min(a.V, j0 + a.seg_ids);
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            const int j = j0 + (int)threadIdx.x + i * NT;
            v[i] = j < j1 ? z[j] : -INFINITY;
        }
    }
    template <class F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int i = 0; i < kKeep; ++i) f(v[i], j0 + (int)threadIdx.x + i * NT);        // (past the end: minus infinity)
        for (int j = j0 + (int)threadIdx.x + kKeep * NT; j < j1; j += NT) f(z[j], j);
    }
    // largest logit, not a number if one is none
    __device__ __forceinline__ float top(BlockLds &L) const {
        float m = -INFINITY;
        bool nan = false;
        each([&](float x, int) {
            nan |= x != x;
            m = fmaxf(m, x);
        });
        return block_top(nan ? __uint_as_float(0x7fc00000u) : m, L);
    }
};

// ---------------------------------------------------------------------------------------------------
// 1. largest logits
// ---------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(NT) k_filter_top(FilterArgs a) {
    __shared__ BlockLds L;
    SegLogits z;
    z.load(a, blockIdx.y, blockIdx.x);
    const float m = z.top(L);
    if (threadIdx.x == 0) a.s->seg_top[blockIdx.y][blockIdx.x] = m;
}

// of the row, to every thread (every wavefront looks at all segments, which saves the barriers); *bad: it has no distribution
// PUBLISHED: by other workgroups of this launch
template <bool PUBLISHED = false>
__device__ __forceinline__ float row_top(const FilterArgs &a, int r, bool *bad) {
    constexpr int PER = kFilterMaxSegs / 64;
    const int lane = threadIdx.x & 63;
    auto at = [&](int i) { return PUBLISHED ? __hip_atomic_load(&a.s->seg_top[r][i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : a.s->seg_top[r][i]; };
    float m = lane < a.n_seg ? at(lane) : -INFINITY;
    bool nan = m != m;
    if (a.n_seg > 64) {
        float v[PER - 1];
#pragma unroll
        for (int i = 1; i < PER; ++i) v[i - 1] = lane + 64 * i < a.n_seg ? at(lane + 64 * i) : -INFINITY;
#pragma unroll
        for (int i = 1; i < PER; ++i) {
            nan |= v[i - 1] != v[i - 1];
            m = fmaxf(m, v[i - 1]);
        }
    }
    m = max64(m);
    *bad = __any(nan) || !(fabsf(m) < INFINITY);
    return m;
}

// ---------------------------------------------------------------------------------------------------
// 2. buckets
// ---------------------------------------------------------------------------------------------------
// Weights are needed for top-p, counts for top-k: the other array is left alone.
struct Histogram {
    uint64_t weight[kFilterBuckets];
    uint32_t count[kFilterBuckets];
    __device__ __forceinline__ void clear(const FilterArgs &a) {
        for (int b = threadIdx.x; b < kFilterBuckets; b += NT) {
            if (a.top_p < 1.0) weight[b] = 0;
            if (a.top_k) count[b] = 0;
        }
    }
    __device__ __forceinline__ void add(const FilterArgs &a, float x, float top) {
        if (masked(x)) return;
        const int b = bucket_of(x, top, a.bucket_scale);
        if (a.top_k) atomicAdd(&count[b], 1u);
        if (a.top_p < 1.0) atomicAdd((unsigned long long *)&weight[b], (unsigned long long)whole(weight_of(x, top, a.inv_t), a.weight_bits));
    }
};

// The buckets of the boundaries from those of the whole row, of which thread t has 4 t .. 4 t + 3 (w and c are zero where that step is off).  By one workgroup.
__device__ __forceinline__ void find_buckets(const FilterArgs &a, const uint64_t (&w)[kFilterBuckets / NT], const uint32_t (&c)[kFilterBuckets / NT],
                                             FilterRow &R, BlockLds &L) {
    constexpr int PER = kFilterBuckets / NT;
    const int tid = threadIdx.x;
    __shared__ uint64_t in_k;
    uint64_t w0 = 0, c0 = 0, all_w = 0, all_c = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        w0 += w[i];
        c0 += c[i];
    }
    if (tid == 0) {
        R.p0 = kFilterBuckets;
        R.p1 = -1;
        R.bk = -1;
        R.count_k = 0;
        R.weight_p = R.weight_k = 0;
        in_k = 0;
    }
    block_scan2(w0, c0, L, &all_w, &all_c);
    if (tid == 0) R.weight = all_w;
    // top-k: the bucket of the last id it keeps (none if it keeps them all)
    if (a.top_k && (uint64_t)a.top_k < all_c) {
        uint64_t cb = c0, wb = w0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (cb < (uint64_t)a.top_k && cb + c[i] >= (uint64_t)a.top_k) {
                R.bk = tid * PER + i;
                R.count_k = (uint32_t)cb;
                R.weight_k = wb;
                in_k = w[i];
            }
            cb += c[i];
            wb += w[i];
        }
    }
    __syncthreads();
    if (a.top_p < 1.0) {
        // top-p: its share of what top-k keeps, which is known up to that bucket's weight; the buckets that it may end in
        // (a factor for the roundings of these sums to doubles: more buckets than need be do no harm)
        const uint64_t lo = (uint64_t)(a.top_p * (double)(R.bk >= 0 ? R.weight_k : all_w) * (1.0 - 1e-12));
        const uint64_t hi = (uint64_t)(a.top_p * (double)(R.bk >= 0 ? R.weight_k + in_k : all_w) * (1.0 + 1e-12)) + 1;
        uint64_t wb = w0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            // the first bucket that reaches lo, the last that starts at or before hi (the buckets in between may be empty)
            if (wb + w[i] >= lo && (wb < lo || tid * PER + i == 0)) {
                R.p0 = tid * PER + i;
                R.weight_p = wb;
            }
            if (wb <= hi && (wb + w[i] > hi || tid * PER + i == kFilterBuckets - 1)) R.p1 = tid * PER + i;
            wb += w[i];
        }
    }
    __syncthreads();
}

// One row of 128256 logits 9.7 us.  Each of a row's workgroups adds up to 2048 sums to the row's, the same ones for all: with several rows that is what takes longest, so
// that workgroups beyond one per compute unit take several segments each (eleven rows 17 -> 13.3 us).
__global__ void __launch_bounds__(NT) k_filter_buckets(FilterArgs a) {
    __shared__ BlockLds L;
    __shared__ Histogram H;
    __shared__ FilterRow R;
    const int r = blockIdx.y, tid = threadIdx.x;
    FilterScratch &S = *a.s;
    SegLogits z;
    z.load(a, r, blockIdx.x);
    H.clear(a);
    bool bad;
    const float top = row_top(a, r, &bad);
    __syncthreads();
    for (int seg = blockIdx.x; seg < a.n_seg && !bad; seg += gridDim.x) {
        if (seg != (int)blockIdx.x) z.load(a, r, seg);
        z.each([&](float x, int) { H.add(a, x, top); });
    }
    __syncthreads();
    for (int b = tid; b < kFilterBuckets; b += NT) {
        if (a.top_k && H.count[b]) atomicAdd(&S.count[r][b], H.count[b]);
        if (a.top_p < 1.0 && H.weight[b]) atomicAdd((unsigned long long *)&S.weight[r][b], (unsigned long long)H.weight[b]);
    }
    if (!last_of(S.arrivals[r], gridDim.x, L)) return;
    constexpr int PER = kFilterBuckets / NT;
    uint64_t w[PER];
    uint32_t c[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        w[i] = a.top_p < 1.0 ? seen(&S.weight[r][tid * PER + i]) : 0;
        if ((i & 1) == 0) {                              // (two counts to a load)
            const uint64_t two = a.top_k ? seen((const uint64_t *)&S.count[r][tid * PER + i]) : 0;
            c[i] = (uint32_t)two;
            c[i + 1] = (uint32_t)(two >> 32);
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {                      // zero for the next call
        if (a.top_p < 1.0) leave(&S.weight[r][tid * PER + i], (uint64_t)0);
        if (a.top_k && (i & 1) == 0) leave((uint64_t *)&S.count[r][tid * PER + i], (uint64_t)0);
    }
    find_buckets(a, w, c, R, L);
    if (tid == 0) S.row[r] = R;
}

// ---------------------------------------------------------------------------------------------------
// 3. the rows' outcomes
// ---------------------------------------------------------------------------------------------------
// The ids of a row that lie in some buckets, straight from its logits: where a boundary is looked for if there are more of them than the list has places.
struct Entries {
    const float *z;
    int V, weight_bits;
    float top, scale;
    double inv_t;
    __device__ __forceinline__ int count() const { return V; }
    // logit of id i, if it is one of buckets b0 .. b1
    __device__ __forceinline__ bool get(int i, int b0, int b1, float &x) const {
        x = z[i];
        if (masked(x)) return false;
        const int b = bucket_of(x, top, scale);
        return b >= b0 && b <= b1;
    }
};

struct SelectLds {
    uint64_t m[NT];                                      // measure, or weight, by bin
    uint32_t c[NT];                                      // entries by bin
    uint64_t key[kRank], w[kRank];                       // the entries that are ranked
    int n, bin;
    uint64_t before;
};

// The ids of buckets b0 .. b1 in their order; an id is kept if the measures (1 each, or the weights) of the ones before it add up to less than `limit`.
// Returns the smallest kept key, or one above all of them if none is kept.  Bins of keys narrow it down to kRank entries, which
// are ranked by comparing each with all.
template <bool WEIGHTS>
__device__ uint64_t least_kept(const Entries &E, int b0, int b1, uint64_t limit, SelectLds &S, BlockLds &L) {
    const int tid = threadIdx.x, N = E.count();
    uint64_t lo = ~0ull, hi = 0, cnt = 0;
    for (int i = tid; i < N; i += NT) {
        float x;
        if (!E.get(i, b0, b1, x)) continue;
        const uint64_t k = key_of(x, i);
        lo = k < lo ? k : lo;
        hi = k > hi ? k : hi;
        ++cnt;
    }
    lo = block_extreme<false>(lo, L);
    hi = block_extreme<true>(hi, L);
    uint64_t n = block_sum(cnt, L);
    if (limit == 0 || n == 0) return hi + 1;
    auto measure = [&](float x) { return WEIGHTS ? whole(weight_of(x, E.top, E.inv_t), E.weight_bits) : (uint64_t)1; };
    while (n > kRank) {
        const int shift = 64 - __clzll((long long)((hi - lo) / NT));         // (hi - lo) >> shift < NT
        __syncthreads();
        S.m[tid] = 0;
        S.c[tid] = 0;
        if (tid == 0) S.bin = 0;
        __syncthreads();
        for (int i = tid; i < N; i += NT) {
            float x;
            if (!E.get(i, b0, b1, x)) continue;
            const uint64_t k = key_of(x, i);
            if (k < lo || k > hi) continue;
            const int bin = (int)((hi - k) >> shift);
            atomicAdd(&S.c[bin], 1u);
            atomicAdd((unsigned long long *)&S.m[bin], (unsigned long long)measure(x));
        }
        __syncthreads();
        uint64_t all;
        const uint64_t before = block_scan(S.m[tid], L, &all);
        if (S.c[tid] && before < limit) atomicMax(&S.bin, tid);
        __syncthreads();
        if (tid == S.bin) {
            S.before = before;
            S.n = (int)S.c[tid];
        }
        __syncthreads();
        const int bin = S.bin;
        limit -= S.before;
        n = (uint64_t)S.n;
        const uint64_t new_hi = hi - ((uint64_t)bin << shift), span = ((uint64_t)1 << shift) - 1;
        lo = new_hi - lo > span ? new_hi - span : lo;
        hi = new_hi;
    }
    __syncthreads();
    if (tid == 0) S.n = 0;
    __syncthreads();
    for (int i = tid; i < N; i += NT) {
        float x;
        if (!E.get(i, b0, b1, x)) continue;
        const uint64_t k = key_of(x, i);
        if (k < lo || k > hi) continue;
        const int at = atomicAdd(&S.n, 1);
        S.key[at] = k;
        S.w[at] = measure(x);
    }
    __syncthreads();
    uint64_t least = hi + 1;
    if (tid < S.n) {
        const uint64_t mine = S.key[tid];
        uint64_t before = 0;
        for (int i = 0; i < S.n; ++i) before += S.key[i] > mine ? S.w[i] : 0;
        if (before < limit) least = mine;
    }
    return block_extreme<false>(least, L);
}

__device__ __forceinline__ float logit_of(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ int id_of(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }

// least_kept for the common case, n keys in LDS: the buckets of equal width cut once more into 128 bins, two to a lane of every wavefront, and no more than kRank
// entries in the boundary's bin, which every wavefront ranks for itself: two barriers in all.  False if it is not that case.  *weight: of what is kept (for
// counts; the weights are measured too).
template <bool WEIGHTS>
__device__ __forceinline__ bool least_kept_lds(const FilterArgs &a, const uint64_t *T, int n, int b0, int b1, uint64_t limit, float top, SelectLds &S,
                                               uint64_t *least, uint64_t *weight) {
    constexpr int kBins = 128;
    const int tid = threadIdx.x, lane = tid & 63;
    if (b1 >= kLinear || limit == 0) return false;
    const float fine = (float)kBins / (float)(b1 - b0 + 1);
    auto bin_of = [&](float z) {                         // (monotonic in the logit); negative: of another bucket
        const int in = bucket_of(z, top, a.bucket_scale);
        float x = (top - z) * a.bucket_scale;
        asm("" : "+v"(x));                               // (the same rounding both times)
        const int b = (int)((x - (float)b0) * fine);
        return in < b0 || in > b1 ? -1 : b < 0 ? 0 : b < kBins ? b : kBins - 1;
    };
    auto weight_at = [&](float z) { return whole(weight_of(z, top, a.inv_t), a.weight_bits); };
    __syncthreads();
    if (tid < kBins) {
        S.m[tid] = 0;
        S.c[tid] = 0;
    }
    if (tid == 0) S.n = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
        const float z = logit_of(T[i]);
        const int b = bin_of(z);
        if (b < 0) continue;
        atomicAdd(&S.c[b], 1u);
        atomicAdd((unsigned long long *)&S.m[b], (unsigned long long)weight_at(z));
    }
    __syncthreads();
    // lane l: bins 2 l and 2 l + 1; the last bin with entries before which the measures stay below the limit
    const uint32_t c0 = S.c[2 * lane], c1 = S.c[2 * lane + 1];
    const uint64_t m0 = S.m[2 * lane], m1 = S.m[2 * lane + 1];
    const uint64_t w0 = wave_scan(m0 + m1, lane) - (m0 + m1), w1 = w0 + m0;
    uint64_t at0 = w0, at1 = w1;
    if (!WEIGHTS) {
        at0 = wave_scan((uint64_t)c0 + c1, lane) - ((uint64_t)c0 + c1);
        at1 = at0 + c0;
    }
    const unsigned long long in0 = __ballot(c0 && at0 < limit), in1 = __ballot(c1 && at1 < limit);
    const int l0 = 63 - __clzll(in0), l1 = 63 - __clzll(in1);            // (-1: none)
    if (l0 < 0 && l1 < 0) return false;
    const bool odd = l1 >= l0;
    const int l = odd ? l1 : l0, bin = 2 * l + odd;
    const int nb = __builtin_amdgcn_readlane((int)(odd ? c1 : c0), l);
    const uint64_t before = lane_u64(odd ? at1 : at0, l), before_w = lane_u64(odd ? w1 : w0, l);
    if (nb > kRank) return false;
    for (int i = tid; i < n; i += NT) {
        const float z = logit_of(T[i]);
        if (bin_of(z) != bin) continue;
        const int at = atomicAdd(&S.n, 1);
        S.key[at] = T[i];
        S.w[at] = weight_at(z);
    }
    __syncthreads();
    const uint64_t mine = lane < nb ? S.key[lane] : 0, left = limit - before;
    uint64_t ahead = 0;
    int rank = 0;
    for (int i = 0; i < nb; ++i) {
        const bool greater = S.key[i] > mine;
        rank += greater;
        ahead += greater ? (WEIGHTS ? S.w[i] : 1) : 0;
    }
    const bool kept = lane < nb && ahead < left;
    const int n_kept = __popcll(__ballot(kept));         // one at least: nothing is ahead of the first
    *least = lane_u64(mine, __ffsll(__ballot(lane < nb && rank == n_kept - 1)) - 1);
    *weight = before_w + lane_u64(wave_scan(kept ? S.w[lane] : 0, lane), 63);
    return true;
}

// what the outcome of a row says about an id
struct Kept {
    uint64_t least;
    float top;
    double inv_t;
    __device__ __forceinline__ bool holds(float x, int id) const { return !masked(x) && key_of(x, id) >= least; }
    // weight in 64 bits, 0 if it is not kept
    __device__ __forceinline__ double operator()(float x, int id) const { return holds(x, id) ? weight_of(x, top, inv_t) : 0.0; }
};

// The smallest key that min-p keeps: that of the smallest logit whose weight is at least min_p.  It lies within a step or two of top + min_x; the search goes as far as
// it has to (weights that are all 1 at a temperature beyond the logits' range).
__device__ uint64_t least_by_weight(const FilterArgs &a, float top) {
    if (a.min_p == 0.0) return 0;
    auto kept = [&](uint32_t u) { return weight_of(__uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u), top, a.inv_t) >= a.min_p; };
    const uint32_t first = 0x00800000u, last = (uint32_t)(key_of(top, 0) >> 32);         // of the smallest finite number, of the top (which is kept)
    uint32_t u = (uint32_t)(key_of((float)fmax((double)top + a.min_x, -3.4028234663852886e38), 0) >> 32), no, yes;
    u = u < last ? u : last;
    if (kept(u)) {
        yes = u;
        for (uint32_t s = 1;; s *= 2) {
            if (yes - first <= s) {
                if (kept(first)) return (uint64_t)first << 32;
                no = first;
                break;
            }
            if (!kept(yes - s)) {
                no = yes - s;
                break;
            }
            yes -= s;
        }
    } else {
        no = u;
        for (uint32_t s = 1;; s *= 2) {
            yes = last - no <= s ? last : no + s;
            if (yes == last || kept(yes)) break;
            no = yes;
        }
    }
    while (yes - no > 1) {
        const uint32_t mid = no + (yes - no) / 2;
        if (kept(mid)) yes = mid;
        else no = mid;
    }
    return (uint64_t)yes << 32;                          // whatever the id
}

struct WalkLds { int hit, seg; uint64_t before; double w; };
// The id that a draw falls on, by inversion over the kept ids of row z in id order, thread t having the weight of segment t: in every thread;
// *weight: that id's, *sum: the row's, which is not zero.
__device__ __forceinline__ int draw(const FilterArgs &a, uint64_t mine, float u, const Kept &kept, const float *z, WalkLds &K, BlockLds &L, double *weight,
                                    uint64_t *sum) {
    const int tid = threadIdx.x;
    uint64_t total, ignore;
    const uint64_t before = block_scan(mine, L, &total);
    uint64_t target = (uint64_t)((double)u * (double)total);
    target = target < total ? target : total - 1;
    if (before <= target && target < before + mine) {
        K.seg = tid;
        K.before = before;
    }
    if (tid == 0) K.hit = -1;
    __syncthreads();
    // thread t has consecutive ids of the segment, the logits of the first kKeep of them all on their way at once
    const int seg = K.seg, j0 = seg * a.seg_ids, j1 = min(a.V, j0 + a.seg_ids), per = (a.seg_ids + NT - 1) / NT;
    const int i0 = min(j1, j0 + tid * per), i1 = min(j1, i0 + per);
    float v[kKeep];
    double x[kKeep];
#pragma unroll
    for (int i = 0; i < kKeep; ++i) v[i] = i0 + i < i1 ? z[i0 + i] : -INFINITY;
    uint64_t own = 0;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
        x[i] = kept(v[i], i0 + i);
        own += whole(x[i], a.weight_bits);
    }
    for (int j = i0 + kKeep; j < i1; ++j) own += whole(kept(z[j], j), a.weight_bits);
    const uint64_t at = K.before + block_scan(own, L, &ignore);
    if (at <= target && target < at + own) {
        uint64_t c = at;
        int hit = -1;
        double w_hit = 0.0;
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            c += whole(x[i], a.weight_bits);
            if (hit < 0 && c > target) {
                hit = i0 + i;
                w_hit = x[i];
            }
        }
        for (int j = i0 + kKeep; j < i1 && hit < 0; ++j) {
            w_hit = kept(z[j], j);
            c += whole(w_hit, a.weight_bits);
            if (c > target) hit = j;
        }
        K.hit = hit;
        K.w = w_hit;
    }
    __syncthreads();
    *sum = total;
    if (K.hit < 0) {
        // (the segment's weight was formed of other ids: those next to min_p, if the exponential does not grow from one logit to the next) the row's last kept id
        uint64_t last = 0;
        for (int j = tid; j < a.V; j += NT)
            if (kept.holds(z[j], j)) last = (uint64_t)j + 1;
        const int id = (int)block_extreme<true>(last, L) - 1;
        *weight = id >= 0 ? kept(z[id], id) : 0.0;
        return id;
    }
    *weight = K.w;
    return K.hit;
}

__device__ __forceinline__ void report_draw(const FilterArgs &a, int tok, float prob) {
    report(a.tok_out, tok);
    if (a.prob_out) report(a.prob_out, prob);
    if (a.n_accept_out) report(a.n_accept_out, 0);
    report_done(a.done_flag, a.done_seq);
}

// The smallest key that top-k and top-p keep, R saying which buckets their boundaries lie in.  T: the n keys of those buckets, in LDS (negative: they are not there).
__device__ __forceinline__ uint64_t find_least(const FilterArgs &a, const FilterRow &R, const Entries &E, const uint64_t *T, int n, float top, SelectLds &S, BlockLds &L) {
    uint64_t least = 0, weight = R.weight;
    if (R.bk >= 0) {
        const uint64_t limit = (uint64_t)a.top_k - R.count_k;
        uint64_t in_bucket;
        if (n < 0 || !least_kept_lds<false>(a, T, n, R.bk, R.bk, limit, top, S, &least, &in_bucket)) {
            least = least_kept<false>(E, R.bk, R.bk, limit, S, L);
            in_bucket = 0;
            for (int i = threadIdx.x; i < E.count(); i += NT) {
                float x;
                if (E.get(i, R.bk, R.bk, x) && key_of(x, i) >= least) in_bucket += whole(weight_of(x, top, a.inv_t), a.weight_bits);
            }
            in_bucket = block_sum(in_bucket, L);
        }
        weight = R.weight_k + in_bucket;
    }
    if (R.p0 <= R.p1) {
        // kept: less than top_p * weight before it
        const uint64_t bound = (uint64_t)ceil(a.top_p * (double)weight), limit = bound > R.weight_p ? bound - R.weight_p : 0;
        uint64_t by_p, ignore;
        if (n < 0 || !least_kept_lds<true>(a, T, n, R.p0, R.p1, limit, top, S, &by_p, &ignore)) by_p = least_kept<true>(E, R.p0, R.p1, limit, S, L);
        least = by_p > least ? by_p : least;
    }
    return least;
}

// buckets before `sure` are kept as far as top-k and top-p go, those of the boundaries are listed
struct Classes {
    int sure, p0, p1, bk;
    __device__ __forceinline__ Classes(const FilterRow &R) : sure(R.p0 <= R.p1 ? R.p0 : R.bk >= 0 ? R.bk : kFilterBuckets), p0(R.p0), p1(R.p1), bk(R.bk) {}
    __device__ __forceinline__ bool listed(int b) const { return b == bk || (b >= p0 && b <= p1); }
};

__device__ __forceinline__ void no_distribution(const FilterArgs &a, int r, float top) {
    if (threadIdx.x != 0) return;
    FilterRow &R = a.s->row[r];
    R.bad = 1;
    R.top = top;
    R.least = ~0ull;
    R.total = 0;
    if (a.tok_out) report_draw(a, -1, __uint_as_float(0x7fc00000u));
}

// The row's outcome for the kernels that follow; thread t has the weight of segment t.  Returns the weight of all.
__device__ __forceinline__ uint64_t outcome(const FilterArgs &a, int r, float top, uint64_t least, uint64_t w, BlockLds &L) {
    uint64_t total;
    (void)block_scan(w, L, &total);
    if ((int)threadIdx.x < a.n_seg) a.s->seg_weight[r][threadIdx.x] = w;
    if (threadIdx.x == 0) {
        FilterRow &R = a.s->row[r];
        R.bad = 0;
        R.top = top;
        R.least = least;
        R.total = total;
    }
    return total;
}

__device__ __forceinline__ void draw_and_report(const FilterArgs &a, const Kept &kept, const float *z, uint64_t w, WalkLds &K, BlockLds &L) {
    double x;
    uint64_t total;
    const int tok = draw(a, w, a.u, kept, z, K, L, &x, &total);
    if (threadIdx.x == 0) report_draw(a, tok, (float)(x / ldexp((double)total, -a.weight_bits)));
}

// BOUND: there are boundaries to find (k_filter_buckets has run)
template <bool BOUND>
__global__ void __launch_bounds__(NT) k_filter_row(FilterArgs a) {
    __shared__ BlockLds L;
    __shared__ SelectLds SL;
    __shared__ uint64_t T[kFilterList];
    __shared__ WalkLds K;
    __shared__ uint64_t seg_w[kFilterMaxSegs];
    __shared__ int n_mine;
    const int r = blockIdx.y, tid = threadIdx.x;
    FilterScratch &S = *a.s;
    SegLogits z;
    z.load(a, r, blockIdx.x);
    FilterRow R;
    if constexpr (BOUND) {
        R = S.row[r];
    } else {
        R.p0 = kFilterBuckets;
        R.p1 = R.bk = -1;
    }
    const Classes in(R);
    if (tid == 0) n_mine = 0;
    bool bad;
    const float top = row_top(a, r, &bad);
    if (BOUND) __syncthreads();
    uint64_t mine = 0;
    if (!bad) {
        auto sure = [&](float x) {
            const double w = weight_of(x, top, a.inv_t);
            if (w >= a.min_p) mine += whole(w, a.weight_bits);
        };
        if constexpr (!BOUND) {
            z.each([&](float x, int) {
                if (!masked(x)) sure(x);
            });
        } else {
            // listed ids go to places of the segment's own (no workgroup waits for a number from another); unused places say so, and the
            // first one says it if there are too few
            z.each([&](float x, int j) {
                if (masked(x)) return;
                const int b = bucket_of(x, top, a.bucket_scale);
                if (b < in.sure) sure(x);
                else if (in.listed(b)) {
                    const int at = atomicAdd(&n_mine, 1);
                    if (at < a.places) T[at] = (uint64_t)__float_as_uint(x) << 32 | (uint32_t)j;
                }
            });
            __syncthreads();
            if (tid < a.places)
                leave(&S.list[r][blockIdx.x * a.places + tid], n_mine > a.places ? kTooMany : tid < n_mine ? T[tid] : kUnused);
        }
    }
    mine = block_sum(mine, L);
    if (tid == 0) leave(&S.seg_weight[r][blockIdx.x], mine);
    if (!last_of(S.arrivals[r], a.n_seg, L)) return;

    if (bad) {
        no_distribution(a, r, top);
        return;
    }
    uint64_t w = tid < a.n_seg ? seen(&S.seg_weight[r][tid]) : 0;
    Kept kept{least_by_weight(a, top), top, a.inv_t};
    if constexpr (BOUND) {
        // (every place of the list is on its way before the first is looked at)
        constexpr int PER = kFilterList / NT;
        uint64_t e[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) e[i] = tid + i * NT < a.n_seg * a.places ? seen(&S.list[r][tid + i * NT]) : kUnused;
        if (tid == 0) n_mine = 0;
        __syncthreads();
        bool too_many = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            too_many |= e[i] == kTooMany;
            if (e[i] < kTooMany) T[atomicAdd(&n_mine, 1)] = key_of(__uint_as_float((uint32_t)(e[i] >> 32)), (int)(uint32_t)e[i]);
        }
        too_many = __syncthreads_or(too_many);
        const int n = too_many ? -1 : n_mine;
        const Entries E{z.z, a.V, a.weight_bits, top, a.bucket_scale, a.inv_t};
        const uint64_t least = find_least(a, R, E, T, n, top, SL, L);
        kept.least = least > kept.least ? least : kept.least;
        // the listed ones that are kept join their segments
        seg_w[tid] = w;
        __syncthreads();
        auto join = [&](float x, int id) {
            const uint64_t y = whole(kept(x, id), a.weight_bits);
            if (y) atomicAdd((unsigned long long *)&seg_w[id / a.seg_ids], (unsigned long long)y);
        };
        if (n >= 0) {
            for (int i = tid; i < n; i += NT)
                if (T[i] >= kept.least) join(logit_of(T[i]), id_of(T[i]));
        } else {
            for (int i = tid; i < E.count(); i += NT) {
                float x;
                if (E.get(i, R.p0, R.p1, x) || E.get(i, R.bk, R.bk, x)) join(x, i);
            }
        }
        __syncthreads();
        w = seg_w[tid];
    }
    if (a.tok_out) draw_and_report(a, kept, z.z, w, K, L);
    else (void)outcome(a, r, top, kept.least, w, L);
}

// the distribution of a row of one segment
__device__ __forceinline__ void write_probs(const FilterArgs &a, int r, const SegLogits &z, const Kept &kept, uint64_t total, float *probs) {
    const double inv = 1.0 / ldexp((double)total, -a.weight_bits);
    z.each([&](float x, int j) {
        if (j < a.V) probs[(size_t)r * a.V + j] = (float)(kept(x, j) * inv);
    });
}
__device__ __forceinline__ void write_no_probs(const FilterArgs &a, int r, const SegLogits &z, float *probs) {
    z.each([&](float, int j) {
        if (j < a.V) probs[(size_t)r * a.V + j] = __uint_as_float(0x7fc00000u);
    });
}

// A row of one segment: everything, with what the kernels above leave one another in LDS.  It writes the distribution if that is asked for.
__global__ void __launch_bounds__(NT) k_filter_one(FilterArgs a, float *probs) {
    __shared__ BlockLds L;
    __shared__ SelectLds SL;
    __shared__ union { Histogram H; uint64_t T[kFilterSegIds]; } M;
    __shared__ WalkLds K;
    __shared__ FilterRow R;
    __shared__ int n_listed;
    const int r = blockIdx.x, tid = threadIdx.x;
    SegLogits z;
    z.load(a, r, 0);
    const float top = z.top(L);
    if (!(fabsf(top) < INFINITY)) {
        no_distribution(a, r, top);
        if (probs) write_no_probs(a, r, z, probs);
        return;
    }
    Kept kept{least_by_weight(a, top), top, a.inv_t};
    uint64_t mine = 0;
    if (a.top_k || a.top_p < 1.0) {
        M.H.clear(a);
        if (tid == 0) n_listed = 0;
        __syncthreads();
        z.each([&](float x, int) { M.H.add(a, x, top); });
        __syncthreads();
        constexpr int PER = kFilterBuckets / NT;
        uint64_t w[PER];
        uint32_t c[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            w[i] = a.top_p < 1.0 ? M.H.weight[tid * PER + i] : 0;
            c[i] = a.top_k ? M.H.count[tid * PER + i] : 0;
        }
        find_buckets(a, w, c, R, L);                     // (the histogram's place is free behind its barriers)
        const Classes in(R);
        z.each([&](float x, int j) {
            if (masked(x)) return;
            const int b = bucket_of(x, top, a.bucket_scale);
            if (b < in.sure) {
                const double y = weight_of(x, top, a.inv_t);
                if (y >= a.min_p) mine += whole(y, a.weight_bits);
            } else if (in.listed(b)) {
                M.T[atomicAdd(&n_listed, 1)] = key_of(x, j);
            }
        });
        __syncthreads();
        const int n = n_listed;                          // (a segment's ids: they fit)
        const Entries E{z.z, a.V, a.weight_bits, top, a.bucket_scale, a.inv_t};
        const uint64_t least = find_least(a, R, E, M.T, n, top, SL, L);
        kept.least = least > kept.least ? least : kept.least;
        for (int i = tid; i < n; i += NT)
            if (M.T[i] >= kept.least) mine += whole(kept(logit_of(M.T[i]), id_of(M.T[i])), a.weight_bits);
    } else {
        z.each([&](float x, int) {
            if (masked(x)) return;
            const double y = weight_of(x, top, a.inv_t);
            if (y >= a.min_p) mine += whole(y, a.weight_bits);
        });
    }
    mine = block_sum(mine, L);
    if (a.tok_out) {
        draw_and_report(a, kept, z.z, tid == 0 ? mine : 0, K, L);
        return;
    }
    const uint64_t total = outcome(a, r, top, kept.least, tid == 0 ? mine : 0, L);
    if (probs) write_probs(a, r, z, kept, total, probs);
}

// ---------------------------------------------------------------------------------------------------
// a small top-k
// ---------------------------------------------------------------------------------------------------
// The smallest key of the first k of the entries that `each` goes through (a callable given the logit and id of each entry of this thread), 0 if there are no more than
// k; top: their largest logit.  By buckets, of which the last is ranked; one of more than kRank entries is cut by key until it is short enough.
template <class Each>
__device__ __forceinline__ uint64_t first_k(const FilterArgs &a, Each each, float top, uint32_t k, uint32_t *count, SelectLds &S, BlockLds &L) {
    constexpr int PER = kFilterBuckets / NT;
    const int tid = threadIdx.x, lane = tid & 63;
    __syncthreads();
    for (int b = tid; b < kFilterBuckets; b += NT) count[b] = 0;
    if (tid == 0) S.n = 0;
    __syncthreads();
    each([&](float x, int) {
        if (!masked(x)) atomicAdd(&count[bucket_of(x, top, a.bucket_scale)], 1u);
    });
    __syncthreads();
    uint32_t c[PER];
    uint64_t sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = count[tid * PER + i];
        sum += c[i];
    }
    uint64_t at = block_scan(sum, L, &all);
    if (all <= k) return 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (at < k && at + c[i] >= k) {
            S.bin = tid * PER + i;
            S.before = at;
        }
        at += c[i];
    }
    __syncthreads();
    const int bucket = S.bin;
    uint32_t left = k - (uint32_t)S.before;                  // of the bucket's entries, 1 at least
    uint64_t n = count[bucket], lo = 0, hi = ~0ull;
    auto inside = [&](float x, uint64_t key) { return !masked(x) && bucket_of(x, top, a.bucket_scale) == bucket && key >= lo && key <= hi; };
    if (n > kRank) {
        uint64_t kl = ~0ull, kh = 0;
        each([&](float x, int id) {
            const uint64_t key = key_of(x, id);
            if (!inside(x, key)) return;
            kl = key < kl ? key : kl;
            kh = key > kh ? key : kh;
        });
        lo = block_extreme<false>(kl, L);
        hi = block_extreme<true>(kh, L);
        while (n > kRank) {
            const int shift = 64 - __clzll((long long)((hi - lo) / NT));         // (hi - lo) >> shift < NT
            __syncthreads();
            S.c[tid] = 0;
            __syncthreads();
            each([&](float x, int id) {
                const uint64_t key = key_of(x, id);
                if (inside(x, key)) atomicAdd(&S.c[(hi - key) >> shift], 1u);
            });
            __syncthreads();
            const uint64_t before = block_scan(S.c[tid], L, &all);
            if (before < left && before + S.c[tid] >= left) {
                S.bin = tid;
                S.before = before;
            }
            __syncthreads();
            const uint64_t new_hi = hi - ((uint64_t)S.bin << shift), span = ((uint64_t)1 << shift) - 1;
            left -= (uint32_t)S.before;
            n = S.c[S.bin];
            lo = new_hi - lo > span ? new_hi - span : lo;
            hi = new_hi;
        }
    }
    each([&](float x, int id) {
        const uint64_t key = key_of(x, id);
        if (inside(x, key)) S.key[atomicAdd(&S.n, 1)] = key;
    });
    __syncthreads();
    // every wavefront ranks them for itself
    const uint64_t mine = lane < (int)n ? S.key[lane] : 0;
    uint32_t rank = 0;
    for (int i = 0; i < (int)n; ++i) rank += S.key[i] > mine;
    return lane_u64(mine, __ffsll(__ballot(lane < (int)n && rank == left - 1)) - 1);
}

// Every workgroup lists its segment's first top_k; the row's last one finds the row's among those and takes the other steps and the draw on what is left.
// PER: of the list's places, to a thread; 0: a row of one segment, which is all there (its distribution too, if that is asked for).
template <int PER>
__global__ void __launch_bounds__(NT) k_filter_few(FilterArgs a, float *probs) {
    __shared__ BlockLds L;
    __shared__ SelectLds SL;
    __shared__ uint32_t count[kFilterBuckets];
    __shared__ uint64_t T[NT];
    __shared__ uint64_t key[kFilterFew], weight[kFilterFew];
    __shared__ int n_listed;
    const int r = blockIdx.y, tid = threadIdx.x;
    FilterScratch &S = *a.s;
    SegLogits z;
    z.load(a, r, blockIdx.x);
    const float seg_top = z.top(L);
    if (tid == 0) n_listed = 0;
    if (fabsf(seg_top) < INFINITY) {
        const uint64_t least = first_k(a, [&](auto f) { z.each(f); }, seg_top, (uint32_t)a.top_k, count, SL, L);
        z.each([&](float x, int j) {
            if (!masked(x) && key_of(x, j) >= least) T[atomicAdd(&n_listed, 1)] = (uint64_t)__float_as_uint(x) << 32 | (uint32_t)j;
        });
    }
    __syncthreads();
    float top = seg_top;
    if constexpr (PER == 0) {
        if (!(fabsf(top) < INFINITY)) {
            no_distribution(a, r, top);
            if (probs) write_no_probs(a, r, z, probs);
            return;
        }
        if (tid < n_listed) key[tid] = key_of(__uint_as_float((uint32_t)(T[tid] >> 32)), (int)(uint32_t)T[tid]);
    } else {
        if (tid < a.places) leave(&S.list[r][blockIdx.x * a.places + tid], tid < n_listed ? T[tid] : kUnused);
        if (tid == 0) leave(&S.seg_top[r][blockIdx.x], seg_top);
        if (!last_of(S.arrivals[r], a.n_seg, L)) return;

        // (every place of the list is on its way before the first is looked at)
        uint64_t e[PER > 0 ? PER : 1];
#pragma unroll
        for (int i = 0; i < PER; ++i) e[i] = tid + i * NT < a.n_seg * a.places ? seen(&S.list[r][tid + i * NT]) : kUnused;
        bool bad;
        top = row_top<true>(a, r, &bad);
        if (bad) {
            no_distribution(a, r, top);
            return;
        }
        auto listed = [&](auto f) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (e[i] != kUnused) f(__uint_as_float((uint32_t)(e[i] >> 32)), (int)(uint32_t)e[i]);
        };
        const uint64_t least_k = first_k(a, listed, top, (uint32_t)a.top_k, count, SL, L);
        if (tid == 0) n_listed = 0;
        __syncthreads();
        listed([&](float x, int id) {
            const uint64_t k = key_of(x, id);
            if (k >= least_k) key[atomicAdd(&n_listed, 1)] = k;
        });
    }
    __syncthreads();
    // four threads to an id, each with every fourth of the others (a thread to an id: 128 ids take 1 us more)
    static_assert(4 * kFilterFew <= NT, "a thread for each quarter");
    const int n = n_listed, id = tid >> 2, quarter = tid & 3;                    // n: top_k, or fewer
    const uint64_t mine = id < n ? key[id] : 0;
    const double w = id < n ? weight_of(logit_of(mine), top, a.inv_t) : 0.0;
    if (id < n && quarter == 0) weight[id] = whole(w, a.weight_bits);
    T[tid] = 0;
    __syncthreads();
    auto of_four = [](uint64_t v) {
        v += dpp_u64<0xB1>(v);
        return v + dpp_u64<0x4E>(v);
    };
    // kept: less than top_p of the weight of all before it, and at least min_p of the largest
    bool keep = id < n && w >= a.min_p;
    if (a.top_p < 1.0) {
        uint64_t before = 0, all = 0;
        for (int i = quarter; i < n; i += 4) {
            before += key[i] > mine ? weight[i] : 0;
            all += weight[i];
        }
        before = of_four(before);
        all = of_four(all);
        keep = keep && before < (uint64_t)ceil(a.top_p * (double)all);
    }
    __syncthreads();
    if (id < n && !keep && quarter == 0) weight[id] = 0;
    if (!a.tok_out) {
        if (keep && quarter == 0) atomicAdd((unsigned long long *)&T[id_of(mine) / a.seg_ids], (unsigned long long)weight[id]);
        const uint64_t least = block_extreme<false>(keep ? mine : ~0ull, L);     // (its barriers: the segments' weights are complete)
        const uint64_t total = outcome(a, r, top, least, T[tid], L);
        if (PER == 0 && probs) write_probs(a, r, z, Kept{least, top, a.inv_t}, total, probs);
        return;
    }
    __syncthreads();
    uint64_t total = 0, ahead = 0;
    for (int i = quarter; i < n; i += 4) {
        total += weight[i];
        ahead += id_of(key[i]) < id_of(mine) ? weight[i] : 0;
    }
    total = of_four(total);
    ahead = of_four(ahead);
    uint64_t target = (uint64_t)((double)a.u * (double)total);
    target = target < total ? target : total - 1;
    if (id < n && quarter == 0 && ahead <= target && target < ahead + weight[id]) report_draw(a, id_of(mine), (float)(w / ldexp((double)total, -a.weight_bits)));
}

// ---------------------------------------------------------------------------------------------------
// the distributions
// ---------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(NT) k_filter_probs(FilterArgs a, float *probs) {
    const int r = blockIdx.y;
    SegLogits z;
    z.load(a, r, blockIdx.x);
    float *p = probs + (size_t)r * a.V;
    const FilterRow &R = a.s->row[r];
    const Kept kept{R.least, R.top, a.inv_t};
    const double inv = 1.0 / ldexp((double)R.total, -a.weight_bits);
    const bool bad = R.bad;
    z.each([&](float x, int j) {
        if (j < z.j1) p[j] = bad ? __uint_as_float(0x7fc00000u) : (float)(kept(x, j) * inv);
    });
}

// ---------------------------------------------------------------------------------------------------
// accept / resample between filtered distributions
// ---------------------------------------------------------------------------------------------------
struct Side { Kept kept; double log_total, inv_total; bool bad; };
__device__ __forceinline__ Side side_of(const FilterArgs &a, int r) {
    const FilterRow &R = a.s->row[r];
    const double total = ldexp((double)R.total, -a.weight_bits);
    return Side{Kept{R.least, R.top, a.inv_t}, log(total), 1.0 / total, R.bad != 0};
}

// max(0, p(j) - q(j)), from the logarithms: where the two nearly agree, or all that is left is far below the smallest fp32 number, their
// difference keeps its precision
struct Residual {
    Side p, q;
    const float *zp, *zq;
    // its logarithm; minus infinity where p does not exceed q
    __device__ __forceinline__ double operator()(int j) const {
        if (!p.kept.holds(zp[j], j)) return -INFINITY;
        const double a = ((double)zp[j] - (double)p.kept.top) * p.kept.inv_t - p.log_total;
        if (!q.kept.holds(zq[j], j)) return a;
        const double d = ((double)zq[j] - (double)q.kept.top) * q.kept.inv_t - q.log_total - a;
        return d < 0.0 ? a + log(-expm1(d)) : -INFINITY;
    }
};

// A segment of the residual per workgroup, the last one draws.  12.7 us for 6 rows of 128256 logits if a draft is rejected, 6 if none is.  The residual takes two
// exponentials and a logarithm in 64 bits an id: only the ids that p keeps, gathered first, come that far (all of a wavefront's turns waited for one such id before: 15.2).
__global__ void __launch_bounds__(NT) k_filter_verify(FilterVerifyArgs v) {
    __shared__ BlockLds L;
    __shared__ WalkLds K;
    __shared__ double ratio_of[8], top_of[NW];
    __shared__ int ids[kFilterSegIds], n_kept;
    const FilterArgs &a = v.f;
    FilterScratch &S = *a.s;
    const int tid = threadIdx.x, n_draft = v.m - 1;
    // Eq. 2 over the drafts, by every workgroup
    if (tid < n_draft) {
        const int t = v.draft[tid];
        const Side p = side_of(a, tid), q = side_of(a, v.m + tid);
        const float zp = row_of(a, tid)[t], zq = row_of(a, v.m + tid)[t];
        const double wp = p.bad ? 0.0 : p.kept(zp, t), wq = q.bad ? 0.0 : q.kept(zq, t);
        double ratio = wp == 0.0 ? 0.0 : wq == 0.0 ? INFINITY : (wp * p.inv_total) / (wq * q.inv_total);
        if (p.bad || q.bad) ratio = (double)__uint_as_float(0x7fc00000u);
        ratio_of[tid] = ratio;
    }
    __syncthreads();
    int r = 0;
    while (r < n_draft && (double)v.u_accept[r] < fmin(1.0, ratio_of[r]) && ratio_of[r] == ratio_of[r]) ++r;
    const bool rejected = r < n_draft;
    const Side p = side_of(a, r);
    const float *zp = row_of(a, r);
    int tok = -1;
    double x, total_c = -INFINITY;
    uint64_t total;
    const bool bad = p.bad || (rejected && side_of(a, v.m + r).bad);
    if (rejected && !bad) {
        // this workgroup's segment of the residual: its largest weight, and the weights relative to that
        const Residual res{p, side_of(a, v.m + r), zp, row_of(a, v.m + r)};
        const int j0 = blockIdx.x * a.seg_ids, j1 = min(a.V, j0 + a.seg_ids);
        auto block_max = [&](double c) {
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) c = fmax(c, __shfl_xor(c, d));
            __syncthreads();
            if ((tid & 63) == 0) top_of[tid >> 6] = c;
            __syncthreads();
            for (int w = 0; w < NW; ++w) c = fmax(c, top_of[w]);
            return c;
        };
        // the ids that p keeps, one after the other: few, and the arithmetic behind them is long (segments beyond the usual length: as they come)
        const bool usual = a.seg_ids <= kFilterSegIds;
        float z[kKeep];
        if (usual)
#pragma unroll
            for (int i = 0; i < kKeep; ++i) z[i] = j0 + tid + i * NT < j1 ? zp[j0 + tid + i * NT] : -INFINITY;
        if (tid == 0) n_kept = 0;
        __syncthreads();
        if (usual)
#pragma unroll
            for (int i = 0; i < kKeep; ++i)
                if (p.kept.holds(z[i], j0 + tid + i * NT)) ids[atomicAdd(&n_kept, 1)] = j0 + tid + i * NT;
        __syncthreads();
        const double first = usual && tid < n_kept ? res(ids[tid]) : -INFINITY;
        double c = first;
        auto others = [&](auto f) {
            if (usual)
                for (int i = tid + NT; i < n_kept; i += NT) f(ids[i]);
            else
                for (int j = j0 + tid; j < j1; j += NT) f(j);
        };
        others([&](int j) { c = fmax(c, res(j)); });
        c = block_max(c);
        uint64_t sum = 0;
        if (c > -INFINITY) {
            sum = whole(exp(first - c), a.weight_bits);
            others([&](int j) { sum += whole(exp(res(j) - c), a.weight_bits); });
        }
        sum = block_sum(sum, L);
        if (tid == 0) {
            leave(&S.res[2 * blockIdx.x], __builtin_bit_cast(uint64_t, c));
            leave(&S.res[2 * blockIdx.x + 1], sum);
        }
        if (!last_of(S.arrivals[kFilterRows], a.n_seg, L)) return;
        const double sc = tid < a.n_seg ? __builtin_bit_cast(double, seen(&S.res[2 * tid])) : -INFINITY;
        const uint64_t sw = tid < a.n_seg ? seen(&S.res[2 * tid + 1]) : 0;
        total_c = block_max(sc);
        if (total_c > -INFINITY) {
            // the segments' weights relative to the row's largest
            const uint64_t mine = sc > -INFINITY ? (uint64_t)((double)sw * exp(sc - total_c)) : 0;
            uint64_t before, all, ignore;
            before = block_scan(mine, L, &all);
            uint64_t target = (uint64_t)((double)v.u_resample[r] * (double)all);
            target = target < all ? target : all - 1;
            if (before <= target && target < before + mine) {
                K.seg = tid;
                K.before = before;
            }
            if (tid == 0) K.hit = -1;
            __syncthreads();
            // its ids: rounded one by one their weights may add up to a little less than the segment's, whose last id of some weight then stands in.
            // Those that p keeps first, in their order, so that a thread has one (or a few) of them
            const int s0 = K.seg * a.seg_ids, s1 = min(a.V, s0 + a.seg_ids), per = (a.seg_ids + NT - 1) / NT;
            const int i0 = min(s1, s0 + tid * per), i1 = min(s1, i0 + per);
            int e0 = i0, e1 = i1;
            if (usual) {
                // (per <= kKeep: their logits all on their way at once)
                unsigned held = 0;
#pragma unroll
                for (int i = 0; i < kKeep; ++i) z[i] = i0 + i < i1 ? zp[i0 + i] : -INFINITY;
#pragma unroll
                for (int i = 0; i < kKeep; ++i) held |= p.kept.holds(z[i], i0 + i) ? 1u << i : 0;
                uint64_t all_held;
                int at = (int)block_scan(__popc(held), L, &all_held);
                for (int i = 0; i < i1 - i0; ++i)
                    if (held >> i & 1) ids[at++] = i0 + i;
                __syncthreads();
                const int n = (int)all_held, each = (n + NT - 1) / NT;
                e0 = min(n, tid * each);
                e1 = min(n, e0 + each);
            }
            auto id = [&](int e) { return usual ? ids[e] : e; };
            const double w_first = e0 < e1 ? exp(res(id(e0)) - total_c) : 0.0;
            uint64_t own = 0;
            int last = -1;
            for (int e = e0; e < e1; ++e) {
                const double y = e == e0 ? w_first : exp(res(id(e)) - total_c);
                own += whole(y, a.weight_bits);
                if (y > 0.0) last = id(e);
            }
            const uint64_t at = K.before + block_scan(own, L, &ignore);
            int hit = -1;
            if (at <= target && target < at + own) {
                uint64_t s = at;
                for (int e = e0; e < e1 && hit < 0; ++e) {
                    s += whole(e == e0 ? w_first : exp(res(id(e)) - total_c), a.weight_bits);
                    if (s > target) hit = id(e);
                }
            }
            const int found = (int)block_extreme<true>((uint64_t)(hit + 1), L) - 1;
            const int latest = (int)block_extreme<true>((uint64_t)(last + 1), L) - 1;
            tok = found >= 0 ? found : latest;
        }
    } else {
        __syncthreads();
        if (!last_of(S.arrivals[kFilterRows], a.n_seg, L)) return;
    }
    if (tok < 0 && !bad) {   // nothing rejected, or a residual that is identically zero: the row's own distribution
        const uint64_t w = tid < a.n_seg ? S.seg_weight[r][tid] : 0;
        tok = draw(a, w, rejected ? v.u_resample[r] : v.u_final, p.kept, zp, K, L, &x, &total);
    }
    if (tid < 64) {
        if (v.ratio_out && tid < n_draft) report(v.ratio_out + tid, tid <= r ? (float)ratio_of[tid] : 0.f);
        if (tid == 0) {
            report(v.n_accept_out, r);
            report(v.next_out, tok);
            report_done(a.done_flag, a.done_seq);
        }
    }
}

// probs: null, or where rows of one segment are written (others: k_filter_probs)
int launch_rows(const FilterArgs &a, const LaunchCtx &c, float *probs = nullptr) {
    if (a.V < 1 || a.rows < 1 || a.rows > kFilterRows || a.n_seg > kFilterMaxSegs || !(a.inv_t > 0.0)) return (int)hipErrorInvalidValue;
    const dim3 grid(a.n_seg, a.rows), wg(NT);
    // (the distribution of 2048 logits by the largest 50 and top-p: 7.7 us, in k_filter_one 11.3)
    if (a.n_seg == 1 && a.top_k && a.top_k <= kFilterFew) return launch<k_filter_few<0>>(c, grid, wg, 0, a, probs);
    if (a.n_seg == 1) return launch<k_filter_one>(c, dim3(a.rows), wg, 0, a, probs);
    // A small top-k takes one kernel and not three: a draw from 32016 logits by the largest 128 of them takes 13.6 us where one by the largest 129 takes 22.7,
    // 8 rows' distributions of 128256 by the largest 50 take 17.6 and by 129 31.5.  The list of fewer places has a shorter program (top-k 50 of
    // 128256: 12.7 us, and 14.1 with 16 places to a thread); kept in LDS, it leaves a compute unit room for one workgroup (8 rows 27.6).
    if (a.top_k && a.top_k <= kFilterFew && a.top_k * a.n_seg <= kFilterFewList) {
        FilterArgs few = a;
        few.places = a.top_k;
        constexpr int PER = kFilterFewList / NT;
        return a.top_k * a.n_seg <= kFilterFewList / 2 ? launch<k_filter_few<PER / 2>>(c, grid, wg, 0, few, (float *)nullptr) : launch<k_filter_few<PER>>(c, grid, wg, 0, few, (float *)nullptr);
    }
    int rc = launch<k_filter_top>(c, grid, wg, 0, a);
    if (rc) return rc;
    if (a.top_k || a.top_p < 1.0) {
        // (at least one workgroup a row)
        const int most = c.n_wg / a.rows > 1 ? c.n_wg / a.rows : 1;
        if ((rc = launch<k_filter_buckets>(c, dim3(a.n_seg < most ? a.n_seg : most, a.rows), wg, 0, a))) return rc;
        return launch<k_filter_row<true>>(c, grid, wg, 0, a);
    }
    return launch<k_filter_row<false>>(c, grid, wg, 0, a);
}

}  // namespace

void filter_finish(FilterArgs &a, float temperature, int top_k, float top_p, float min_p) {
    const int n = (a.V + kFilterSegIds - 1) / kFilterSegIds, most = n < kFilterMaxSegs ? n : kFilterMaxSegs;
    a.seg_ids = (a.V + most - 1) / most;
    a.n_seg = (a.V + a.seg_ids - 1) / a.seg_ids;
    a.places = kFilterList / a.n_seg < 64 ? kFilterList / a.n_seg : 64;
    a.inv_t = 1.0 / (double)temperature;
    a.bucket_scale = 64.0 * a.inv_t < 3e38 ? (float)(64.0 * a.inv_t) : 3e38f;
    a.top_k = top_k < a.V ? top_k : 0;
    a.top_p = top_p > 0.f && top_p < 1.f ? (double)top_p : 1.0;
    a.min_p = (double)min_p;
    a.min_x = min_p > 0.f ? (double)temperature * log((double)min_p) : 0.0;
    a.weight_bits = 62;                                  // V weights of up to 2^weight_bits add up to less than 2^63
    for (int v = a.V; v > 0; v >>= 1) --a.weight_bits;
}

int launch_filter_sample(const FilterArgs &a, const LaunchCtx &c) {
    if (a.rows != 1 || !a.tok_out) return (int)hipErrorInvalidValue;
    return launch_rows(a, c);
}

int launch_filter_probs(const FilterArgs &a, float *probs, const LaunchCtx &c) {
    if (a.tok_out) return (int)hipErrorInvalidValue;
    const int rc = launch_rows(a, c, probs);
    return rc || a.n_seg == 1 ? rc : launch<k_filter_probs>(c, dim3(a.n_seg, a.rows), dim3(NT), 0, a, probs);
}

int launch_filter_verify(const FilterVerifyArgs &v, const LaunchCtx &c) {
    if (v.m < 1 || v.m > 8) return (int)hipErrorInvalidValue;
    if (v.m == 1) {                                      // no drafts: a draw from the row
        FilterArgs a = v.f;
        a.u = v.u_final; a.tok_out = v.next_out; a.prob_out = nullptr; a.n_accept_out = v.n_accept_out;
        return launch_filter_sample(a, c);
    }
    if (v.f.tok_out || v.f.rows != 2 * v.m - 1 || v.f.n_first != v.m) return (int)hipErrorInvalidValue;
    for (int k = 0; k + 1 < v.m; ++k)
        if (v.draft[k] < 0 || v.draft[k] >= v.f.V) return (int)hipErrorInvalidValue;
    const int rc = launch_rows(v.f, c);
    return rc ? rc : launch<k_filter_verify>(c, dim3(v.f.n_seg), dim3(NT), 0, v);
}

}  // namespace ad
