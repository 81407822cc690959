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
//   k_filter_probs, k_filter_verify: from the rows' outcomes
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
constexpr int kRank = NT;                                // entries that are ranked against each other

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
    constexpr int kLinear = 1792;
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
    uint64_t u[NW];
    uint64_t total;
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
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, int lane) {     // inclusive
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_up((unsigned long long)v, d);
        if (lane >= d) v += o;
    }
    return v;
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
__device__ __forceinline__ uint32_t seen(const uint32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <class T>
__device__ __forceinline__ void leave(T *p, T v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// the last workgroup of n on this counter, when everything that any wavefront of any of them has left is in memory
__device__ __forceinline__ bool last_of(uint32_t *counter, int n, BlockLds &L) {
    reported();
    __syncthreads();
    return last_to_arrive(counter, n, &L.last_wg);
}

// ---------------------------------------------------------------------------------------------------
// 1. largest logits
// ---------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(NT) k_filter_top(FilterArgs a) {
    __shared__ BlockLds L;
    const int r = blockIdx.y, j0 = blockIdx.x * a.seg_ids, j1 = min(a.V, j0 + a.seg_ids);
    const float *z = row_of(a, r);
    float m = -INFINITY;
    bool nan = false;
    for (int j = j0 + (int)threadIdx.x; j < j1; j += NT) {
        const float x = z[j];
        nan |= x != x;
        m = fmaxf(m, x);
    }
    m = block_top(nan ? __uint_as_float(0x7fc00000u) : m, L);
    if (threadIdx.x == 0) a.s->seg_top[r][blockIdx.x] = m;
}

// of the row, to every thread; *bad: it has no distribution
__device__ __forceinline__ float row_top(const FilterArgs &a, int r, BlockLds &L, bool *bad) {
    const float m = block_top((int)threadIdx.x < a.n_seg ? a.s->seg_top[r][threadIdx.x] : -INFINITY, L);
    *bad = !(fabsf(m) < INFINITY);
    return m;
}

// ---------------------------------------------------------------------------------------------------
// 2. buckets
// ---------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(NT) k_filter_buckets(FilterArgs a) {
    __shared__ BlockLds L;
    __shared__ uint64_t hw[kFilterBuckets];
    __shared__ uint32_t hc[kFilterBuckets];
    const int r = blockIdx.y, tid = threadIdx.x, j0 = blockIdx.x * a.seg_ids, j1 = min(a.V, j0 + a.seg_ids);
    const float *z = row_of(a, r);
    FilterScratch &S = *a.s;
    bool bad;
    const float top = row_top(a, r, L, &bad);
    for (int b = tid; b < kFilterBuckets; b += NT) {
        hw[b] = 0;
        hc[b] = 0;
    }
    __syncthreads();
    if (!bad) {
        for (int j = j0 + tid; j < j1; j += NT) {
            const float x = z[j];
            if (masked(x)) continue;
            const int b = bucket_of(x, top, a.bucket_scale);
            atomicAdd(&hc[b], 1u);
            atomicAdd((unsigned long long *)&hw[b], (unsigned long long)whole(weight_of(x, top, a.inv_t), a.weight_bits));
        }
    }
    __syncthreads();
    for (int b = tid; b < kFilterBuckets; b += NT)
        if (hc[b]) {
            atomicAdd(&S.count[r][b], hc[b]);
            atomicAdd((unsigned long long *)&S.weight[r][b], (unsigned long long)hw[b]);
        }
    if (!last_of(S.arrivals[r], a.n_seg, L)) return;

    // the last workgroup: thread t has buckets 4 t .. 4 t + 3
    constexpr int PER = kFilterBuckets / NT;
    uint64_t w[PER], c[PER], ws = 0, cs = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        w[i] = seen(&S.weight[r][tid * PER + i]);
        c[i] = seen(&S.count[r][tid * PER + i]);
        ws += w[i];
        cs += c[i];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {                      // zero for the next call
        leave(&S.weight[r][tid * PER + i], (uint64_t)0);
        leave(&S.count[r][tid * PER + i], 0u);
    }
    uint64_t all_w, all_c;
    const uint64_t w0 = block_scan(ws, L, &all_w), c0 = block_scan(cs, L, &all_c);
    __shared__ FilterRow R;
    if (tid == 0) {
        R.p0 = kFilterBuckets;
        R.p1 = -1;
        R.bk = -1;
        R.count_k = 0;
        R.weight_p = R.weight_k = 0;
        R.weight = all_w;
    }
    __syncthreads();
    // top-k: the bucket of the last id it keeps (none if it keeps them all)
    uint64_t cb = c0, wb = w0;
    __shared__ uint64_t in_k;
    if (tid == 0) in_k = 0;
    __syncthreads();
    if (a.top_k && (uint64_t)a.top_k < all_c) {
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
    // top-p: its share of what top-k keeps, which is known up to that bucket's weight; the buckets that it may end in
    if (a.top_p < 1.0) {
        const double lo = a.top_p * (double)(R.bk >= 0 ? R.weight_k : all_w), hi = a.top_p * (double)(R.bk >= 0 ? R.weight_k + in_k : all_w);
        wb = w0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            // (a factor for the roundings of these sums to doubles: more buckets than need be do no harm)
            const bool before = (double)(wb + w[i]) < lo * (1.0 - 1e-12), behind = (double)wb > hi * (1.0 + 1e-12);
            if (c[i] && !before && !behind) {
                atomicMin(&R.p0, tid * PER + i);
                atomicMax(&R.p1, tid * PER + i);
            }
            wb += w[i];
        }
        __syncthreads();
        wb = w0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (R.p0 == tid * PER + i) R.weight_p = wb;
            wb += w[i];
        }
    }
    __syncthreads();
    if (tid == 0) S.row[r] = R;
}

// ---------------------------------------------------------------------------------------------------
// 3. the rows' outcomes
// ---------------------------------------------------------------------------------------------------
// The entries that a boundary is looked for among: the row's list or, if more ids lie in those buckets than it holds, the row itself.
struct Entries {
    const float *z;
    const uint64_t *list;
    int n;                                               // length of the list; < 0: the row
    int V, weight_bits;
    float top, scale;
    double inv_t;
    __device__ __forceinline__ int count() const { return n >= 0 ? n : V; }
    // the i-th, if it is one of buckets b0 .. b1
    __device__ __forceinline__ bool get(int i, int b0, int b1, float &x, int &id) const {
        if (n >= 0) {
            const uint64_t e = seen(list + i);
            x = __uint_as_float((uint32_t)(e >> 32));
            id = (int)(uint32_t)e;
        } else {
            x = z[i];
            id = i;
            if (masked(x)) return false;
        }
        const int b = bucket_of(x, top, scale);
        return b >= b0 && b <= b1;
    }
};

struct SelectLds {
    uint64_t m[NT];                                      // measure by bin; then of the entries that are ranked
    uint64_t key[kRank];
    uint32_t c[NT];
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
        int id;
        if (!E.get(i, b0, b1, x, id)) continue;
        const uint64_t k = key_of(x, id);
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
            int id;
            if (!E.get(i, b0, b1, x, id)) continue;
            const uint64_t k = key_of(x, id);
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
        int id;
        if (!E.get(i, b0, b1, x, id)) continue;
        const uint64_t k = key_of(x, id);
        if (k < lo || k > hi) continue;
        const int at = atomicAdd(&S.n, 1);
        S.key[at] = k;
        S.m[at] = measure(x);
    }
    __syncthreads();
    uint64_t least = hi + 1;
    if (tid < S.n) {
        const uint64_t mine = S.key[tid];
        uint64_t before = 0;
        for (int i = 0; i < S.n; ++i) before += S.key[i] > mine ? S.m[i] : 0;
        if (before < limit) least = mine;
    }
    return block_extreme<false>(least, L);
}

// what the outcome of a row says about an id
struct Kept {
    uint64_t least;
    float top;
    double inv_t, min_p;
    // weight in 64 bits, 0 if it is not kept
    __device__ __forceinline__ double operator()(float x, int id) const {
        if (masked(x) || key_of(x, id) < least) return 0.0;
        const double w = weight_of(x, top, inv_t);
        return w >= min_p ? w : 0.0;
    }
};

struct WalkLds { int hit, seg; uint64_t before; double w; };
// The id that a draw falls on, by inversion over weights w(j) >= 0 in id order, in segments whose weights (multiples of 2^-bits, as w's) thread t holds of segment t:
// in every thread; *weight: w of it.  The total is not zero.
template <class W>
__device__ int draw(const FilterArgs &a, uint64_t mine, float u, W w, WalkLds &K, BlockLds &L, double *weight, uint64_t *sum) {
    const int tid = threadIdx.x;
    uint64_t total, ignore;
    const uint64_t before = block_scan(mine, L, &total);
    uint64_t target = (uint64_t)((double)u * (double)total);
    target = target < total ? target : total - 1;
    if (before <= target && target < before + mine) {
        K.seg = tid;
        K.before = before;
    }
    if (tid == 0) K.hit = 0x7fffffff;
    __syncthreads();
    const int seg = K.seg, j0 = seg * a.seg_ids, j1 = min(a.V, j0 + a.seg_ids), per = (a.seg_ids + NT - 1) / NT;
    const int i0 = min(j1, j0 + tid * per), i1 = min(j1, i0 + per);
    uint64_t own = 0;
    for (int j = i0; j < i1; ++j) own += whole(w(j), a.weight_bits);
    const uint64_t at = K.before + block_scan(own, L, &ignore);
    if (at <= target && target < at + own) {
        uint64_t c = at;
        for (int j = i0; j < i1; ++j) {
            const double x = w(j);
            c += whole(x, a.weight_bits);
            if (c > target) {
                K.hit = j;
                K.w = x;
                break;
            }
        }
    }
    __syncthreads();
    *weight = K.w;
    *sum = total;
    return K.hit;
}

__device__ __forceinline__ void report_draw(const FilterArgs &a, int tok, float prob) {
    report(a.tok_out, tok);
    if (a.prob_out) report(a.prob_out, prob);
    if (a.n_accept_out) report(a.n_accept_out, 0);
    report_done(a.done_flag, a.done_seq);
}

// BOUND: there are boundaries to find (k_filter_buckets has run)
template <bool BOUND>
__global__ void __launch_bounds__(NT) k_filter_row(FilterArgs a) {
    __shared__ BlockLds L;
    __shared__ SelectLds SL;
    __shared__ WalkLds K;
    __shared__ uint64_t seg_w[kFilterMaxSegs];
    __shared__ int n_mine, at_mine;
    const int r = blockIdx.y, tid = threadIdx.x, j0 = blockIdx.x * a.seg_ids, j1 = min(a.V, j0 + a.seg_ids);
    const float *z = row_of(a, r);
    FilterScratch &S = *a.s;
    bool bad;
    const float top = row_top(a, r, L, &bad);
    FilterRow R;
    if constexpr (BOUND) {
        R = S.row[r];
    } else {
        R.p0 = kFilterBuckets;
        R.p1 = R.bk = -1;
    }
    // buckets before `sure` are kept, those of the boundaries are listed
    const int sure = R.p0 <= R.p1 ? R.p0 : R.bk >= 0 ? R.bk : kFilterBuckets;
    uint64_t mine = 0;
    if (!bad) {
        for (int base = j0; base < j1; base += NT) {
            const int j = base + tid;
            const float x = j < j1 ? z[j] : -INFINITY;
            bool listed = false;
            if (!masked(x)) {
                const int b = BOUND ? bucket_of(x, top, a.bucket_scale) : 0;
                if (b < sure) {
                    const double w = weight_of(x, top, a.inv_t);
                    if (w >= a.min_p) mine += whole(w, a.weight_bits);
                } else {
                    listed = b == R.bk || (b >= R.p0 && b <= R.p1);
                }
            }
            if constexpr (BOUND) {
                if (tid == 0) n_mine = 0;
                __syncthreads();
                int at = 0;
                if (listed) at = atomicAdd(&n_mine, 1);
                __syncthreads();
                if (tid == 0 && n_mine) at_mine = (int)atomicAdd(&S.list_n[r][0], (uint32_t)n_mine);
                __syncthreads();
                if (listed && at_mine + at < kFilterList) leave(&S.list[r][at_mine + at], (uint64_t)__float_as_uint(x) << 32 | (uint32_t)j);
            }
        }
    }
    mine = block_sum(mine, L);
    if (tid == 0) leave(&S.seg_weight[r][blockIdx.x], mine);
    if (!last_of(S.arrivals[r], a.n_seg, L)) return;

    if (bad) {
        if (tid == 0) {
            S.row[r].bad = 1;
            S.row[r].top = top;
            S.row[r].least = ~0ull;
            S.row[r].total = 0;
            if (a.tok_out) report_draw(a, -1, __uint_as_float(0x7fc00000u));
        }
        return;
    }
    uint64_t w = tid < a.n_seg ? seen(&S.seg_weight[r][tid]) : 0, least = 0;
    Kept kept{0, top, a.inv_t, a.min_p};
    if constexpr (BOUND) {
        const uint32_t n = seen(&S.list_n[r][0]);
        const Entries E{z, S.list[r], n <= kFilterList ? (int)n : -1, a.V, a.weight_bits, top, a.bucket_scale, a.inv_t};
        uint64_t weight = R.weight;
        if (R.bk >= 0) {
            least = least_kept<false>(E, R.bk, R.bk, (uint64_t)a.top_k - R.count_k, SL, L);
            weight = 0;
            for (int i = tid; i < E.count(); i += NT) {
                float x;
                int id;
                if (E.get(i, R.bk, R.bk, x, id) && key_of(x, id) >= least) weight += whole(weight_of(x, top, a.inv_t), a.weight_bits);
            }
            weight = R.weight_k + block_sum(weight, L);
        }
        if (R.p0 <= R.p1) {
            // kept: less than top_p * weight before it
            const uint64_t bound = (uint64_t)ceil(a.top_p * (double)weight);
            const uint64_t by_p = least_kept<true>(E, R.p0, R.p1, bound > R.weight_p ? bound - R.weight_p : 0, SL, L);
            least = by_p > least ? by_p : least;
        }
        kept.least = least;
        // the listed ones that are kept join their segments
        __syncthreads();
        seg_w[tid] = w;
        __syncthreads();
        auto join = [&](float x, int id) {
            const uint64_t y = whole(kept(x, id), a.weight_bits);
            if (y) atomicAdd((unsigned long long *)&seg_w[id / a.seg_ids], (unsigned long long)y);
        };
        for (int i = tid; i < E.count(); i += NT) {
            float x;
            int id;
            const bool in_p = E.get(i, R.p0, R.p1, x, id);
            if (in_p || E.get(i, R.bk, R.bk, x, id)) join(x, id);
        }
        __syncthreads();
        w = seg_w[tid];
        if (tid == 0) leave(&S.list_n[r][0], 0u);
    }
    if (a.tok_out) {
        double x;
        uint64_t total;
        const int tok = draw(a, w, a.u, [&](int j) { return kept(z[j], j); }, K, L, &x, &total);
        if (tid == 0) report_draw(a, tok, (float)(x / ldexp((double)total, -a.weight_bits)));
        return;
    }
    uint64_t total;
    (void)block_scan(w, L, &total);
    if (tid < a.n_seg) S.seg_weight[r][tid] = w;
    if (tid == 0) {
        S.row[r].bad = 0;
        S.row[r].top = top;
        S.row[r].least = least;
        S.row[r].total = total;
    }
}

// ---------------------------------------------------------------------------------------------------
// the distributions
// ---------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(NT) k_filter_probs(FilterArgs a, float *probs) {
    const int r = blockIdx.y, j0 = blockIdx.x * a.seg_ids, j1 = min(a.V, j0 + a.seg_ids);
    const float *z = row_of(a, r);
    float *p = probs + (size_t)r * a.V;
    const FilterRow &R = a.s->row[r];
    const Kept kept{R.least, R.top, a.inv_t, a.min_p};
    const double inv = 1.0 / ldexp((double)R.total, -a.weight_bits);
    const bool bad = R.bad;
    for (int j = j0 + (int)threadIdx.x; j < j1; j += NT) p[j] = bad ? __uint_as_float(0x7fc00000u) : (float)(kept(z[j], j) * inv);
}

// ---------------------------------------------------------------------------------------------------
// accept / resample between filtered distributions
// ---------------------------------------------------------------------------------------------------
struct Side { Kept kept; double log_total, inv_total; bool bad; };
__device__ __forceinline__ Side side_of(const FilterArgs &a, int r) {
    const FilterRow &R = a.s->row[r];
    const double total = ldexp((double)R.total, -a.weight_bits);
    return Side{Kept{R.least, R.top, a.inv_t, a.min_p}, log(total), 1.0 / total, R.bad != 0};
}

// max(0, p(j) - q(j)), from the logarithms: where the two nearly agree, or all that is left is far below the smallest fp32 number, their
// difference keeps its precision
struct Residual {
    Side p, q;
    const float *zp, *zq;
    // its logarithm; minus infinity where p does not exceed q
    __device__ __forceinline__ double operator()(int j) const {
        if (p.kept(zp[j], j) == 0.0) return -INFINITY;
        const double a = ((double)zp[j] - (double)p.kept.top) * p.kept.inv_t - p.log_total;
        if (q.kept(zq[j], j) == 0.0) return a;
        const double d = ((double)zq[j] - (double)q.kept.top) * q.kept.inv_t - q.log_total - a;
        return d < 0.0 ? a + log(-expm1(d)) : -INFINITY;
    }
};

__global__ void __launch_bounds__(NT) k_filter_verify(FilterVerifyArgs v) {
    __shared__ BlockLds L;
    __shared__ WalkLds K;
    __shared__ double ratio_of[8], top_of[NW];
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
        double c = -INFINITY;
        for (int j = j0 + tid; j < j1; j += NT) c = fmax(c, res(j));
        c = block_max(c);
        uint64_t sum = 0;
        if (c > -INFINITY)
            for (int j = j0 + tid; j < j1; j += NT) sum += whole(exp(res(j) - c), a.weight_bits);
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
            // its ids: rounded one by one their weights may add up to a little less than the segment's, whose last id of some weight then stands in
            const int s0 = K.seg * a.seg_ids, s1 = min(a.V, s0 + a.seg_ids), per = (a.seg_ids + NT - 1) / NT;
            const int i0 = min(s1, s0 + tid * per), i1 = min(s1, i0 + per);
            uint64_t own = 0;
            int last = -1;
            for (int j = i0; j < i1; ++j) {
                const uint64_t y = whole(exp(res(j) - total_c), a.weight_bits);
                own += y;
                if (y) last = j;
            }
            const uint64_t at = K.before + block_scan(own, L, &ignore);
            int hit = -1;
            if (at <= target && target < at + own) {
                uint64_t s = at;
                for (int j = i0; j < i1 && hit < 0; ++j) {
                    s += whole(exp(res(j) - total_c), a.weight_bits);
                    if (s > target) hit = j;
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
        tok = draw(a, w, rejected ? v.u_resample[r] : v.u_final, [&](int j) { return p.kept(zp[j], j); }, K, L, &x, &total);
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

int launch_rows(const FilterArgs &a, const LaunchCtx &c) {
    if (a.V < 1 || a.rows < 1 || a.rows > kFilterRows || a.n_seg > kFilterMaxSegs || !(a.inv_t > 0.0)) return (int)hipErrorInvalidValue;
    const dim3 grid(a.n_seg, a.rows), wg(NT);
    int rc = launch<k_filter_top>(c, grid, wg, 0, a);
    if (rc) return rc;
    if (a.top_k || a.top_p < 1.0) {
        if ((rc = launch<k_filter_buckets>(c, grid, wg, 0, a))) return rc;
        return launch<k_filter_row<true>>(c, grid, wg, 0, a);
    }
    return launch<k_filter_row<false>>(c, grid, wg, 0, a);
}

}  // namespace

void filter_finish(FilterArgs &a, float temperature, int top_k, float top_p, float min_p) {
    const int n = (a.V + kFilterSegIds - 1) / kFilterSegIds, most = n < kFilterMaxSegs ? n : kFilterMaxSegs;
    a.seg_ids = (a.V + most - 1) / most;
    a.n_seg = (a.V + a.seg_ids - 1) / a.seg_ids;
    a.inv_t = 1.0 / (double)temperature;
    a.bucket_scale = 64.0 * a.inv_t < 3e38 ? (float)(64.0 * a.inv_t) : 3e38f;
    a.top_k = top_k < a.V ? top_k : 0;
    a.top_p = top_p > 0.f && top_p < 1.f ? (double)top_p : 1.0;
    a.min_p = (double)min_p;
    a.weight_bits = 62;                                  // V weights of up to 2^weight_bits add up to less than 2^63
    for (int v = a.V; v > 0; v >>= 1) --a.weight_bits;
}

int launch_filter_sample(const FilterArgs &a, const LaunchCtx &c) {
    if (a.rows != 1 || !a.tok_out) return (int)hipErrorInvalidValue;
    return launch_rows(a, c);
}

int launch_filter_probs(const FilterArgs &a, float *probs, const LaunchCtx &c) {
    if (a.tok_out) return (int)hipErrorInvalidValue;
    const int rc = launch_rows(a, c);
    return rc ? rc : launch<k_filter_probs>(c, dim3(a.n_seg, a.rows), dim3(NT), 0, a, probs);
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
