// The 8-bit cache: storing key and value rows, reading them out, and attention over them (layout: ad_kvq.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "ad_device.h"
#include "ad_internal.h"
#include "ad_kvq.h"
#include "ad_launch.h"

namespace ad {

namespace {

typedef __attribute__((__vector_size__(2 * sizeof(uint32_t)))) uint32_t u32x2;
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------------------------------------------
// quantisation
// ---------------------------------------------------------------------------------------------------
// The exponent byte of a row whose largest magnitude is amax: e the smallest with amax <= 448 * 2^e (448 = 1.75 * 2^8 is the largest code), not
// below -126, where 2^e and 2^-e are both normal numbers.
__device__ __forceinline__ uint32_t scale_byte(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int b = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)(b < 1 ? 1 : b);
}
__device__ __forceinline__ float two_to(uint32_t byte) { return __uint_as_float(byte << 23); }             // the scale itself
__device__ __forceinline__ float two_to_minus(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// magnitude for the scale: entries that are infinite or not numbers have no part in it
__device__ __forceinline__ float finite_abs(float x) {
    const float a = fabsf(x);
    return a <= 3.402823466e38f ? a : 0.f;
}
// codes of four values already divided by the scale: rounded to nearest even by the conversion, within range by the choice of the scale.  Values that are infinite or
// no numbers become the code that is no number.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// largest value over N = 8 or 16 neighbouring lanes
template <int N>
__device__ __forceinline__ float max_lanes(float v) {
    v = fmaxf(v, dpp<0xB1>(v));
    v = fmaxf(v, dpp<0x4E>(v));
    v = fmaxf(v, dpp<0x141>(v));
    if (N == 16) v = fmaxf(v, dpp<0x140>(v));
    return v;
}
template <int SEL>
__device__ __forceinline__ f32x2 values2(uint32_t w) {
    const auto v = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, SEL);
    return (f32x2){v[0], v[1]};
}

// ---------------------------------------------------------------------------------------------------
// store and read-out: a workgroup per block of 64 positions and kv head
// ---------------------------------------------------------------------------------------------------
// Half of the threads have K, half V.  DH / 8 lanes hold a row, 8 entries each, so that the largest magnitude is a matter of three (four) moves between lanes,
// and each of them four rows, which are all on their way before the first is looked at.  K rows are stored as they are; V's four codes of a dimension make a
// word, and go through LDS, so that a block of 64 positions that is stored whole leaves in 16-byte pieces.  Bound by memory: 131072 rows of 8 heads of 128
// dimensions (1.34 GB) 268 us, 5.0 TB/s, which is what a large copy reaches (with a byte at a time into LDS and 256 threads 296); 1024 rows 6.0 us, one row 3.3,
// a launch's latency.
constexpr int kStoreThreads = 512;
template <int DH>
__global__ void __launch_bounds__(kStoreThreads) k_kvq_store(KvqRows a) {
    constexpr int LR = DH / 8, T = kStoreThreads / 2, NG = T / LR;         // lanes per row, threads of K, groups of four rows at a time
    __shared__ uint32_t vt[DH][kKvqBlock / 4 + 1];
    const int tid = threadIdx.x, g = blockIdx.y, p0 = (a.pos0 / kKvqBlock + (int)blockIdx.x) * kKvqBlock;
    const int first = p0 > a.pos0 ? p0 : a.pos0, last = a.pos0 + a.n;
    const int end = p0 + kKvqBlock < last ? p0 + kKvqBlock : last;
    const bool is_v = tid >= T;
    const int d = tid % LR * 8;
    const KvqCache &c = a.c;
    for (int grp = tid % T / LR; grp < kKvqBlock / 4; grp += NG) {
        const int pg = p0 + grp * 4;
        f32x4 x[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i][0] = x[i][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
            if (pg + i >= first && pg + i < end) {
                const float *src = (is_v ? a.v : a.k) + (size_t)(pg + i - a.pos0) * a.ld + g * DH + d;
                x[i][0] = *(const f32x4 *)src;
                x[i][1] = *(const f32x4 *)(src + 4);
            }
        }
        u32x2 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float m = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) m = fmaxf(m, fmaxf(fabsf(x[i][0][e]), fabsf(x[i][1][e])));
            m = max_lanes<LR>(m);
            if (m == INFINITY) {                           // (the same in all lanes of a row)
                m = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, fmaxf(finite_abs(x[i][0][e]), finite_abs(x[i][1][e])));
                m = max_lanes<LR>(m);
            }
            const uint32_t b = scale_byte(m);
            const float mul = two_to_minus(b);
            w[i] = (u32x2){codes4(x[i][0][0] * mul, x[i][0][1] * mul, x[i][0][2] * mul, x[i][0][3] * mul),
                           codes4(x[i][1][0] * mul, x[i][1][1] * mul, x[i][1][2] * mul, x[i][1][3] * mul)};
            if (pg + i >= first && pg + i < end) {
                const size_t row = (size_t)g * c.stride + pg + i;
                if (d == 0) (is_v ? c.Vs : c.Ks)[row] = (uint8_t)b;
                if (!is_v) *(u32x2 *)(c.Kc + row * DH + d) = w[i];
            }
        }
        if (is_v) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // 4 x 4 bytes turned over: [position][dimension] -> [dimension][position]
                const uint32_t lo01 = __builtin_amdgcn_perm(w[1][h], w[0][h], 0x05010400u), hi01 = __builtin_amdgcn_perm(w[1][h], w[0][h], 0x07030602u);
                const uint32_t lo23 = __builtin_amdgcn_perm(w[3][h], w[2][h], 0x05010400u), hi23 = __builtin_amdgcn_perm(w[3][h], w[2][h], 0x07030602u);
                vt[d + 4 * h][grp] = (lo01 & 0xffffu) | lo23 << 16;
                vt[d + 4 * h + 1][grp] = lo01 >> 16 | (lo23 & 0xffff0000u);
                vt[d + 4 * h + 2][grp] = (hi01 & 0xffffu) | hi23 << 16;
                vt[d + 4 * h + 3][grp] = hi01 >> 16 | (hi23 & 0xffff0000u);
            }
        }
    }
    __syncthreads();
    uint8_t *V = c.Vc + ((size_t)g * c.stride + p0) * DH;
    if (first == p0 && end == p0 + kKvqBlock) {
        for (int i = tid; i < DH * 4; i += kStoreThreads) {
            const uint32_t *src = &vt[i >> 2][(i & 3) * 4];
            *(u32x4 *)(V + i * 16) = (u32x4){src[0], src[1], src[2], src[3]};
        }
    } else {
        const int n = end - first;
        for (int i = tid; i < DH * n; i += kStoreThreads) {
            const int e = i / n, p = first - p0 + i % n;
            V[e * kKvqBlock + p] = (uint8_t)(vt[e][p >> 2] >> (8 * (p & 3)));
        }
    }
}

template <int DH>
__global__ void __launch_bounds__(256) k_kvq_read(KvqRows a) {
    constexpr int LR = DH / 8, RP = 256 / LR;
    __shared__ __attribute__((aligned(16))) uint8_t vt[DH][kKvqBlock + 16];
    const int tid = threadIdx.x, g = blockIdx.y, p0 = (a.pos0 / kKvqBlock + (int)blockIdx.x) * kKvqBlock;
    const int first = p0 > a.pos0 ? p0 : a.pos0, last = a.pos0 + a.n;
    const int end = p0 + kKvqBlock < last ? p0 + kKvqBlock : last;
    const int d = tid % LR * 8;
    const KvqCache &c = a.c;
    const uint8_t *V = c.Vc + ((size_t)g * c.stride + p0) * DH;
    for (int i = tid; i < DH * 4; i += 256) *(u32x4 *)&vt[i >> 2][(i & 3) * 16] = *(const u32x4 *)(V + i * 16);
    __syncthreads();
    for (int p = first + tid / LR; p < end; p += RP) {
        const size_t at = (size_t)(p - a.pos0) * a.ld + g * DH + d, row = (size_t)g * c.stride + p;
        auto put = [&](float *dst, u32x2 w, float s) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 lo = values2<0>(w[h]), hi = values2<1>(w[h]);
                *(f32x4 *)(dst + 4 * h) = (f32x4){lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
            }
        };
        put(a.k_out + at, *(const u32x2 *)(c.Kc + row * DH + d), two_to(c.Ks[row]));
        u32x2 w = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)vt[d + e][p - p0] << (8 * (e & 3));
        put(a.v_out + at, w, two_to(c.Vs[row]));
    }
}

// ---------------------------------------------------------------------------------------------------
// the values in bf16 for the prompt pass (exact: four significant bits and a power of two)
// ---------------------------------------------------------------------------------------------------
template <int DH>
__global__ void __launch_bounds__(256) k_kvq_expand(KvqExpand a) {
    const int tid = threadIdx.x, g = blockIdx.y, p0 = blockIdx.x * kKvqBlock;
    const KvqCache &c = a.c;
    __shared__ float vs[kKvqBlock];
    if (tid < kKvqBlock) vs[tid] = p0 + tid < a.n ? two_to(c.Vs[(size_t)g * c.stride + p0 + tid]) : 0.f;
    __syncthreads();
    // 8 codes of a K row per thread and turn
    for (int i = tid; i < kKvqBlock * (DH / 8); i += 256) {
        const int p = p0 + i / (DH / 8), d = i % (DH / 8) * 8;
        const size_t row = (size_t)g * c.stride + p;
        u16x8 o = {0, 0, 0, 0, 0, 0, 0, 0};
        if (p < a.n) {
            const u32x2 w = *(const u32x2 *)(c.Kc + row * DH + d);
            const float s = two_to(c.Ks[row]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x2 lo = values2<0>(w[h]), hi = values2<1>(w[h]);
                o[4 * h] = to16<false>(lo[0] * s);
                o[4 * h + 1] = to16<false>(lo[1] * s);
                o[4 * h + 2] = to16<false>(hi[0] * s);
                o[4 * h + 3] = to16<false>(hi[1] * s);
            }
        }
        *(u16x8 *)(a.K + row * DH + d) = o;
    }
    // 8 positions of a dimension
    const uint8_t *V = c.Vc + ((size_t)g * c.stride + p0) * DH;
    for (int i = tid; i < DH * (kKvqBlock / 8); i += 256) {
        const int d = i / (kKvqBlock / 8), p = i % (kKvqBlock / 8) * 8;
        const u32x2 w = *(const u32x2 *)(V + d * kKvqBlock + p);
        u16x8 o;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x2 lo = values2<0>(w[h]), hi = values2<1>(w[h]);
            const float x[4] = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
            for (int e = 0; e < 4; ++e) o[4 * h + e] = p0 + p + 4 * h + e < a.n ? to16<false>(x[e] * vs[p + 4 * h + e]) : (uint16_t)0;
        }
        *(u16x8 *)(a.V + ((size_t)g * DH + d) * c.stride + p0 + p) = o;
    }
}

// ---------------------------------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------------------------------
// Work item (kv head, split): a workgroup whose wavefronts take the item's blocks of 64 positions in turn, under an online softmax of their
// own; their results meet in LDS, the items' in k_kvq_combine.  All of a pass's query rows (16 or 32) of the kv head's group meet a block's codes.
//
// Products.  S^T = K q^T: codes are exact in fp16, queries are scaled to a largest magnitude in [128, 256) and split into fp16 hi and lo parts (22 bits), sums are
// fp32.  A lane has 16 consecutive dimensions of a key: the first eight are its part of one k-step, the other eight of the next, and the queries are
// dealt out the same way.  Rows of the four score tiles are assigned to keys so that lane (n, gq) ends up with keys gq * 16 .. + 15 of query row n, which is, eight by
// eight, the B operand of O^T = V^T P^T against 16 consecutive positions of a dimension.  The scales never touch the codes: K's multiply the scores, V's the
// probabilities, relative to the largest that the row has seen so that fp16 has them all in range (again hi and lo).
//
// Copies.  Every wavefront has room for one block's codes in LDS, filled from memory without a way through registers and in operand order: the next block's
// K is on its way as soon as the scores are formed, its V after the second product, and nobody else reads or writes there, so the loop has no barriers.
//
// Bound, at long contexts, by the read of the cache: 32 query heads on 8 kv heads of 128 dimensions at context 131072 (270 MB), 1 row 48 us in this kernel, 5.6 TB/s of
// the 6.6 that a kernel that only reads reaches, 8 rows 56 us, 4.8 (a row tile more: conversions, softmax and products of a block take about as long as its
// copies).  With K and V by way of registers, a block ahead, and 4 wavefronts it was 71 us.  At short ones by the chain through one block, 5 to 7.4 us, and the fold's kernel.
//
// A layer step's own rows are stored by the last item of each kv head, which attends to them as one more block of its last wavefront; the others see the cache as it
// was.  With a kernel of its own for the rotation and the store the step took 1 to 2 us more.
template <int DH, int RT, int NW>
struct KvqAttnLds {
    static constexpr int KU = DH / 64 * 4 * 64, VU = DH / 16 * 64;      // 16-byte units of a block: [tile][pair of k-steps][lane], [16 dimensions][lane]
    union {
        u32x4 codes[NW][KU + VU];
        float part[NW][16][DH + 4];                        // the wavefronts' results, one row tile at a time (rows padded to 16 bytes)
    };
    u32x4 scales[NW][16];                                  // 64 bytes of K's, 64 of V's (and the same again)
    f16x8 q[RT][DH / 64][2][2][64];                        // [row tile][pair of k-steps][of the pair][hi, lo][lane]
    float q_mul[RT * 16];
    int see[RT * 16], tok[RT * 16];
    float mx[NW][16], sum[NW][16];
    // a layer step's own rows: codes [token][dimension], [dimension][token], scales of K, of V
    uint8_t own_k[8][DH], own_v[DH][8], own_scales[2][8];
};

// x / d for any x >= 0: the rounded-up reciprocal is never too small and, below 2^32, at most one too large
__device__ __forceinline__ int quotient(int x, int d, unsigned mul) {
    const int q = div_small(x, mul);
    return q * d > x ? q - 1 : q;
}

// 8 codes as an MFMA operand
__device__ __forceinline__ f16x8 operand(uint32_t w0, uint32_t w1) {
    const half2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, 1.0f, true);
    const half2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, 1.0f, true);
    return (f16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f32x4 mma(const f16x8 &a, const f16x8 &b, const f32x4 &c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// output of query row r (of kv head g), dimensions d, d + 1
__device__ __forceinline__ void kvq_output(const KvqAttn &a, int g, int r, int d, float y0, float y1) {
    const int t = quotient(r, a.G, a.mul_G), col = (g * a.G + (r - t * a.G)) * a.c.dh + d;
    if (a.out) {
        *(f32x2 *)(a.out + (size_t)t * a.Hq * a.c.dh + col) = (f32x2){y0, y1};
    } else if (a.f16) {
        store_act<true>(a.Bo, a.Bo_KT, col, t, y0);
        store_act<true>(a.Bo, a.Bo_KT, col + 1, t, y1);
    } else {
        store_act<false>(a.Bo, a.Bo_KT, col, t, y0);
        store_act<false>(a.Bo, a.Bo_KT, col + 1, t, y1);
    }
}

// waits until at most N copies are in flight and what has been read from LDS is there
template <int N>
__device__ __forceinline__ void copies_left() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4 << 14));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
// lane l's 16 bytes, 4 bytes go to place l of dst (the same for all lanes)
__device__ __forceinline__ void units_to_lds(const void *src, void *dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
}
__device__ __forceinline__ void words_to_lds(const void *src, void *dst) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)dst, 4, 0, 0);
}

template <int DH, int RT, int NW, bool OWN>
__global__ void __launch_bounds__(64 * NW, NW / 4) k_kvq_attn(KvqAttn a) {
    constexpr int J = DH / 64, DT = DH / 16, RP = RT * 16, PR = DH + 2, NTH = 64 * NW, KU = KvqAttnLds<DH, RT, NW>::KU;
    constexpr int NK = 4 * J + 1, NV = DT;                 // copies of a block's K (with the scales), of its V
    warm_kernel_args<sizeof(KvqAttn)>();
    constexpr int kPBits = 14;                             // probabilities times 2^14: those of 2^-17 and more keep 21 bits in fp16 hi and lo
    extern __shared__ __attribute__((aligned(16))) char lds_raw[];
    KvqAttnLds<DH, RT, NW> &L = *reinterpret_cast<KvqAttnLds<DH, RT, NW> *>(lds_raw);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, gq = lane >> 4;
    const int item = blockIdx.x, g = quotient(item, a.S, a.mul_S), s = item - g * a.S;
    const int r0 = blockIdx.y * RP, nr = a.R - r0 < RP ? a.R - r0 : RP;
    const int b_end = (a.n + kKvqBlock - 1) / kKvqBlock, b0 = s * a.per, b1 = b0 + a.per < b_end ? b0 + a.per : b_end;
    const uint8_t *Kg = a.c.Kc + (size_t)g * a.c.stride * DH, *Vg = a.c.Vc + (size_t)g * a.c.stride * DH;
    const uint8_t *Sg = ((lane & 31) < 16 ? a.c.Ks : a.c.Vs) + (size_t)g * a.c.stride + (lane & 15) * 4;
    u32x4 *const my = L.codes[wave];
    auto copy_k = [&](int b) {
        const uint8_t *base = Kg + (size_t)b * kKvqBlock * DH + ((n >> 2) * 16 + (n & 3)) * DH + gq * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < J; ++j) units_to_lds(base + t * 4 * DH + j * 64, my + (t * J + j) * 64);
        words_to_lds(Sg + (size_t)b * kKvqBlock, &L.scales[wave][0]);
    };
    auto copy_v = [&](int b) {
        const uint8_t *base = Vg + (size_t)b * kKvqBlock * DH + n * kKvqBlock + gq * 16;
#pragma unroll
        for (int d = 0; d < DT; ++d) units_to_lds(base + d * 16 * kKvqBlock, my + KU + d * 64);
    };
    // queries: a thread takes 16 dimensions of a row; rows past the last are zeros.  Their loads come before the copies: what waits for them does not wait for those.
    constexpr int LR = DH / 16;                            // threads per row
    static_assert(RP * LR <= NTH, "a turn for all rows");
    const int rr = tid / LR, ch = tid % LR, r_q = r0 + (rr < nr ? rr : 0), t_q = quotient(r_q, a.G, a.mul_G);
    constexpr int half = DH / 2;
    f32x4 x[4], y[4], turn[8];                             // (a layer step: the other half's dimensions, and (cos, sin) of each)
    if (tid < RP * LR) {
        const float *qp = a.q + (size_t)t_q * a.ld_q + (size_t)(g * a.G + (r_q - t_q * a.G)) * DH + ch * 16;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = *(const f32x4 *)(qp + e * 4);
        if constexpr (OWN) {
            const float *other = ch * 16 < half ? qp + half : qp - half, *rp = a.rope + ((size_t)t_q * half + (ch * 16) % half) * 2;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = *(const f32x4 *)(other + e * 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) turn[e] = *(const f32x4 *)(rp + e * 4);
        }
    }
    // a layer step's own rows (a wavefront per row: lane i has dimensions i and i + half), the first of each wavefront's as early as the queries
    const bool own_item = OWN && s == a.S - 1;
    const int i_own = lane & (half - 1);
    f32x2 own_x = {0.f, 0.f}, own_cs = {0.f, 0.f};
    auto load_own = [&](int row) {
        const bool is_v = row >= a.m;
        const int t = is_v ? row - a.m : row;
        const float *src = a.q + (size_t)t * a.ld_q + (size_t)(a.Hq + (is_v ? a.c.Hkv : 0) + g) * DH + i_own;
        own_x = (f32x2){src[0], src[half]};
        if (!is_v) own_cs = *(const f32x2 *)(a.rope + (t * half + i_own) * 2);
    };
    if (own_item && wave < 2 * a.m) load_own(wave);
    __builtin_amdgcn_sched_barrier(0);
    int b = b0 + wave;
    if (b < b1) {
        copy_k(b);
        copy_v(b);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (tid < RP * LR) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if constexpr (OWN) {
                    const float cs = turn[e * 2 + c / 2][c % 2 * 2], sn = turn[e * 2 + c / 2][c % 2 * 2 + 1];
                    x[e][c] = ch * 16 < half ? x[e][c] * cs - y[e][c] * sn : y[e][c] * sn + x[e][c] * cs;
                }
                x[e][c] = rr < nr ? x[e][c] : 0.f;
                m = fmaxf(m, finite_abs(x[e][c]));
            }
        m = fmaxf(m, dpp<0xB1>(m));                        // over the row's 4 or 8 neighbouring lanes
        m = fmaxf(m, dpp<0x4E>(m));
        if (LR == 8) m = fmaxf(m, dpp<0x141>(m));
        // 2^(7 - exponent of m): both it and its inverse stay normal numbers
        int ex = (int)(__float_as_uint(m) >> 23) - 127;
        ex = ex < -100 ? -100 : ex;
        const float up = __uint_as_float((uint32_t)(127 + 7 - ex) << 23);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u16x8 hi8, lo8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint16_t hi, lo;
                split16<true>(x[h * 2 + (e >> 2)][e & 3] * up, hi, lo);
                hi8[e] = hi;
                lo8[e] = lo;
            }
            L.q[rr >> 4][ch >> 2][h][0][(rr & 15) + 16 * (ch & 3)] = __builtin_bit_cast(f16x8, hi8);
            L.q[rr >> 4][ch >> 2][h][1][(rr & 15) + 16 * (ch & 3)] = __builtin_bit_cast(f16x8, lo8);
        }
        if (ch == 0) {
            L.q_mul[rr] = __uint_as_float((uint32_t)(127 - 7 + ex) << 23) * a.scale;
            int see = a.see[0];
#pragma unroll
            for (int c = 1; c < 8; ++c) see = t_q == c ? a.see[c] : see;
            L.see[rr] = see;
            L.tok[rr] = t_q;
        }
    }
    if (own_item) {
        for (int row = wave; row < 2 * a.m; row += NW) {
            if (row != wave) load_own(row);
            const bool is_v = row >= a.m;
            const int t = is_v ? row - a.m : row, i = i_own, p = a.pos0 + t;
            float v0 = own_x[0], v1 = own_x[1];
            if (!is_v) {
                const float k0 = v0 * own_cs[0] - v1 * own_cs[1], k1 = v0 * own_cs[1] + v1 * own_cs[0];
                v0 = k0;
                v1 = k1;
            }
            const uint32_t bits = scale_byte(max64(fmaxf(finite_abs(v0), finite_abs(v1))));
            const float mul = two_to_minus(bits);
            const uint32_t cc = codes4(v0 * mul, v1 * mul, 0.f, 0.f);
            const uint8_t c0 = (uint8_t)cc, c1 = (uint8_t)(cc >> 8);
            if (lane < half) {
                const size_t at = (size_t)g * a.c.stride + p;
                const bool store = blockIdx.y == 0;        // (every pass has the rows in LDS; one stores them)
                if (is_v) {
                    L.own_v[i][t] = c0;
                    L.own_v[i + half][t] = c1;
                    if (store) {
                        uint8_t *V = a.c.Vc + ((size_t)g * a.c.stride + (p & ~(kKvqBlock - 1))) * DH + (p & (kKvqBlock - 1));
                        V[i * kKvqBlock] = c0;
                        V[(i + half) * kKvqBlock] = c1;
                    }
                } else {
                    L.own_k[t][i] = c0;
                    L.own_k[t][i + half] = c1;
                    if (store) {
                        a.c.Kc[at * DH + i] = c0;
                        a.c.Kc[at * DH + i + half] = c1;
                    }
                }
                if (i == 0) {
                    L.own_scales[is_v][t] = (uint8_t)bits;
                    if (store) (is_v ? a.c.Vs : a.c.Ks)[at] = (uint8_t)bits;
                }
            }
        }
    }
    // (a barrier that leaves the copies in flight)
    copies_left<63>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    float q_mul[RT], mx[RT], sum[RT];
    int see[RT], e_ref[RT];                                // o is in units of 2^(e_ref - 127 - kPBits)
    f32x4 o[RT][DT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        q_mul[i] = L.q_mul[i * 16 + n];
        see[i] = L.see[i * 16 + n];
        mx[i] = -INFINITY;
        sum[i] = 0.f;
        e_ref[i] = 0;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[i][d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    bool own_left = own_item && wave == NW - 1;
    for (;; b += NW) {
        int p0 = b * kKvqBlock, next = b + NW, n_live = a.n;           // first position, the wavefront's next block, the positions that are live
        bool part_hidden = p0 + kKvqBlock > a.n_all;                   // some row does not see all of the block
        if (b < b1) {
            copies_left<NV>();
        } else if (own_left) {
            // the call's own rows, as a block that starts at the first of them (what is behind the last may be anything)
            own_left = false;
            p0 = a.pos0;
            next = b1;
            n_live = a.pos0 + a.m;
            part_hidden = true;
            const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int j = 0; j < J; ++j) my[(t * J + j) * 64 + lane] = t < 2 && n < 4 ? *(const u32x4 *)&L.own_k[(t & 1) * 4 + (n & 3)][j * 64 + gq * 16] : zero;
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const u32x2 w = *(const u32x2 *)L.own_v[d * 16 + n];
                my[KU + d * 64 + lane] = gq == 0 ? (u32x4){w[0], w[1], 0, 0} : zero;
            }
            if (lane < 2) {
                const u32x2 w = *(const u32x2 *)L.own_scales[lane];
                L.scales[wave][lane * 4] = (u32x4){w[0], w[1], 0, 0};
            }
            copies_left<0>();
        } else {
            break;
        }
        f32x4 sc[RT][4];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) sc[i][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        const u32x4 ks = L.scales[wave][gq];
        u32x4 vs = L.scales[wave][4 + gq];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            u32x4 k[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) k[t] = my[(t * J + j) * 64 + lane];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                f16x8 q[RT][2];
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int x = 0; x < 2; ++x) q[i][x] = L.q[i][j][h][x][lane];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const f16x8 kk = operand(k[t][2 * h], k[t][2 * h + 1]);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < RT; ++i) sc[i][t] = mma(kk, q[i][x], sc[i][t]);
                }
            }
        }
        if (next < b1) {
            copies_left<NV>();                             // (what has been read of K is there: its place is free)
            copy_k(next);
        }
        // entries behind the last position that is seen may be anything: their codes and scales are taken out
        const int live = n_live - p0 - gq * 16;            // of this lane's 16 positions
        const bool ragged = p0 + kKvqBlock > n_live;
        u32x4 keep = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
        auto keep_first = [&](int count) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int l = count - 4 * w;
                keep[w] = l >= 4 ? 0xffffffffu : l <= 0 ? 0u : (1u << (8 * l)) - 1u;
            }
        };
        if (ragged) {
            keep_first(live);
            vs &= keep;
        }
        float k_mul[16];
        int vb[16], top = 0;
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            k_mul[c] = two_to((ks[c >> 2] >> (8 * (c & 3))) & 0xffu);
            vb[c] = (int)((vs[c >> 2] >> (8 * (c & 3))) & 0xffu);
            top = vb[c] > top ? vb[c] : top;
        }
        f16x8 p[RT][2][2];                                 // [.][k-step][hi, lo]
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float w[16], bm = -INFINITY;
            int e_new = top;
            if (part_hidden) {                             // (what a row does not see has no part in its scale)
                e_new = 0;
                const int last = see[i] < n_live ? see[i] : n_live - 1;
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    const bool seen = p0 + gq * 16 + c <= last;
                    w[c] = seen ? sc[i][c >> 2][c & 3] * k_mul[c] : -INFINITY;
                    e_new = seen && vb[c] > e_new ? vb[c] : e_new;
                    bm = fmaxf(bm, w[c]);
                }
            } else {
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    w[c] = sc[i][c >> 2][c & 3] * k_mul[c];
                    bm = fmaxf(bm, w[c]);
                }
            }
            bm = max_rows(bm);
            e_new = (int)max_rows((float)e_new);
            e_new = e_new > e_ref[i] ? e_new : e_ref[i];
            const float shrink = ldexpf(1.0f, e_ref[i] - e_new);
            e_ref[i] = e_new;
            const float nm = fmaxf(mx[i], bm * q_mul[i]), ref = softmax_ref(nm), alpha = exp2_fast(mx[i] - ref);
            mx[i] = nm;
            float add = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const int c = h * 8 + e;
                    const float x0 = exp2_fast(fmaf(w[c], q_mul[i], -ref)), x1 = exp2_fast(fmaf(w[c + 1], q_mul[i], -ref));
                    add += x0 + x1;
                    const float y0 = ldexpf(x0, vb[c] - e_new + kPBits), y1 = ldexpf(x1, vb[c + 1] - e_new + kPBits);
                    // (both parts cut off, two values an instruction: what is lost is below 2^-21 of the value)
                    const auto hi = __builtin_amdgcn_cvt_pkrtz(y0, y1);
                    const auto lo = __builtin_amdgcn_cvt_pkrtz(y0 - (float)hi[0], y1 - (float)hi[1]);
                    p[i][h][0][e] = (_Float16)hi[0];
                    p[i][h][0][e + 1] = (_Float16)hi[1];
                    p[i][h][1][e] = (_Float16)lo[0];
                    p[i][h][1][e + 1] = (_Float16)lo[1];
                }
            sum[i] = sum[i] * alpha + add;
            const float f = alpha * shrink;
            if (!__all(f == 1.0f)) {
#pragma unroll
                for (int d = 0; d < DT; ++d) o[i][d] *= f;
            }
        }
        if (next < b1) copies_left<NK>();
        else copies_left<0>();
        // a value that is not a number, at a position that only some rows see, must not reach the others by way of 0 * NaN
        bool bad = false;
        if (part_hidden) {
#pragma unroll 1
            for (int d = 0; d < DT; ++d) {
                const u32x4 v = my[KU + d * 64 + lane] & keep;
#pragma unroll
                for (int w = 0; w < 4; ++w) bad |= (((v[w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
            }
            bad = __any(bad);
        }
        if (bad) {
#pragma unroll 1
            for (int t = 0; t < a.m; ++t) {
                keep_first((a.see[t] < n_live ? a.see[t] + 1 : n_live) - p0 - gq * 16);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const bool mine = L.tok[i * 16 + n] == t;
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const u32x4 v = my[KU + d * 64 + lane] & keep;
                        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const f16x8 vv = operand(v[2 * h], v[2 * h + 1]);
                            x = mma(vv, p[i][h][0], x);
                            x = mma(vv, p[i][h][1], x);
                        }
                        if (mine) o[i][d] += x;
                        __builtin_amdgcn_sched_barrier(0);             // (rare: as few registers as it takes)
                    }
                }
            }
        } else {
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                u32x4 v = my[KU + d * 64 + lane];
                if (ragged) v &= keep;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const f16x8 vv = operand(v[2 * h], v[2 * h + 1]);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < RT; ++i) o[i][d] = mma(vv, p[i][h][x], o[i][d]);
                }
            }
        }
        if (next < b1) {
            copies_left<NK>();                             // (likewise V's)
            copy_v(next);
        }
    }
    // lane (n, gq): row n of a tile, dimensions d * 16 + gq * 4 .. + 3.  The wavefronts' results are folded in wavefront order.
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int ni = nr - i * 16 < 16 ? nr - i * 16 : 16;            // rows of this tile
        if (ni <= 0) break;
        const float den = sum_rows(sum[i]), unit = ldexpf(1.0f, e_ref[i] - 127 - kPBits);
        if (gq == 0) {
            L.mx[wave][n] = mx[i];
            L.sum[wave][n] = den;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) *(f32x4 *)&L.part[wave][n][d * 16 + gq * 4] = o[i][d] * unit;
        __syncthreads();
        for (int idx = tid; idx < ni * (DH / 2); idx += NTH) {
            const int rr = idx / (DH / 2), d = idx % (DH / 2) * 2, r = r0 + i * 16 + rr;
            float M = -INFINITY, sums = 0.f;
            f32x2 num = {0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) M = fmaxf(M, L.mx[w][rr]);
            const float ref = softmax_ref(M);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = exp2_fast(L.mx[w][rr] - ref);           // a wavefront without keys: exp(-inf) = 0, of sums that are 0
                const f32x2 x = *(const f32x2 *)&L.part[w][rr][d];
                sums += f * L.sum[w][rr];
                num[0] += f * x[0];
                num[1] += f * x[1];
            }
            if (a.S == 1) {
                kvq_output(a, g, r, d, num[0] / sums, num[1] / sums);
                continue;
            }
            float *out = a.part + (((size_t)g * a.S + s) * a.R + r) * PR;
            *(f32x2 *)(out + d) = num;
            if (d == 0) *(f32x2 *)(out + DH) = (f32x2){M, sums};
        }
        __syncthreads();
    }
}

// Folds the items of a query row in their order: a workgroup per row, DH / 2 threads (two dimensions each) times groups that take every
// NG-th item, a batch of them in flight.
template <int DH>
__global__ void __launch_bounds__(256) k_kvq_combine(KvqAttn a) {
    constexpr int PR = DH + 2, TG = DH / 2, NG = 256 / TG, KB = 8;
    __shared__ float st[NG][2];
    __shared__ f32x2 part[NG][TG];
    const int tid = threadIdx.x, grp = tid / TG, d = 2 * (tid % TG);
    const int g = quotient((int)blockIdx.x, a.R, a.mul_R), r = (int)blockIdx.x - g * a.R;
    const float *base = a.part + ((size_t)g * a.S * a.R + r) * PR;
    float M = -INFINITY, den = 0.f;
    f32x2 o = {0.f, 0.f};
    for (int s0 = grp; s0 < a.S; s0 += NG * KB) {
        f32x2 x[KB], ms[KB];
#pragma unroll
        for (int i = 0; i < KB; ++i) {                          // items past the end repeat the group's first (weight 0)
            const int s = s0 + i * NG < a.S ? s0 + i * NG : s0;
            const float *p = base + (size_t)s * a.R * PR;
            ms[i] = *(const f32x2 *)(p + DH);
            x[i] = *(const f32x2 *)(p + d);
        }
        float nm = M;
#pragma unroll
        for (int i = 0; i < KB; ++i) {
            if (s0 + i * NG >= a.S) ms[i] = (f32x2){-INFINITY, 0.f};
            nm = fmaxf(nm, ms[i][0]);
        }
        const float ref = softmax_ref(nm), alpha = exp2_fast(M - ref);
        M = nm;
        den *= alpha;
        o *= alpha;
#pragma unroll
        for (int i = 0; i < KB; ++i) {
            // (an item that this row sees nothing of has sums of 0 and a maximum of minus infinity)
            const float w = exp2_fast(ms[i][0] - ref);
            den += w * ms[i][1];
            o[0] += w * x[i][0];
            o[1] += w * x[i][1];
        }
    }
    part[grp][tid % TG] = o;
    if (d == 0) {
        st[grp][0] = M;
        st[grp][1] = den;
    }
    __syncthreads();
    if (tid >= TG) return;
    float m = -INFINITY, sum = 0.f;
    f32x2 y = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; ++i) m = fmaxf(m, st[i][0]);
    const float ref = softmax_ref(m);
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        const float w = exp2_fast(st[i][0] - ref);
        sum += w * st[i][1];
        y += w * part[i][tid];
    }
    kvq_output(a, g, r, d, y[0] / sum, y[1] / sum);
}

// LDS beyond 64 KiB is asked for once per kernel and device, with that device current
template <int DH, int RT, int NW, bool OWN>
int allow_lds(int device) {
    static std::atomic<uint64_t> done{0};
    constexpr size_t lds = sizeof(KvqAttnLds<DH, RT, NW>);
    static_assert(lds <= 160 * 1024, "LDS of a compute unit");
    int current = 0;
    if (hipGetDevice(&current) != hipSuccess) return (int)hipGetLastError();
    if (device < 0) device = current;
    const uint64_t bit = (uint64_t)1 << (device & 63);
    if (device < 64 && (done.load(std::memory_order_acquire) & bit)) return 0;
    hipError_t e = device != current ? hipSetDevice(device) : hipSuccess;
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)k_kvq_attn<DH, RT, NW, OWN>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (device != current) (void)hipSetDevice(current);
    if (e == hipSuccess && device < 64) done.fetch_or(bit, std::memory_order_release);
    return (int)e;
}

template <int DH, int RT, int NW, bool OWN>
int launch_attn_as(const KvqAttn &a, const LaunchCtx &c) {
    const int rc = allow_lds<DH, RT, NW, OWN>(c.device);
    if (rc) return rc;
    return launch<k_kvq_attn<DH, RT, NW, OWN>>(c, dim3(a.c.Hkv * a.S, (a.R + RT * 16 - 1) / (RT * 16)), dim3(64 * NW), sizeof(KvqAttnLds<DH, RT, NW>), a);
}

template <int DH, bool OWN>
int launch_attn_dh(const KvqAttn &a, const LaunchCtx &c) {
    int rc;
    if (a.tiles == 1) rc = a.waves == 4 ? launch_attn_as<DH, 1, 4, OWN>(a, c) : launch_attn_as<DH, 1, 8, OWN>(a, c);
    else rc = a.waves == 4 ? launch_attn_as<DH, 2, 4, OWN>(a, c) : launch_attn_as<DH, 2, 8, OWN>(a, c);
    if (rc || a.S == 1) return rc;
    return launch<k_kvq_combine<DH>>(c, dim3(a.c.Hkv * a.R), dim3(256), 0, a);
}

bool rows_ok(const KvqRows &a) { return a.n >= 1 && a.pos0 >= 0 && (int64_t)a.pos0 + a.n <= a.c.stride && a.ld % 4 == 0; }
dim3 rows_grid(const KvqRows &a) { return dim3((a.pos0 + a.n - 1) / kKvqBlock - a.pos0 / kKvqBlock + 1, a.c.Hkv); }

}  // namespace

int launch_kvq_store(const KvqRows &a, const LaunchCtx &c) {
    if (!rows_ok(a)) return (int)hipErrorInvalidValue;
    if (a.c.dh == 128) return launch<k_kvq_store<128>>(c, rows_grid(a), dim3(kStoreThreads), 0, a);
    if (a.c.dh == 64) return launch<k_kvq_store<64>>(c, rows_grid(a), dim3(kStoreThreads), 0, a);
    return (int)hipErrorInvalidValue;
}

int launch_kvq_read(const KvqRows &a, const LaunchCtx &c) {
    if (!rows_ok(a)) return (int)hipErrorInvalidValue;
    if (a.c.dh == 128) return launch<k_kvq_read<128>>(c, rows_grid(a), dim3(256), 0, a);
    if (a.c.dh == 64) return launch<k_kvq_read<64>>(c, rows_grid(a), dim3(256), 0, a);
    return (int)hipErrorInvalidValue;
}

int launch_kvq_expand(const KvqExpand &a, const LaunchCtx &c) {
    if (a.n < 1 || a.n > a.c.stride) return (int)hipErrorInvalidValue;
    const dim3 grid((a.n + kKvqBlock - 1) / kKvqBlock, a.c.Hkv);
    if (a.c.dh == 128) return launch<k_kvq_expand<128>>(c, grid, dim3(256), 0, a);
    if (a.c.dh == 64) return launch<k_kvq_expand<64>>(c, grid, dim3(256), 0, a);
    return (int)hipErrorInvalidValue;
}

// How the work is divided, for n_wg compute units.  A block of 64 positions per wavefront and 16 query rows per workgroup (the shortest chain) while every workgroup
// has a compute unit to itself; else 32 rows, which a block's codes are converted once for, and beyond four blocks per compute unit 8 wavefronts and as many
// blocks each as it takes.  Contexts of up to eight blocks are one item per kv head, which writes the output itself.
// Measured, 32 query heads on 8 kv heads of 128 dimensions, 1 / 8 rows, us a call: context 300, 4 wavefronts 9.6 / 15.4, 8 8.9 / 13.1; 4096, 4 10.4 / 14.3, 8 11.5 / 15.9;
// 9203 (both 8) 12.3 / 16.5.
void kvq_attn_finish(KvqAttn &a, int n_wg) {
    a.G = a.Hq / a.c.Hkv;
    a.R = a.G * a.m;
    a.n = a.n_all = a.see[0] + 1;
    for (int t = 1; t < a.m; ++t) {
        a.n = a.see[t] + 1 > a.n ? a.see[t] + 1 : a.n;
        a.n_all = a.see[t] + 1 < a.n_all ? a.see[t] + 1 : a.n_all;
    }
    if (a.rope) a.n = a.n_all = a.pos0;                    // (the rows' own positions are not cached yet)
    const int blocks = (a.n + kKvqBlock - 1) / kKvqBlock;
    const int tiles = (a.R + 15) / 16, heads = a.c.Hkv;
    if (blocks <= 8) {
        a.waves = blocks <= 4 ? 4 : 8;
        a.per = 8;
        a.tiles = tiles == 1 || (int64_t)heads * tiles <= n_wg ? 1 : 2;
    } else {
        const int fours = (blocks + 3) / 4;
        a.tiles = tiles == 1 || (int64_t)heads * tiles * fours <= n_wg ? 1 : 2;
        const int64_t wide = (int64_t)heads * ((tiles + a.tiles - 1) / a.tiles);
        int most = (int)(n_wg / wide);                     // items per kv head
        most = most < 1 ? 1 : most > kKvqMaxSplits ? kKvqMaxSplits : most;
        a.waves = fours <= most ? 4 : 8;
        const int least = (blocks + most - 1) / most;
        a.per = (least + a.waves - 1) / a.waves * a.waves;
    }
    a.S = blocks ? (blocks + a.per - 1) / a.per : 1;
    // the own rows are a second chain behind the last item's own: on a compute unit of their own if there is one to spare.  Layer step of the 8B shape,
    // 1 row at context 4096 89.0 -> 85.5 us, 8 rows at 9203 108.7 -> 103.4 (a 16-bit cache: 85.1, 102.3)
    const int passes = (tiles + a.tiles - 1) / a.tiles;
    if (a.rope && a.S > 1 && a.S < kKvqMaxSplits && (int64_t)heads * passes * (a.S + 1) <= n_wg) ++a.S;
    a.mul_S = div_multiplier(a.S);
    a.mul_G = div_multiplier(a.G);
    a.mul_R = div_multiplier(a.R);
}

int launch_kvq_attn(const KvqAttn &a, const LaunchCtx &c) {
    if (a.m < 1 || a.m > 8 || a.n < (a.rope ? 0 : 1) || a.n > a.c.stride || a.S < 1 || a.S > kvq_max_splits(a.c.stride) || (int64_t)a.S * a.per * kKvqBlock < a.n)
        return (int)hipErrorInvalidValue;
    if (a.rope && (a.n != a.pos0 || (int64_t)a.pos0 + a.m > a.c.stride)) return (int)hipErrorInvalidValue;
    if (a.c.dh == 128) return a.rope ? launch_attn_dh<128, true>(a, c) : launch_attn_dh<128, false>(a, c);
    if (a.c.dh == 64) return a.rope ? launch_attn_dh<64, true>(a, c) : launch_attn_dh<64, false>(a, c);
    return (int)hipErrorInvalidValue;
}

}  // namespace ad
