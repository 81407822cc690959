// Internal interface of the 8-bit cache's kernels (ad_kvq.hip).  Not installed.
//
// Storage of one layer, stride = max_pos rounded up to 64:
//   K codes  [kv head][position][head_dim]                 one byte each (e4m3)
//   V codes  [kv head][position / 64][head_dim][64 positions]
//   K scales [kv head][position], V scales likewise        one byte each: the exponent e of 2^e, plus 127
// The scale is a token's and kv head's own, so that an entry depends on nothing but the value stored there: not on the
// tokens that were appended in the same call, nor on those that a rollback took back.  A power of two costs a code of three mantissa bits
// nothing but range, and makes every stored value exact in bf16, and every code exact in fp16.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "ad_internal.h"

namespace ad {

constexpr int kKvqBlock = 64;            // positions per block of V, and per step of the attention kernel
constexpr int kKvqMaxSplits = 512;       // most work items of a kv head

struct KvqCache {
    uint8_t *Kc, *Vc, *Ks, *Vs;          // of one layer
    int stride, Hkv, dh;
};

// bytes of one layer
inline size_t kvq_layer_bytes(int64_t Hkv, int64_t stride, int64_t dh) { return ((size_t)(2 * Hkv * stride * (dh + 1)) + 255) / 256 * 256; }
inline KvqCache kvq_cache(void *layer, int stride, int Hkv, int dh) {
    KvqCache c;
    const size_t codes = (size_t)Hkv * stride * dh, scales = (size_t)Hkv * stride;
    c.Kc = (uint8_t *)layer;
    c.Vc = c.Kc + codes;
    c.Ks = c.Vc + codes;
    c.Vs = c.Ks + scales;
    c.stride = stride; c.Hkv = Hkv; c.dh = dh;
    return c;
}
// most partials that an attention call over max_pos positions leaves per query row (also the room that a cache has for them)
inline int kvq_max_splits(int max_pos) {
    const int n = (max_pos + kKvqBlock - 1) / kKvqBlock;
    return n < kKvqMaxSplits ? n : kKvqMaxSplits;
}

struct KvqRows {                         // fp32 rows of n tokens at positions pos0 ..: [n][ld], a token's kv heads next to each other
    KvqCache c;
    const float *k, *v;
    float *k_out, *v_out;                // (read-out)
    int64_t ld;
    int n, pos0;
};
struct KvqExpand {                       // the cache's values in bf16, in the layout of a 16-bit cache of the same stride
    KvqCache c;
    uint16_t *K, *V;
    int n;                               // positions 0 .. n - 1; behind them zeros up to the next multiple of 64
};
struct KvqAttn {
    KvqCache c;
    const float *q;                      // [m][ld_q] rotated queries
    int ld_q;
    int m, Hq, G, R;                     // tokens, query heads, those per kv head, query rows per kv head
    int see[8];                          // last position that token t's queries see
    // a layer step (rope not null): q is the step's q, k, v as they come from their projection, [m][ld_q], the rows' positions are pos0 .. pos0 + m - 1;
    // queries and keys are rotated, keys and values stored, and attended to
    const float *rope;                   // rows pos0 .. of the cache's rotary table
    int pos0;
    int n, n_all;                        // cached positions (before the call) that some row sees, that all rows see
    int S, per, waves, tiles;            // work items per kv head, blocks of 64 positions and wavefronts per item, tiles of 16 query rows per workgroup
    unsigned mul_S, mul_G, mul_R;
    float scale;                         // of the scores, in powers of two: log2(e) / sqrt(head_dim)
    float *part;                         // [Hkv][S][R][dh + 2]
    float *out;                          // fp32 rows [m][Hq * dh], or null: packed for the Wo projection
    void *Bo;
    int Bo_KT, f16;
};

int launch_kvq_store(const KvqRows &, const LaunchCtx &);
int launch_kvq_read(const KvqRows &, const LaunchCtx &);
int launch_kvq_expand(const KvqExpand &, const LaunchCtx &);
// fills in what follows from the other fields (G, R, n, n_all, S, per, multipliers), for a grid of n_wg compute units
void kvq_attn_finish(KvqAttn &, int n_wg);
int launch_kvq_attn(const KvqAttn &, const LaunchCtx &);

}  // namespace ad
