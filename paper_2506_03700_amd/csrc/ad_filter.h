// Internal interface of the filtered distributions (ad_filter.hip).  Not installed.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "ad_internal.h"

namespace ad {

constexpr int kFilterThreads = 512;
constexpr int kFilterSegIds = 2048;                  // ids per segment, until there are as many segments as a workgroup has threads
constexpr int kFilterMaxSegs = kFilterThreads;
constexpr int kFilterBuckets = 2048;                 // of logits, by their distance from the row's largest
constexpr int kFilterRows = 15;                      // 8 final and 7 draft rows of a verification
constexpr int kFilterList = 4096;                    // ids of the buckets that a boundary lies in, that a row's list has places for
constexpr int kFilterFew = 128;                      // largest top-k that a single kernel takes,
constexpr int kFilterFewList = 8192;                 // if a list of this many has places for that many ids of each segment

// What the kernels leave one another, for one row.
struct FilterRow {
    // from the histogram: the kept ids' boundary by top-p lies in buckets p0 .. p1, that by top-k in bucket bk (none: p0 > p1, bk < 0); ids of buckets
    // before the first of them are kept (as far as top-k and top-p go)
    int p0, p1, bk;
    uint32_t count_k;                                // ids before bucket bk
    uint64_t weight_p, weight_k;                     // weight before bucket p0, bk
    uint64_t weight;                                 // of all ids
    // the outcome
    uint64_t least;                                  // smallest key of a kept id (see key_of)
    uint64_t total;                                  // weight of the kept ids
    float top;                                       // largest logit
    int bad;                                         // no distribution: a logit is no number or plus infinity, or all are minus infinity
};
struct FilterScratch {                               // dev; histograms and arrivals are zero between calls
    uint64_t weight[kFilterRows][kFilterBuckets];
    uint32_t count[kFilterRows][kFilterBuckets];
    float seg_top[kFilterRows][kFilterMaxSegs];
    uint64_t seg_weight[kFilterRows][kFilterMaxSegs];
    uint64_t list[kFilterRows][kFilterFewList];      // per segment: logit's bits, id
    uint32_t arrivals[kFilterRows + 1][32];
    FilterRow row[kFilterRows];
    uint64_t res[2 * kFilterMaxSegs];                // residual, per segment: the bits of the logarithm of its largest weight, its weight
};

struct FilterArgs {
    const float *z0, *z1;                            // dev: rows 0 .. n_first - 1, then the others; [V] each
    int n_first, rows, V, n_seg, seg_ids;
    int places;                                      // of a segment in its row's list
    int top_k;                                       // 0: off
    double inv_t, top_p, min_p;                      // 1 / temperature; 1: off; 0: off
    double min_x;                                    // temperature * log(min_p), near enough
    float bucket_scale;                              // 64 / temperature
    int weight_bits;                                 // weights are multiples of 2^-weight_bits of the largest
    FilterScratch *s;
    // a draw from row 0 (tok_out), or nothing more than the rows' outcomes
    float u;
    int32_t *tok_out;                                // pinned host or dev
    float *prob_out;
    int32_t *n_accept_out;                           // null, or set to 0 (the verification of one row)
    int32_t *done_flag;                              // null, or as in GemmArgs
    int32_t done_seq;
};
struct FilterVerifyArgs {
    FilterArgs f;                                    // z0: final rows [m], z1: draft rows [m - 1]
    int m;
    int32_t draft[8];
    float u_accept[8], u_resample[8], u_final;
    int32_t *n_accept_out, *next_out;
    float *ratio_out;
};

// fills in what follows from V, temperature and the filter's parameters (0: off)
void filter_finish(FilterArgs &, float temperature, int top_k, float top_p, float min_p);
int launch_filter_sample(const FilterArgs &, const LaunchCtx &);
int launch_filter_probs(const FilterArgs &, float *probs, const LaunchCtx &);      // dev [rows][V]
int launch_filter_verify(const FilterVerifyArgs &, const LaunchCtx &);

}  // namespace ad
