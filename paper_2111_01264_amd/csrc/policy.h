// Drawing an index from a row of scores: what net.hip and the C entry of policy.hip share.
#pragma once
#include "common.h"

namespace dqn {

struct PolicyArgs {
    const void* scores; int64_t ld; int32_t n;
    const float* temperature; const int32_t* top_k; const float* top_p; const float* min_p;   // per row, each may be null
    const float* u;                    // null: row r draws u at counter (r, kTagPolicy, step) of the generator keyed by seed
    uint64_t seed, step;
    int32_t* index; float* logp;       // logp may be null
};

// Enqueue only; arguments have been checked.
int enqueue_policy_sample(const PolicyArgs& a, int32_t type, int64_t rows, void* work, hipStream_t st);

// The quantised actor's head: rows of 512 hidden values as q8_quantize_rows makes levels of them, their products with fc2's levels [n][512] as q8_linear makes Q rows, into
// q [rows][n], and the draw from them (a.scores is not read; n <= 32).  Where *made != *now (the levels are not those of the present parameters) q and logp are NaN and the index is -1.
int enqueue_policy_q8_head(const PolicyArgs& a, const float* hidden, const int8_t* w, const float* scales, const float* bias, const uint64_t* made, const uint64_t* now,
                           float* q, int64_t rows, hipStream_t st);

}  // namespace dqn
