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

// Enqueues only; arguments have been checked.
int enqueue_policy_sample(const PolicyArgs& a, int32_t type, int64_t rows, void* work, hipStream_t st);

}  // namespace dqn
