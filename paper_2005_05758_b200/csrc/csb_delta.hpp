// What the kernels of the gated delta rule are given.
#pragma once

#include <stdint.h>

namespace csb {

struct DeltaArgs {
    const void *q, *k, *v;
    const float *g, *beta;
    void* o;
    float* state;                       // [slots][v_heads][k_dim][v_dim], or NULL
    const int32_t *seq_begin, *slot;    // [sequences + 1] or NULL (one sequence of all tokens); [sequences] or NULL
    const uint8_t* fresh;
    long long tokens, slots, ldq, ldk, ldv, ldg, ldb, ldo;
    int sequences, k_heads, v_heads, k_dim, v_dim;
    float scale;
    int normalize, step;                // step: a token a sequence
};

constexpr float kDeltaEps = 1e-6f;      // added to the sum of squares that a query or key is divided by the root of

}  // namespace csb
