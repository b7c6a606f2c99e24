// What the kernels of the gated delta rule are given.
#pragma once

#include <stdint.h>

#include "csb_internal.hpp"

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
    int shortest, longest;              // tokens of the sequences that the kernel serves (others are served by the other one)
    int normalize, step;                // step: a token a sequence
};

constexpr float kDeltaEps = 1e-6f;      // added to the sum of squares that a query or key is divided by the root of

// Chunks of tokens (csb_delta_chunk.cu).  Chunk c of sequence i, whose first token is t, has a record that depends on no length:
// t / kChunk + i + c of tokens / kChunk + sequences; or, where there are more sequences than the call can have long ones (those of
// fewer than kLong tokens have no chunks then), t / kLong for the first chunk, and behind those t / kChunk + c for the others.
constexpr int kLong = 9;
constexpr int kChunk = 32;
struct DeltaChunkArgs {
    int* gave_up;                       // 1 behind a call whose copies did not come within a second, else 0
    uint8_t *keys, *heads;              // [records][k_heads] operands of a chunk, [records][v_heads] its matrices and factors
    long long records, firsts;          // in all; in the second way for first chunks (0: the first way)
    int key_bytes, groups;              // of a key record; CTAs of a head
    int pairs, values_async;            // whether two neighbouring outputs are one access; whether v is copied 16 bytes at a time
    int ranked;                         // whether long sequences go first
    int rows_aligned;                   // whether a lane's values of q and k are whole loads
};

// csb_delta_chunk.cu
int64_t delta_chunk_bytes(int64_t tokens, int64_t sequences, int k_heads, int v_heads, int k_dim, int dtype);
int launch_delta_chunks(int dtype, const DeltaArgs& a, void* workspace, void* stream);

}  // namespace csb
