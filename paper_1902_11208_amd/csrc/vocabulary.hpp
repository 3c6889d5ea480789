// Internal launcher interface of the loss over a vocabulary. All launchers
// enqueue on `stream` and return the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "packed.hpp"

namespace mdl {

constexpr int64_t kMaxVocabularyRows = 1 << 22;  // a tile's rows stay within 32 bits of bytes of each other
constexpr int32_t kMaxVocabulary = 1 << 24, kMaxVocabularyDim = 1 << 16;

struct VocabularyArgs {
    int dtype, dim, vocab;
    int64_t rows;
    RowView x, w;            // [rows][dim], [vocab][dim]
    const int64_t* targets;  // [rows]
    float* losses;           // [rows], forward output
    float* stats;            // [2][rows]: m and s of the sum over the others, 2^m s (forward output, backward input)
    const float* dloss;      // [rows], backward
    void* dx;                // backward outputs
    void* dw;
    void* ws;                // vocabulary_workspace_bytes
};

size_t vocabulary_workspace_bytes(const VocabularyArgs& a, bool backward);
hipError_t launch_vocabulary_fwd(const VocabularyArgs& a, hipStream_t s);
hipError_t launch_vocabulary_bwd(const VocabularyArgs& a, hipStream_t s);

}  // namespace mdl
