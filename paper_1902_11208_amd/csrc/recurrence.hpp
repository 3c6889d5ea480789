// Internal launcher interface of the gated recurrence. All launchers enqueue on
// `stream` and return the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "packed.hpp"

namespace mdl {

constexpr int kRecurrenceTile = 128;  // tokens of a tile; a state is kept at every tile's start but the first

struct RecurrenceArgs {
    Packed seqs;
    int channels, dtype, sigmoid;
    RowView z, x, dh;      // dh: backward only
    const float* state;    // [n][channels] or NULL
    const float* dfinal;   // backward: gradient of the final states, or NULL
    float* marks;          // [tokens / kRecurrenceTile + 1][channels]: states at the tiles' starts; forward: or NULL
    void* h;               // forward output
    float* final_state;    // forward output or NULL
    void* dz;              // backward outputs
    void* dx;
    float* dstate;         // or NULL
    void* ws;              // recurrence_workspace_bytes
    // set by the launchers (as seqs.seg and seqs.slots): edges between segments at most, the A and B of the segments
    // before them (backward: behind them) [2][edges][channels], the states that meet the edges [edges][channels]
    int64_t edges;
    float* sums;
    float* starts;
};

size_t recurrence_workspace_bytes(const RecurrenceArgs& a);
hipError_t launch_recurrence_fwd(const RecurrenceArgs& a, hipStream_t s);
hipError_t launch_recurrence_bwd(const RecurrenceArgs& a, hipStream_t s);

struct AdvanceArgs {
    int n, channels, dtype, sigmoid;
    RowView z, x;
    float* state;
    int64_t slots;
    const int32_t* slot;  // [n] or NULL
    void* out;
};
hipError_t launch_advance(const AdvanceArgs& a, hipStream_t s);

}  // namespace mdl
