// Internal launcher interface of the group norm. All launchers enqueue on
// `stream` and return the hipError_t of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "packed.hpp"

namespace mdl {

constexpr int kMaxGroupChannels = 4096;  // a workgroup holds whole groups of a row

struct GroupNormArgs {
    Packed seqs;
    int channels, groups, dtype, act;  // act: mdlstm_activation
    float eps;
    const float* w;
    const float* b;
    RowView x, dy;     // dy: backward only
    void* y;           // forward output
    float* mean;       // [n][groups], forward outputs and backward inputs
    float* rstd;
    void* dx;          // backward outputs
    float* dw;
    float* db;
    void* ws;          // groupnorm_workspace_bytes
    // set by the launchers: channels of a workgroup (whole groups), blocks of them in a row, lanes of a row, tokens
    // that a workgroup takes at once, workgroups along the slots, long sequences' sums of each slot
    // [slots][groups][2], what dw and db add up from [parts][2][channels], group means of long sequences [n][groups][2]
    int per, block, blocks, lanes, held;  // per: channels of a group, held: tokens
    int64_t parts;
    float* sums;
    float* part;
    float* means;
};

size_t groupnorm_workspace_bytes(const GroupNormArgs& a, bool backward);
hipError_t launch_groupnorm_fwd(const GroupNormArgs& a, hipStream_t s);
hipError_t launch_groupnorm_bwd(const GroupNormArgs& a, hipStream_t s);

}  // namespace mdl
