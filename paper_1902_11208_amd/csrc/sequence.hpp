// Internal launcher interface of the sequence operators (attention with decay,
// residual norm, dropout). All launchers enqueue on `stream` and return the
// hipError_t of the launch.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mdl {

// A grid of at least `blocks` workgroups. The runtime takes less than 2^32
// threads along x, so more come as rows of a multiple of 8 workgroups, which
// keeps a workgroup's XCD its index modulo 8. False beyond 65535 rows.
inline bool grid_of(int64_t blocks, int threads, dim3& grid) {
    const int64_t most = (0xffffffffll / threads) & ~7ll;
    const int64_t rows = blocks > most ? (blocks + most - 1) / most : 1;
    if (rows > 65535) return false;
    grid = dim3((unsigned)(rows > 1 ? ((blocks + rows - 1) / rows + 7) & ~7ll : blocks), (unsigned)rows);
    return true;
}
__device__ __forceinline__ int64_t block_index() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// A token tensor as a scan reads it: element (t, h, i) at
// p[t * token_stride + (h / group) * head_stride + i], i < dim.
struct HeadView {
    const void* p;
    int64_t token_stride, head_stride;
    int group, dim;
};

// One scan over the packed sequences, for every head (g = exp(-rate)):
//     S_t = g S_{t-1} + in_scale k_t v_t^T      out_t = out_scale q_t^T S_t
// forward in time, or (reverse) from each sequence's last token to its first,
// where the state a sequence starts from meets its first scanned token without
// decay and the state it leaves has decayed once more: the recurrence of the
// adjoint. The layer's forward pass and its three gradients are all this scan:
//     o   q = q,  k = k,  v = v    forward      out_scale = scale
//     dq  q = do, k = v,  v = k    forward      out_scale = scale, state transposed
//     dk  q = v,  k = do, v = q    reverse      in_scale = scale,  state transposed
//     dv  q = k,  k = q,  v = do   reverse      in_scale = scale
struct ScanRole {
    HeadView q, k, v;
    void* out;             // [tokens][heads][v.dim], storage type, or fp32 where out_f32
    const float* state;    // [n][heads][q.dim][v.dim], transposed where state_t, or NULL
    float* final_state;    // the same, or NULL
    float out_scale, in_scale;
    int reverse, state_t, out_f32;
};

struct ScanArgs {
    int n, heads, dtype;
    int64_t tokens, longest;
    const int64_t* offsets;
    const int32_t* order;  // sequences in the order they are started, or NULL
    const float* rates;
    int n_roles;
    ScanRole role[3];
    int group;             // query heads of a key head
    void* ws;              // scan_workspace_bytes
    // set by launch_scan: tokens of a segment (0: whole sequences), slots of
    // segments or sequences, heads that one XCD takes together, the states between
    // segments [role][head][slot][q.dim][v.dim]
    int64_t seg, slots;
    int together;
    float* states;
};

size_t scan_workspace_bytes(const ScanArgs& a);
hipError_t launch_scan(const ScanArgs& a, hipStream_t s);

// dst[t][j][i] = sum over c < group of src[t][j * group + c][i] in that order, i < dim, rounded to the storage type.
hipError_t launch_sum_heads(int64_t tokens, int kv_heads, int group, int dim, int dtype, const float* src, void* dst,
                            hipStream_t s);

struct StepArgs {
    int n, heads, dtype;
    HeadView q, k, v;
    const float* rates;
    float* state;
    int64_t slots;
    const int32_t* slot;   // [n] or NULL
    void* out;
    float scale;
};
hipError_t launch_step(const StepArgs& a, hipStream_t s);

// --- dropout, residual norm --------------------------------------------------
// drop: threshold on 16 bits, 0 (keep all) to 65536 (drop all).
struct Drop {
    uint64_t seed, call;
    uint32_t threshold;
    float scale;
};

struct DropoutArgs {
    int dtype;
    int64_t rows, cols, x_stride, r_stride;
    const void* x;
    const void* residual;  // or NULL
    void* y;
    Drop drop;
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);

struct NormArgs {
    int cols, dtype;
    int64_t rows;
    float eps;
    Drop drop;
    const float* w;
    // forward
    const void* x;
    const void* residual;  // or NULL
    int64_t x_stride, r_stride;
    void* h;               // or NULL
    void* y;               // or NULL with y8
    uint8_t* y8;
    float* scale;
    float* rstd;           // forward output (or NULL), backward input
    // backward
    const void* hin;
    int64_t h_stride;
    const void* dy;
    const void* dh;        // or NULL
    void* dx;
    void* dres;            // or NULL
    float* part;           // [norm_bwd_groups][cols]
    float* dw;
};
constexpr int MAX_NORM_COLS = 32768;
int norm_bwd_groups(int cols, int dtype, int64_t rows);
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s);

}  // namespace mdl
