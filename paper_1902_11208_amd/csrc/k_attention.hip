// Linear attention with a decay for each head: the scan over packed sequences,
// the sum over shared heads, and the single-token step.
#include "common.hpp"
#include "sequence.hpp"

namespace mdl {
namespace {

template <typename T>
__device__ __forceinline__ const T* at(const HeadView& v, int64_t t, int head) {
    return static_cast<const T*>(v.p) + t * v.token_stride + (int64_t)(head / v.group) * v.head_stride;
}

// First token and length of sequence i, cut to the tensors and to `longest`.
__device__ __forceinline__ void sequence(const int64_t* offsets, int i, int64_t tokens, int64_t longest, int64_t& t0,
                                         int64_t& len) {
    t0 = min(max(offsets[i], (int64_t)0), tokens);
    const int64_t t1 = min(max(offsets[i + 1], t0), tokens);
    len = min(t1 - t0, longest);
}

// One workgroup per (sequence, head), a thread per column of the state, which
// lies in LDS; one token at a time.
template <typename T>
__global__ __launch_bounds__(128) void k_scan(ScanArgs a) {
    extern __shared__ float lds[];
    const ScanRole& R = a.role[blockIdx.z];
    const int seq = blockIdx.x, head = blockIdx.y, c = threadIdx.x, dk = R.q.dim, dv = R.v.dim;
    float* S = lds;  // [dk][dv]
    float* q = S + dk * dv;
    float* k = q + dk;
    int64_t t0, len;
    sequence(a.offsets, seq, a.tokens, a.longest, t0, len);
    const int64_t so = ((int64_t)seq * a.heads + head) * dk * dv;
    if (c < dv)
        for (int i = 0; i < dk; ++i) S[i * dv + c] = R.state ? R.state[so + (R.state_t ? c * dk + i : i * dv + c)] : 0.0f;
    const float g = expf(-a.rates[head]);
    for (int64_t j = 0; j < len; ++j) {
        const int64_t t = t0 + (R.reverse ? len - 1 - j : j);
        __syncthreads();
        if (c < dk) {
            q[c] = St<T>::ld1(at<T>(R.q, t, head) + c);
            k[c] = St<T>::ld1(at<T>(R.k, t, head) + c);
        }
        __syncthreads();
        if (c < dv) {
            const float v = St<T>::ld1(at<T>(R.v, t, head) + c) * R.in_scale, f = R.reverse && j == 0 ? 1.0f : g;
            float o = 0.0f;
            for (int i = 0; i < dk; ++i) {
                const float s = fmaf(k[i], v, S[i * dv + c] * f);
                S[i * dv + c] = s;
                o = fmaf(q[i], s, o);
            }
            const int64_t oo = (t * a.heads + head) * dv + c;
            if (R.out_f32)
                static_cast<float*>(R.out)[oo] = o * R.out_scale;
            else
                St<T>::st1(static_cast<T*>(R.out) + oo, o * R.out_scale);
        }
    }
    if (R.final_state && c < dv)
        for (int i = 0; i < dk; ++i)
            R.final_state[so + (R.state_t ? c * dk + i : i * dv + c)] = S[i * dv + c] * (R.reverse && len > 0 ? g : 1.0f);
}

template <typename T>
__global__ __launch_bounds__(256) void k_sum_heads(int64_t n, int group, int dim, const float* src, T* dst) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;  // (token, kv head, element)
    if (i >= n) return;
    const int64_t th = i / dim;
    const float* p = src + th * group * dim + (i - th * dim);
    float s = 0.0f;
    for (int c = 0; c < group; ++c) s += p[(int64_t)c * dim];
    St<T>::st1(dst + i, s);
}

template <typename T>
__global__ __launch_bounds__(128) void k_step(StepArgs a) {
    __shared__ float q[128], k[128];
    const int row = blockIdx.x, head = blockIdx.y, c = threadIdx.x, dk = a.q.dim, dv = a.v.dim;
    const int64_t slot = a.slot ? a.slot[row] : row;
    const int64_t oo = ((int64_t)row * a.heads + head) * dv + c;
    if (slot < 0 || slot >= a.slots) {
        if (c < dv) St<T>::st1(static_cast<T*>(a.out) + oo, 0.0f);
        return;
    }
    if (c < dk) {
        q[c] = St<T>::ld1(at<T>(a.q, row, head) + c);
        k[c] = St<T>::ld1(at<T>(a.k, row, head) + c);
    }
    __syncthreads();
    if (c >= dv) return;
    const float g = expf(-a.rates[head]), v = St<T>::ld1(at<T>(a.v, row, head) + c);
    float* S = a.state + (slot * a.heads + head) * dk * dv + c;
    float o = 0.0f;
    for (int i = 0; i < dk; ++i) {
        const float s = fmaf(k[i], v, S[(int64_t)i * dv] * g);
        S[(int64_t)i * dv] = s;
        o = fmaf(q[i], s, o);
    }
    St<T>::st1(static_cast<T*>(a.out) + oo, o * a.scale);
}

}  // namespace

size_t scan_workspace_bytes(const ScanArgs&) { return 16; }

hipError_t launch_scan(const ScanArgs& a, hipStream_t s) {
    int dk = 0, dv = 0;
    for (int r = 0; r < a.n_roles; ++r) dk = std::max(dk, a.role[r].q.dim), dv = std::max(dv, a.role[r].v.dim);
    const dim3 grid(a.n, a.heads, a.n_roles);
    const size_t lds = (size_t)(dk * dv + 2 * dk) * 4;
    auto f = a.dtype ? k_scan<bf16_t> : k_scan<float>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)lds);
    if (e != hipSuccess) return e;
    f<<<grid, 128, lds, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_sum_heads(int64_t tokens, int kv_heads, int group, int dim, int dtype, const float* src, void* dst,
                            hipStream_t s) {
    const int64_t n = tokens * kv_heads * dim, blocks = (n + 255) / 256;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    if (dtype)
        k_sum_heads<<<(unsigned)blocks, 256, 0, s>>>(n, group, dim, src, static_cast<bf16_t*>(dst));
    else
        k_sum_heads<<<(unsigned)blocks, 256, 0, s>>>(n, group, dim, src, static_cast<float*>(dst));
    return hipGetLastError();
}

hipError_t launch_step(const StepArgs& a, hipStream_t s) {
    const dim3 grid(a.n, a.heads);
    if (a.dtype)
        k_step<bf16_t><<<grid, 128, 0, s>>>(a);
    else
        k_step<float><<<grid, 128, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace mdl
