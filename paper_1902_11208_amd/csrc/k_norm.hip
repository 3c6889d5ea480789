// Dropout from a counter-based generator, and the root-mean-square norm of a
// residual sum with its gradients and an 8-bit output.
//
// All three are elementwise or one reduction along a row, so HBM bounds them:
// every kernel reads each input once and writes each output once, a row's
// values staying in registers between the reduction and their use.
#include "common.hpp"
#include "philox.hpp"
#include "sequence.hpp"

namespace mdl {
namespace {

// Eight consecutive elements, `valid` of them inside the row (the others read
// as 0 and are not written). WIDE: a whole vector is 16-byte aligned.
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T* p, int valid, float (&v)[8]) {
    if (WIDE && valid == 8) {
        const floatx4 a = St<T>::ld4(p), b = St<T>::ld4(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? St<T>::ld1(p + i) : 0.0f;
    }
}
template <>
__device__ __forceinline__ void load8<bf16_t, true>(const bf16_t* p, int valid, float (&v)[8]) {
    if (valid == 8) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? bf2f(p[i]) : 0.0f;
    }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store8(T* p, int valid, const float (&v)[8]) {
    if (WIDE && valid == 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(p) =
                make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
        } else {
            St<T>::st4(p, floatx4{v[0], v[1], v[2], v[3]});
            St<T>::st4(p + 4, floatx4{v[4], v[5], v[6], v[7]});
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) St<T>::st1(p + i, v[i]);
    }
}

__device__ __forceinline__ uint32_t keep_bits(uint4 u, uint32_t t) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m |= (w[i] & 0xffffu) >= t ? 1u << (2 * i) : 0u;
        m |= (w[i] >> 16) >= t ? 2u << (2 * i) : 0u;
    }
    return m;
}

// Dropout of the elements e .. e + 7 of a tensor: a select, so that a dropped
// element is 0 whatever it held. ALIGNED: e is a multiple of 8, and one block
// of the generator covers them.
template <bool ALIGNED>
__device__ __forceinline__ void drop8(const Drop& d, uint64_t e, float (&v)[8]) {
    if (d.threshold == 0) return;
    uint32_t m = keep_bits(philox(e >> 3, d.call, d.seed), d.threshold);
    if (!ALIGNED && (e & 7)) {
        m |= keep_bits(philox((e >> 3) + 1, d.call, d.seed), d.threshold) << 8;
        m >>= e & 7;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (m >> i) & 1 ? v[i] * d.scale : 0.0f;
}

// ---------------------------------------------------------------------------
// Dropout
// ---------------------------------------------------------------------------
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs a, int64_t vecs) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.rows * vecs) return;
    const int64_t row = i / vecs, c = (i - row * vecs) * 8;
    const int valid = (int)(a.cols - c < 8 ? a.cols - c : 8);
    const uint64_t e = (uint64_t)(row * a.cols + c);
    float v[8];
    load8<T, WIDE>(static_cast<const T*>(a.x) + row * a.x_stride + c, valid, v);
    drop8<WIDE>(a.drop, e, v);
    if (a.residual) {
        float r[8];
        load8<T, WIDE>(static_cast<const T*>(a.residual) + row * a.r_stride + c, valid, r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
    store8<T, WIDE>(static_cast<T*>(a.y) + e, valid, v);
}

// ---------------------------------------------------------------------------
// Norm. LANES threads share a row, each holding NV vectors of 8 of it.
// ---------------------------------------------------------------------------
template <int LANES>
constexpr int block_of() { return LANES <= 256 ? 256 : LANES; }

// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

template <int LANES, bool MAX>
__device__ __forceinline__ float row_reduce(float s, float* lds) {
    auto join = [](float x, float y) { return MAX ? max_nan(x, y) : x + y; };
#pragma unroll
    for (int o = (LANES < 64 ? LANES : 64) / 2; o > 0; o >>= 1) s = join(s, __shfl_xor(s, o));
    if (LANES > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
        __syncthreads();
        s = lds[0];
#pragma unroll
        for (int i = 1; i < LANES / 64; ++i) s = join(s, lds[i]);
    }
    return s;
}

template <typename T, bool WIDE, int LANES, int NV, bool F8>
__global__ __launch_bounds__(block_of<LANES>()) void k_norm_fwd(NormArgs a) {
    __shared__ float lds[LANES > 64 ? LANES / 64 : 1];
    const int64_t row = (int64_t)blockIdx.x * (block_of<LANES>() / LANES) + threadIdx.x / LANES;
    if (row >= a.rows) return;
    const int lane = threadIdx.x % LANES;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* r = a.residual ? static_cast<const T*>(a.residual) + row * a.r_stride : nullptr;
    const int64_t e0 = row * a.cols;
    float v[NV][8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LANES) * 8, valid = min(8, a.cols - c);
        load8<T, WIDE>(x + c, valid, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LANES) * 8, valid = min(8, a.cols - c);
        if (valid > 0) drop8<WIDE>(a.drop, e0 + c, v[i]);
        if (r) {
            float t[8];
            load8<T, WIDE>(r + c, valid, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] += t[j];
        }
        if (a.h) store8<T, WIDE>(static_cast<T*>(a.h) + e0 + c, valid, v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (WIDE || j < valid) sum = fmaf(v[i][j], v[i][j], sum);
    }
    const float rstd = 1.0f / sqrtf(row_reduce<LANES, false>(sum, lds) / (float)a.cols + a.eps);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * LANES) * 8, valid = min(8, a.cols - c);
        float w[8];
        load8<float, WIDE>(a.w + c, valid, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[i][j] = v[i][j] * rstd * w[j];
            if (F8 && j < valid) top = max_nan(fabsf(v[i][j]), top);
        }
        if (!F8) store8<T, WIDE>(static_cast<T*>(a.y) + e0 + c, valid, v[i]);
    }
    if (F8) {
        const float m = row_reduce<LANES, true>(top, lds) / 448.0f;
        const float scale = m < 0x1p-126f ? 0x1p-126f : m;
        if (lane == 0) a.scale[row] = scale;
        const float inv = 1.0f / scale;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * LANES) * 8, valid = min(8, a.cols - c);
            uint32_t q[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * j] * inv, v[i][4 * j + 1] * inv, 0, false);
                p = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * j + 2] * inv, v[i][4 * j + 3] * inv, p, true);
                q[j] = (uint32_t)p;
            }
            uint8_t* y = a.y8 + e0 + c;
            if (WIDE && valid == 8) {
                *reinterpret_cast<uint2*>(y) = make_uint2(q[0], q[1]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < valid) y[j] = (uint8_t)(q[j / 4] >> (8 * (j % 4)));
            }
        }
    }
}

template <typename T, bool WIDE, int LANES, int NV>
__global__ __launch_bounds__(block_of<LANES>()) void k_norm_bwd(NormArgs a, int64_t groups) {
    constexpr int ROWS = block_of<LANES>() / LANES;  // rows of a workgroup at once
    __shared__ float lds[LANES > 64 ? LANES / 64 : 1];
    __shared__ float acc[ROWS > 1 ? ROWS * LANES * NV * 8 : 1];
    const int lane = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    float dw[NV][8] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += groups * ROWS) {
        const int64_t row = r0 + sub;
        if (row >= a.rows) break;  // the whole row's lanes
        const T* h = static_cast<const T*>(a.hin) + row * a.h_stride;
        const int64_t e0 = row * a.cols;
        const float rstd = a.rstd[row];
        float g[NV][8], c[NV][8], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (lane + i * LANES) * 8, valid = min(8, a.cols - col);
            float w[8];
            load8<T, WIDE>(h + col, valid, c[i]);
            load8<T, WIDE>(static_cast<const T*>(a.dy) + e0 + col, valid, g[i]);
            load8<float, WIDE>(a.w + col, valid, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                c[i][j] *= rstd;
                if (WIDE || j < valid) dw[i][j] = fmaf(g[i][j], c[i][j], dw[i][j]);
                g[i][j] *= w[j];
                if (WIDE || j < valid) sum = fmaf(g[i][j], c[i][j], sum);
            }
        }
        const float mean = row_reduce<LANES, false>(sum, lds) / (float)a.cols;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (lane + i * LANES) * 8, valid = min(8, a.cols - col);
            float d[8] = {};
            if (a.dh) load8<T, WIDE>(static_cast<const T*>(a.dh) + e0 + col, valid, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = fmaf(rstd, fmaf(-c[i][j], mean, g[i][j]), d[j]);
            if (a.dres) store8<T, WIDE>(static_cast<T*>(a.dres) + e0 + col, valid, d);
            if (valid > 0) drop8<WIDE>(a.drop, e0 + col, d);
            store8<T, WIDE>(static_cast<T*>(a.dx) + e0 + col, valid, d);
        }
    }
    // the workgroup's share of dw, rows of a workgroup added in order
    float* part = a.part + (int64_t)blockIdx.x * a.cols;
    if (ROWS > 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[(sub * NV + i) * LANES * 8 + lane * 8 + j] = dw[i][j];
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += block_of<LANES>()) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < ROWS; ++k) s += acc[k * NV * LANES * 8 + c];
            part[c] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (lane + i * LANES) * 8;
            store8<float, WIDE>(part + col, min(8, a.cols - col), dw[i]);
        }
    }
}

// dw[c] = sum of the workgroups' shares: 16 slices of them, each in order, added in order.
__global__ __launch_bounds__(1024) void k_norm_dw(int cols, int groups, const float* part, float* dw) {
    __shared__ float lds[16][64];
    const int c = blockIdx.x * 64 + threadIdx.x % 64, slice = threadIdx.x / 64;
    const int lo = (int)((int64_t)groups * slice / 16), hi = (int)((int64_t)groups * (slice + 1) / 16);
    float s = 0.0f;
    if (c < cols)
        for (int g = lo; g < hi; ++g) s += part[(int64_t)g * cols + c];
    lds[slice][threadIdx.x % 64] = s;
    __syncthreads();
    if (slice == 0 && c < cols) {
        s = 0.0f;
        for (int i = 0; i < 16; ++i) s += lds[i][threadIdx.x];
        dw[c] = s;
    }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Calls f with the number of lanes of a row and of vectors a lane holds.
template <typename F>
hipError_t with_shape(int cols, F&& f) {
    const int v = (cols + 7) / 8;
#define SHAPE(L, N) \
    if (v <= L * N) return f(std::integral_constant<int, L>(), std::integral_constant<int, N>());
    SHAPE(8, 1)
    SHAPE(16, 1)
    SHAPE(32, 1)
    SHAPE(64, 1)
    SHAPE(64, 2)
    SHAPE(64, 4)
    SHAPE(256, 2)
    SHAPE(256, 4)
    SHAPE(1024, 2)
    SHAPE(1024, 4)
#undef SHAPE
    return hipErrorInvalidValue;
}

template <typename T, bool WIDE>
hipError_t norm_fwd(const NormArgs& a, hipStream_t s) {
    return with_shape(a.cols, [&](auto L, auto N) {
        constexpr int rows = block_of<L()>() / L();
        const dim3 grid((unsigned)((a.rows + rows - 1) / rows));
        if (a.y8)
            k_norm_fwd<T, WIDE, L(), N(), true><<<grid, block_of<L()>(), 0, s>>>(a);
        else
            k_norm_fwd<T, WIDE, L(), N(), false><<<grid, block_of<L()>(), 0, s>>>(a);
        return hipGetLastError();
    });
}

template <typename T, bool WIDE>
hipError_t norm_bwd(const NormArgs& a, hipStream_t s) {
    const int groups = norm_bwd_groups(a.cols, a.rows);
    hipError_t e = with_shape(a.cols, [&](auto L, auto N) {
        if (groups == 0) return hipSuccess;  // no rows: dw is zero
        k_norm_bwd<T, WIDE, L(), N()><<<groups, block_of<L()>(), 0, s>>>(a, groups);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    k_norm_dw<<<(a.cols + 63) / 64, 1024, 0, s>>>(a.cols, groups, a.part, a.dw);
    return hipGetLastError();
}

}  // namespace

int norm_bwd_groups(int cols, int64_t rows) {
    int per = 1;
    (void)with_shape(cols, [&](auto L, auto) {
        per = block_of<L()>() / L();
        return hipSuccess;
    });
    const int64_t want = (rows + per - 1) / per;
    return (int)(want < 1024 ? want : 1024);
}

hipError_t launch_dropout(const DropoutArgs& in, hipStream_t s) {
    DropoutArgs a = in;
    // contiguous tensors are one row
    if (a.rows > 1 && a.x_stride == a.cols && (!a.residual || a.r_stride == a.cols)) {
        a.cols *= a.rows;
        a.rows = 1;
    }
    const int es = a.dtype ? 2 : 4;
    bool wide = aligned16(a.x) && aligned16(a.y) && (!a.residual || aligned16(a.residual));
    if (a.rows > 1)
        wide = wide && a.cols % 8 == 0 && a.x_stride * es % 16 == 0 && (!a.residual || a.r_stride * es % 16 == 0);
    const int64_t vecs = (a.cols + 7) / 8, blocks = (a.rows * vecs + 255) / 256;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks);
    if (a.dtype)
        wide ? k_dropout<bf16_t, true><<<grid, 256, 0, s>>>(a, vecs) : k_dropout<bf16_t, false><<<grid, 256, 0, s>>>(a, vecs);
    else
        wide ? k_dropout<float, true><<<grid, 256, 0, s>>>(a, vecs) : k_dropout<float, false><<<grid, 256, 0, s>>>(a, vecs);
    return hipGetLastError();
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
    const int es = a.dtype ? 2 : 4;
    const bool wide = a.cols % 8 == 0 && aligned16(a.x) && a.x_stride * es % 16 == 0 &&
                      (!a.residual || (aligned16(a.residual) && a.r_stride * es % 16 == 0)) && aligned16(a.w) &&
                      aligned16(a.h) && aligned16(a.y) && (reinterpret_cast<uintptr_t>(a.y8) & 7) == 0;
    if (a.dtype) return wide ? norm_fwd<bf16_t, true>(a, s) : norm_fwd<bf16_t, false>(a, s);
    return wide ? norm_fwd<float, true>(a, s) : norm_fwd<float, false>(a, s);
}

hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t s) {
    const int es = a.dtype ? 2 : 4;
    const bool wide = a.cols % 8 == 0 && aligned16(a.hin) && a.h_stride * es % 16 == 0 && aligned16(a.w) &&
                      aligned16(a.dy) && aligned16(a.dh) && aligned16(a.dx) && aligned16(a.dres) && aligned16(a.part);
    if (a.dtype) return wide ? norm_bwd<bf16_t, true>(a, s) : norm_bwd<bf16_t, false>(a, s);
    return wide ? norm_bwd<float, true>(a, s) : norm_bwd<float, false>(a, s);
}

}  // namespace mdl
