// Dropout from a counter-based generator, and the root-mean-square norm of a
// residual sum with its gradients and an 8-bit output.
//
// All three are elementwise or one reduction along a row, so HBM bounds them:
// every kernel reads each input once and writes each output once, a row's
// values staying in registers between the reduction and their use. Measured:
// dropout with a residual, 48000 x 2048 bf16, 99 us (590 MB, 6.0 TB/s); norm with
// residual and dropout, 96000 x 512 bf16, 66 us forward (6.0 TB/s) and 100 us
// backward (4.9 TB/s) with 4 us for dw's shares; 8-bit output, 16383 x 5000 bf16,
// 117 us (4.9 TB/s). A block of the generator (ten rounds of two 32-bit products)
// serves eight elements, 16 bits each, so it stays below the memory's time.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "philox.hpp"
#include "sequence.hpp"

namespace mdl {
namespace {

// Eight consecutive elements, `valid` of them inside the row (the others read
// as 0 and are not written). WIDE: a whole vector is 16-byte aligned; else it is
// moved by the same 16-byte instructions at its element's alignment (rows of 100
// bf16, 60 million elements: 182 us forward, 330 us with single elements).
template <typename V, bool WIDE>
struct Vec;
template <typename V>
struct Vec<V, true> {
    typedef V type;
};
template <typename V>
struct Vec<V, false> {
    typedef V type __attribute__((aligned(1)));
};
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T* p, int valid, float (&v)[8]) {
    if (valid == 8) {
        if constexpr (sizeof(T) == 2) {
            const u32x4 u = *reinterpret_cast<const typename Vec<u32x4, WIDE>::type*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(u[i] << 16);
                v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
        } else {
            typedef typename Vec<floatx4, WIDE>::type V;
            const floatx4 a = *reinterpret_cast<const V*>(p), b = *reinterpret_cast<const V*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? St<T>::ld1(p + i) : 0.0f;
    }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store8(T* p, int valid, const float (&v)[8]) {
    if (valid == 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<typename Vec<u32x4, WIDE>::type*>(p) =
                u32x4{f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])};
        } else {
            typedef typename Vec<floatx4, WIDE>::type V;
            *reinterpret_cast<V*>(p) = floatx4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<V*>(p + 4) = floatx4{v[4], v[5], v[6], v[7]};
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
    const int64_t i = block_index() * 256 + threadIdx.x;
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
// Norm. LANES threads share a row, each holding NV vectors of 8 of it: up to a
// wave, with several rows in a workgroup of 256, or (LANES 0) a workgroup of as
// many waves as the row needs (with_shape below).
// ---------------------------------------------------------------------------
// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

template <int LANES, bool MAX>
__device__ __forceinline__ float row_reduce(float s, float* lds) {
    auto join = [](float x, float y) { return MAX ? max_nan(x, y) : x + y; };
#pragma unroll
    for (int o = (LANES ? LANES : 64) / 2; o > 0; o >>= 1) s = join(s, __shfl_xor(s, o));
    if (LANES == 0) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
        __syncthreads();
        s = lds[0];
        for (int i = 1; i < (int)blockDim.x / 64; ++i) s = join(s, lds[i]);
    }
    return s;
}

template <int LANES>
constexpr int threads_of() { return LANES ? 256 : 1024; }

template <typename T, bool WIDE, int LANES, int NV, bool F8>
__global__ __launch_bounds__(threads_of<LANES>()) void k_norm_fwd(NormArgs a) {
    __shared__ float lds[16];
    const int lanes = LANES ? LANES : blockDim.x;
    const int64_t row = LANES ? block_index() * (256 / lanes) + threadIdx.x / lanes : block_index();
    if (row >= a.rows) return;
    const int lane = LANES ? threadIdx.x % lanes : threadIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* r = a.residual ? static_cast<const T*>(a.residual) + row * a.r_stride : nullptr;
    const int64_t e0 = row * a.cols;
    float v[NV][8], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * lanes) * 8, valid = min(8, a.cols - c);
        load8<T, WIDE>(x + c, valid, v[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (lane + i * lanes) * 8, valid = min(8, a.cols - c);
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
        const int c = (lane + i * lanes) * 8, valid = min(8, a.cols - c);
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
        // The codes are those of the rounded quotient v / scale. From the rounded
        // reciprocal, one correction of the product gives it (Markstein 1990): 120
        // us for the 82 million elements of 16383 x 5000, 125 with divisions.
        const float inv = 1.0f / scale;
        const bool ordinary = scale >= 0x1p-100f && scale <= 0x1p100f;  // no step of it leaves fp32's normal range
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (lane + i * lanes) * 8, valid = min(8, a.cols - c);
            if (ordinary) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float q = v[i][j] * inv;
                    v[i][j] = fmaf(fmaf(-q, scale, v[i][j]), inv, q);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] /= scale;
            }
            uint32_t q[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * j], v[i][4 * j + 1], 0, false);
                p = __builtin_amdgcn_cvt_pk_fp8_f32(v[i][4 * j + 2], v[i][4 * j + 3], p, true);
                q[j] = (uint32_t)p;
            }
            uint8_t* y = a.y8 + e0 + c;
            if (valid == 8) {
                typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                *reinterpret_cast<typename Vec<u32x2, WIDE>::type*>(y) = u32x2{q[0], q[1]};
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < valid) y[j] = (uint8_t)(q[j / 4] >> (8 * (j % 4)));
            }
        }
    }
}

template <typename T, bool WIDE, int LANES, int NV>
__global__ __launch_bounds__(threads_of<LANES>()) void k_norm_bwd(NormArgs a, int64_t groups) {
    constexpr int ROWS = LANES ? 256 / LANES : 1;  // rows of a workgroup at once
    __shared__ float lds[16];
    __shared__ float acc[ROWS > 1 ? ROWS * LANES * NV * 8 : 1];
    const int lanes = LANES ? LANES : blockDim.x;
    const int lane = LANES ? threadIdx.x % lanes : threadIdx.x, sub = LANES ? threadIdx.x / lanes : 0;
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
            const int col = (lane + i * lanes) * 8, valid = min(8, a.cols - col);
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
            const int col = (lane + i * lanes) * 8, valid = min(8, a.cols - col);
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
        for (int c = threadIdx.x; c < a.cols; c += 256) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < ROWS; ++k) s += acc[k * NV * LANES * 8 + c];
            part[c] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (lane + i * lanes) * 8;
            store8<float, WIDE>(part + col, min(8, a.cols - col), dw[i]);
        }
    }
}

// dw[c] = sum of the workgroups' shares: 64 slices of them, each in order, added
// in order. 16 columns a workgroup, eight loads of a thread in flight.
__global__ __launch_bounds__(1024) void k_norm_dw(int cols, int groups, const float* part, float* dw) {
    __shared__ float lds[64][17];
    const int c = blockIdx.x * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
    const int lo = (int)((int64_t)groups * slice / 64), hi = (int)((int64_t)groups * (slice + 1) / 64);
    float s = 0.0f;
    if (c < cols)
        for (int g = lo; g < hi; g += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = g + i < hi ? part[(int64_t)(g + i) * cols + c] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
    lds[slice][threadIdx.x % 16] = s;
    __syncthreads();
    if (threadIdx.x < 64) {  // four threads a column, a quarter of the slices each
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += lds[threadIdx.x / 16 * 16 + i][threadIdx.x % 16];
        const float s1 = __shfl(s, threadIdx.x % 16 + 16), s2 = __shfl(s, threadIdx.x % 16 + 32), s3 = __shfl(s, threadIdx.x % 16 + 48);
        if (threadIdx.x < 16 && c < cols) dw[c] = ((s + s1) + s2) + s3;
    }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Calls f with the lanes of a row (0: a workgroup of `threads`), the vectors a
// lane holds and the threads of a workgroup. Measured at 60 million elements:
// two bytes an element leave a lane 16 bytes of a tensor a vector, and then two
// vectors in one wave beat two waves (rows of 1000: backward 125 against 143 us;
// four bytes: forward 113 against 92), and a forward pass wants few waves on a
// row's barriers: four up to 2048 elements, then two vectors (8-bit output, rows of
// 4096: 79 against 86 us; backward 4096: 184 against 133), from 4097 to 6144 three in
// four waves (5000: 89 with them, 116 with ten waves), and beyond again two, in
// seven or eight waves (8192: 81, with four vectors in four waves 86; 7168: 86
// against 90).
template <typename F>
hipError_t with_shape(int cols, int dtype, bool forward, F&& f) {
    const int v = (cols + 7) / 8, waves = (v + 63) / 64;
    const bool half = dtype == 1;
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 0> block;
    if (v <= 8) return f(std::integral_constant<int, 8>(), one, 256);
    if (v <= 16) return f(std::integral_constant<int, 16>(), one, 256);
    if (v <= 32) return f(std::integral_constant<int, 32>(), one, 256);
    if (v <= 64) return f(std::integral_constant<int, 64>(), one, 256);
    if (v <= 128 && half) return f(std::integral_constant<int, 64>(), two, 256);
    if (waves <= (half && forward ? 4 : 16)) return f(block, one, waves * 64);
    if (half && forward && waves > 8 && waves <= 12) return f(block, std::integral_constant<int, 3>(), 256);
    if (waves <= 32) return f(block, two, (waves + 1) / 2 * 64);
    if (waves <= 64) return f(block, std::integral_constant<int, 4>(), (waves + 3) / 4 * 64);
    return hipErrorInvalidValue;
}

template <typename T, bool WIDE>
hipError_t norm_fwd(const NormArgs& a, hipStream_t s) {
    return with_shape(a.cols, a.dtype, true, [&](auto L, auto N, int threads) {
        constexpr int rows = L() ? 256 / (L() ? L() : 1) : 1;
        dim3 grid;
        if (!grid_of((a.rows + rows - 1) / rows, threads, grid)) return hipErrorInvalidValue;
        if (a.y8)
            k_norm_fwd<T, WIDE, L(), N(), true><<<grid, threads, 0, s>>>(a);
        else
            k_norm_fwd<T, WIDE, L(), N(), false><<<grid, threads, 0, s>>>(a);
        return hipGetLastError();
    });
}

template <typename T, bool WIDE>
hipError_t norm_bwd(const NormArgs& a, hipStream_t s) {
    const int groups = norm_bwd_groups(a.cols, a.dtype, a.rows);
    hipError_t e = with_shape(a.cols, a.dtype, false, [&](auto L, auto N, int threads) {
        if (groups == 0) return hipSuccess;  // no rows: dw is zero
        k_norm_bwd<T, WIDE, L(), N()><<<groups, threads, 0, s>>>(a, groups);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    k_norm_dw<<<(a.cols + 15) / 16, 1024, 0, s>>>(a.cols, groups, a.part, a.dw);
    return hipGetLastError();
}

}  // namespace

// Workgroups of a backward call: 16 waves a CU, each with a share of dw.
int norm_bwd_groups(int cols, int dtype, int64_t rows) {
    int64_t want = 1;
    (void)with_shape(cols, dtype, false, [&](auto L, auto, int threads) {
        const int64_t per = L() ? 256 / (L() ? L() : 1) : 1;
        want = std::min<int64_t>((rows + per - 1) / per, 4096 / (threads / 64));
        return hipSuccess;
    });
    return (int)want;
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
    const int64_t vecs = (a.cols + 7) / 8;
    dim3 grid;
    if (!grid_of((a.rows * vecs + 255) / 256, 256, grid)) return hipErrorInvalidValue;
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
