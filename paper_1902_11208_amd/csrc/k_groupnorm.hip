// Group norm with an activation over packed sequences, channels last: mean and
// variance over the tokens of a sequence and the channels of a group,
//     c = (x - mean) rstd        u = c w + b        y = act(u)
// and its gradients, with e = dy act'(u) and g = e w,
//     dx = rstd (g - mean(g) - c mean(g c))    dw = sum of e c    db = sum of e.
//
// HBM bounds it, so a workgroup keeps the tokens of a sequence in registers
// where they fit (a block of whole groups, `Hold` vectors of four channels a
// thread) between the sums and their use, and each input is read once. Longer
// sequences are cut into segments of as many tokens: a pass for the segments'
// sums, one that joins them in order, and a pass that reads the segments again.
//
// The variance is the mean of squared distances from the mean, found in a second
// look at the registers (a difference of sums of squares would lose it beside a
// large mean); that look also corrects the mean's own rounding. Segments are
// joined from their means and squared distances in 64 bits. Sums are taken in a
// fixed order.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "groupnorm.hpp"
#include "mdlstm.h"
#include "sequence.hpp"

namespace mdl {
namespace {

constexpr int V = 4;  // channels of a vector

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <typename T>
struct RawOf {
    typedef u32x4 type;
    typedef u32x4 anywhere __attribute__((aligned(1)));
};
template <>
struct RawOf<bf16_t> {
    typedef u32x2 type;
    typedef u32x2 anywhere __attribute__((aligned(1)));
};
template <typename T>
using Raw = typename RawOf<T>::type;

// `valid` of the four channels at p; the others read as 0. WIDE: p is aligned to
// the vector and all four are valid; else whole vectors are moved by the same
// instruction at their elements' alignment.
template <typename T, bool WIDE>
__device__ __forceinline__ Raw<T> load_raw(const T* p, int valid) {
    if constexpr (WIDE) return *reinterpret_cast<const Raw<T>*>(p);
    if (valid == V) return *reinterpret_cast<const typename RawOf<T>::anywhere*>(p);
    if constexpr (sizeof(T) == 4) {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
        return u32x4{valid > 0 ? q[0] : 0u, valid > 1 ? q[1] : 0u, valid > 2 ? q[2] : 0u, 0u};
    } else {
        return u32x2{(valid > 0 ? (uint32_t)p[0] : 0u) | (valid > 1 ? (uint32_t)p[1] << 16 : 0u), valid > 2 ? (uint32_t)p[2] : 0u};
    }
}
__device__ __forceinline__ void unpack(u32x4 r, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void unpack(u32x2 r, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[2 * i] = __uint_as_float(r[i] << 16);
        v[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store_vec(T* p, int valid, const float (&v)[V]) {
    Raw<T> r;
    if constexpr (sizeof(T) == 4)
        r = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    else
        r = u32x2{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
    if constexpr (WIDE) {
        *reinterpret_cast<Raw<T>*>(p) = r;
    } else if (valid == V) {
        *reinterpret_cast<typename RawOf<T>::anywhere*>(p) = r;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < valid) St<T>::st1(p + i, v[i]);
    }
}

// How a pass holds a sequence: threads of a workgroup at most, and the vectors of x
// that each holds (backward with the fp32 numbers e beside them).
struct Forward {
    static constexpr bool BACKWARD = false;
    static constexpr int THREADS = 1024, BYTES = 160;
};
struct Backward {
    static constexpr bool BACKWARD = true;
    static constexpr int THREADS = 512, BYTES = 160;
};
struct BackwardOfWideRows {  // a row of a group needs more than 512 threads
    static constexpr bool BACKWARD = true;
    static constexpr int THREADS = 1024, BYTES = 64;
};
template <typename T, typename H>
constexpr int Hold = H::BYTES / (V * sizeof(T));

// EXACT (fp32 storage): to an ulp or two; else the product with log2(e) is rounded,
// |u| 2^-24 off, far below a bf16 u's own rounding.
template <bool EXACT>
__device__ __forceinline__ float sigmoid(float u) {
    constexpr float HIGH = -1.44269502162933349609375f, LOW = -1.925963033500011e-08f, LN2 = 0.693147180559945309f;
    const float t = u * HIGH;
    float e = __builtin_amdgcn_exp2f(t);
    if (EXACT && fabsf(t) < 120.0f) e = fmaf(e, LN2 * fmaf(u, LOW, fmaf(u, HIGH, -t)), e);
    const float d = 1.0f + e;
    float r = __builtin_amdgcn_rcpf(d);
    if (EXACT && d < 0x1p120f) r = fmaf(fmaf(-d, r, 1.0f), r, r);
    return r;
}
template <int ACT, bool EXACT>
__device__ __forceinline__ float activate(float u) {
    if (ACT == MDLSTM_SILU) return u * sigmoid<EXACT>(u);
    if (ACT == MDLSTM_RELU) return u < 0.0f ? 0.0f : u;  // a NaN stays one
    return u;
}
// dy act'(u)
template <int ACT, bool EXACT>
__device__ __forceinline__ float activate_back(float dy, float u) {
    if (ACT == MDLSTM_SILU) {
        const float s = sigmoid<EXACT>(u);
        return dy * (s * fmaf(u, 1.0f - s, 1.0f));
    }
    if (ACT == MDLSTM_RELU) return u > 0.0f ? dy : 0.0f;
    return dy;
}

// What a thread is: every `slices`-th token and four channels of the workgroup's block.
struct Place {
    int lane, slice, slices, c, in_block, valid, width, groups;  // width: channels of this block, groups: of this block
    __device__ __forceinline__ Place(const GroupNormArgs& a, int block) {
        slices = blockDim.x / a.lanes;
        slice = threadIdx.x / a.lanes;
        lane = threadIdx.x % a.lanes;
        width = min(a.block, a.channels - block * a.block);
        groups = width / a.per;
        in_block = lane * V;
        valid = slice < slices ? max(0, min(V, width - in_block)) : 0;
        if (valid == 0) in_block = 0;
        c = block * a.block + in_block;
    }
};

// A segment's rows as a thread takes them: row slice + k slices is `k` steps behind
// a uniform base, at 32 bits of the thread's own offset (slices * stride is less than 2^32
// bytes by the caller's check).
template <typename T, bool WIDE>
struct Rows {
    char* base;
    int64_t step;  // bytes
    uint32_t offset;
    int valid;
    __device__ __forceinline__ Rows(const void* p, int64_t stride, int64_t token, const Place& me)
        : base(static_cast<char*>(const_cast<void*>(p)) + token * stride * (int64_t)sizeof(T)), step(me.slices * stride * (int64_t)sizeof(T)),
          offset((uint32_t)me.slice * (uint32_t)stride * sizeof(T) + me.c * sizeof(T)), valid(me.valid) {}
    __device__ __forceinline__ Raw<T> load(int k) const {
        return load_raw<T, WIDE>(reinterpret_cast<const T*>(base + k * step + offset), valid);
    }
    __device__ __forceinline__ void store(int k, const float (&v)[V]) const {
        store_vec<T, WIDE>(reinterpret_cast<T*>(base + k * step + offset), valid, v);
    }
};

__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ bool find_unit(const GroupNormArgs& a, int64_t slot, Unit& u) {
    if (slot >= a.seqs.slots || !unit_of(a.seqs, slot, u)) return false;
    u.seq = __builtin_amdgcn_readfirstlane(u.seq);
    u.t0 = uniform(u.t0);
    u.len = uniform(u.len);
    u.from = uniform(u.from);
    u.to = uniform(u.to);
    return true;
}

// Sums over the workgroup's tokens and a group's channels of K values a channel, for each of a thread's channels the
// sum of its group. LDS: rows of `lanes` * V channels, a row a slice (or a wave, where waves hold whole rows), then the
// groups' sums. Short groups are added up by a thread each, others by waves in turn.
template <int K>
__device__ __forceinline__ void group_sums(const GroupNormArgs& a, const Place& me, const float (&v)[K][V], float* lds, float (&out)[K][V]) {
    const int per = a.per, row = a.lanes * V;
    const bool whole = a.lanes <= 64 && 64 % a.lanes == 0;  // lanes of a wave that hold the same channels are added first
    const int rows = whole ? (int)blockDim.x / 64 : me.slices;
    float* total = lds + (K * rows) * row;
    float t[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) t[k][i] = i < me.valid ? v[k][i] : 0.0f;
    if (whole) {
        for (int o = a.lanes; o < 64; o <<= 1)
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) t[k][i] += __shfl_xor(t[k][i], o);
    }
    lds_barrier();  // the sums of the call before have been read
    if (whole ? (threadIdx.x & 63) < a.lanes : me.slice < me.slices) {
        const int r = whole ? threadIdx.x / 64 : me.slice;
#pragma unroll
        for (int k = 0; k < K; ++k) *reinterpret_cast<floatx4*>(&lds[(k * rows + r) * row + me.lane * V]) = floatx4{t[k][0], t[k][1], t[k][2], t[k][3]};
    }
    lds_barrier();
    for (int c = threadIdx.x; c < K * me.width; c += blockDim.x) {  // the rows, in order, into the first
        float* at = lds + (c < me.width ? c : rows * row + c - me.width);
        float s = at[0];
#pragma unroll 4
        for (int r = 1; r < rows; ++r) s += at[r * row];
        at[0] = s;
    }
    lds_barrier();
    if (per <= 32) {
        for (int x = threadIdx.x; x < K * me.groups; x += blockDim.x) {
            const float* at = lds + (x < me.groups ? x * per : rows * row + (x - me.groups) * per);
            float s = 0.0f;
#pragma unroll 4
            for (int c = 0; c < per; ++c) s += at[c];
            total[x] = s;
        }
    } else {
        const int wave = threadIdx.x / 64, in_wave = threadIdx.x & 63, waves = blockDim.x / 64;
        for (int x = wave; x < K * me.groups; x += waves) {
            const float* at = lds + (x < me.groups ? x * per : rows * row + (x - me.groups) * per);
            float s = 0.0f;
            for (int c = in_wave; c < per; c += 64) s += at[c];
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
            if (in_wave == 0) total[x] = s;
        }
    }
    lds_barrier();
    int g = me.in_block / per, edge = (g + 1) * per;  // the channel behind the group
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (me.in_block + i == edge) ++g, edge += per;
        g = min(g, me.groups - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) out[k][i] = total[k * me.groups + g];
    }
}

// True for one thread and channel of each group of the block, to write what the group has.
__device__ __forceinline__ bool speaks(const GroupNormArgs& a, const Place& me, int i) {
    return me.slice == 0 && i < me.valid && (me.in_block + i) % a.per == 0;
}

// Forward. AGAIN: a segment of a long sequence whose mean and rstd are known; else
// a sequence that a workgroup holds, or a long one's segment for its sums alone.
template <typename T, int ACT, bool WIDE, bool AGAIN>
__global__ __launch_bounds__(Forward::THREADS) void k_groupnorm_fwd(GroupNormArgs a) {
    constexpr int N = Hold<T, Forward>;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int64_t index = block_index(), slot = uniform(index / a.blocks);
    Unit u;
    if (!find_unit(a, slot, u)) return;
    const bool part = u.from > 0 || u.to < u.len;
    if (AGAIN && !part) return;
    const int block = __builtin_amdgcn_readfirstlane((int)(index - slot * a.blocks)), per = a.per, n = (int)(u.to - u.from);
    const Place me(a, block);
    const Rows<T, WIDE> x(a.x.p, a.x.stride, u.t0 + u.from, me), y(a.y, a.channels, u.t0 + u.from, me);
    const int64_t stat = (int64_t)u.seq * a.groups;
    const bool mine = me.valid > 0;
    float mean[1][V] = {}, rstd[V];
    Raw<T> raw[N];
    // f(k) for the thread's vectors; what no thread of the workgroup has is skipped as a whole
    auto each = [&](auto f) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k * me.slices < n)
                if (mine && me.slice + k * me.slices < n) f(k);
    };
    each([&](int k) { raw[k] = x.load(k); });
    float w[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = i < me.valid ? a.w[me.c + i] : 0.0f;
        b[i] = i < me.valid ? a.b[me.c + i] : 0.0f;
    }
    if constexpr (!AGAIN) {
        const float inv = n > 0 ? 1.0f / ((float)n * (float)per) : 0.0f;
        float sum[1][V] = {};
        each([&](int k) {
            float v[V];
            unpack(raw[k], v);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0][i] += v[i];
        });
        group_sums<1>(a, me, sum, lds, mean);
        float off[2][V] = {}, all[2][V];
#pragma unroll
        for (int i = 0; i < V; ++i) mean[0][i] *= inv;
        each([&](int k) {
            float v[V];
            unpack(raw[k], v);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = v[i] - mean[0][i];
                off[0][i] += d;
                off[1][i] = fmaf(d, d, off[1][i]);
            }
        });
        group_sums<2>(a, me, off, lds, all);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = all[0][i] * inv;  // what rounding left of the mean
            mean[0][i] += d;
            const float squares = fmaxf(fmaf(-all[0][i], d, all[1][i]), 0.0f);
            if (all[1][i] != all[1][i]) mean[0][i] = all[1][i];
            rstd[i] = 1.0f / sqrtf(fmaf(squares, inv, a.eps));
            if (speaks(a, me, i)) {
                const int g = (me.c + i) / per;
                if (part) {
                    float* s = a.sums + (u.slot * a.groups + g) * 2;
                    s[0] = mean[0][i];
                    s[1] = squares;
                } else {
                    a.mean[stat + g] = mean[0][i];
                    a.rstd[stat + g] = rstd[i];
                }
            }
        }
        if (part) return;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = min((me.c + i) / per, a.groups - 1);
            mean[0][i] = a.mean[stat + g];
            rstd[i] = a.rstd[stat + g];
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) rstd[i] *= w[i];
    each([&](int k) {
        float v[V];
        unpack(raw[k], v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = activate<ACT, sizeof(T) == 4>(fmaf(v[i] - mean[0][i], rstd[i], b[i]));
        y.store(k, v);
    });
}

// mean and rstd of the long sequences from their segments': a wave a group.
__global__ __launch_bounds__(64) void k_groupnorm_join(GroupNormArgs a) {
    const int64_t index = block_index();
    const int seq = (int)(index / a.groups), g = (int)(index - (int64_t)seq * a.groups);
    if (seq >= a.seqs.n) return;
    Unit u;
    sequence_of(a.seqs, seq, u);
    if (u.len <= a.seqs.seg) return;
    const int64_t count = (u.len + a.seqs.seg - 1) / a.seqs.seg, slot0 = u.t0 / a.seqs.seg + seq;
    const int per = a.per;
    auto sum = [&](auto f) {
        double s = 0.0;
        for (int64_t k = threadIdx.x; k < count; k += 64) {
            const float* v = a.sums + ((slot0 + k) * a.groups + g) * 2;
            s += f((double)(min(u.len, (k + 1) * a.seqs.seg) - k * a.seqs.seg), (double)v[0], (double)v[1]);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
        return s;
    };
    const double mean = sum([](double n, double m, double) { return n * m; }) / (double)u.len;
    const double squares = sum([=](double n, double m, double q) { return q + n * per * (m - mean) * (m - mean); });
    if (threadIdx.x == 0) {
        a.mean[(int64_t)seq * a.groups + g] = (float)mean;
        a.rstd[(int64_t)seq * a.groups + g] = (float)(1.0 / sqrt(squares / ((double)u.len * per) + (double)a.eps));
    }
}

// Backward, AGAIN as in the forward pass (the group means of g and g c are known).
template <typename T, typename H, int ACT, bool WIDE, bool AGAIN>
__global__ __launch_bounds__(H::THREADS) void k_groupnorm_bwd(GroupNormArgs a) {
    constexpr int N = Hold<T, H>;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int64_t index = block_index(), first = uniform(index / a.blocks);
    if (first >= a.parts) return;  // a launch has whole rows of workgroups
    const int block = __builtin_amdgcn_readfirstlane((int)(index - first * a.blocks)), per = a.per;
    const Place me(a, block);
    const bool mine = me.valid > 0;
    float w[V], b[V], dw[V] = {}, db[V] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = i < me.valid ? a.w[me.c + i] : 0.0f;
        b[i] = i < me.valid ? a.b[me.c + i] : 0.0f;
    }
    for (int64_t slot = first; slot < a.seqs.slots; slot += a.parts) {
        Unit u;
        if (!find_unit(a, slot, u) || u.from >= u.to) continue;
        const bool part = u.from > 0 || u.to < u.len;
        if (AGAIN && !part) continue;
        const int n = (int)(u.to - u.from);
        const int64_t stat = (int64_t)u.seq * a.groups, token = u.t0 + u.from;
        const Rows<T, WIDE> x(a.x.p, a.x.stride, token, me), dy(a.dy.p, a.dy.stride, token, me), dx(a.dx, a.channels, token, me);
        auto each = [&](auto f) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k * me.slices < n)
                    if (mine && me.slice + k * me.slices < n) f(k);
        };
        Raw<T> rx[N], rg[N];
        each([&](int k) { rx[k] = x.load(k), rg[k] = dy.load(k); });
        float mean[V], rstd[V], m[2][V], s[2][V] = {}, e[N][V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = min((me.c + i) / per, a.groups - 1);
            mean[i] = a.mean[stat + g];
            rstd[i] = a.rstd[stat + g];
        }
        each([&](int k) {
            float c[V];
            unpack(rx[k], c);
            unpack(rg[k], e[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                c[i] = (c[i] - mean[i]) * rstd[i];
                e[k][i] = activate_back<ACT, sizeof(T) == 4>(e[k][i], fmaf(c[i], w[i], b[i]));
                if constexpr (!AGAIN) {
                    s[0][i] += e[k][i];
                    s[1][i] = fmaf(e[k][i], c[i], s[1][i]);
                }
            }
        });
        if constexpr (!AGAIN) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                db[i] += s[0][i];
                dw[i] += s[1][i];
                s[0][i] *= w[i];
                s[1][i] *= w[i];
            }
            group_sums<2>(a, me, s, lds, m);
            if (part) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (speaks(a, me, i)) {
                        float* to = a.sums + (u.slot * a.groups + (me.c + i) / per) * 2;
                        to[0] = m[0][i];
                        to[1] = m[1][i];
                    }
                continue;
            }
            const float inv = 1.0f / ((float)n * (float)per);
#pragma unroll
            for (int i = 0; i < V; ++i) m[0][i] *= inv, m[1][i] *= inv;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float* from = a.means + (stat + min((me.c + i) / per, a.groups - 1)) * 2;
                m[0][i] = from[0];
                m[1][i] = from[1];
            }
        }
        each([&](int k) {
            float c[V];
            unpack(rx[k], c);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                c[i] = (c[i] - mean[i]) * rstd[i];
                c[i] = rstd[i] * fmaf(-c[i], m[1][i], fmaf(e[k][i], w[i], -m[0][i]));
            }
            dx.store(k, c);
        });
    }
    if (AGAIN) return;
    // the workgroup's share of dw and db, its slices added in order
    float* to = a.part + first * 2 * a.channels;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
        if (me.slice < me.slices)
#pragma unroll
            for (int i = 0; i < V; ++i) lds[(me.slice * a.lanes + me.lane) * V + i] = i < me.valid ? (k ? db[i] : dw[i]) : 0.0f;
        __syncthreads();
        for (int c = threadIdx.x; c < me.width; c += blockDim.x) {
            float s = 0.0f;
            for (int r = 0; r < me.slices; ++r) s += lds[r * a.lanes * V + c];
            to[k * a.channels + block * a.block + c] = s;
        }
    }
}

// The group means of g and g c of the long sequences: a wave a group.
__global__ __launch_bounds__(64) void k_groupnorm_means(GroupNormArgs a) {
    const int64_t index = block_index();
    const int seq = (int)(index / a.groups), g = (int)(index - (int64_t)seq * a.groups);
    if (seq >= a.seqs.n) return;
    Unit u;
    sequence_of(a.seqs, seq, u);
    if (u.len <= a.seqs.seg) return;
    const int64_t count = (u.len + a.seqs.seg - 1) / a.seqs.seg, slot0 = u.t0 / a.seqs.seg + seq;
    double s0 = 0.0, s1 = 0.0;
    for (int64_t k = threadIdx.x; k < count; k += 64) {
        const float* v = a.sums + ((slot0 + k) * a.groups + g) * 2;
        s0 += v[0];
        s1 += v[1];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s0 += __shfl_xor(s0, o), s1 += __shfl_xor(s1, o);
    if (threadIdx.x == 0) {
        const double size = (double)u.len * (a.channels / a.groups);
        float* to = a.means + ((int64_t)seq * a.groups + g) * 2;
        to[0] = (float)(s0 / size);
        to[1] = (float)(s1 / size);
    }
}

// dw and db: the workgroups' shares, 64 slices of them, each in order, added in
// order. 16 columns a workgroup, eight loads of a thread in flight.
__global__ __launch_bounds__(1024) void k_groupnorm_dw(int channels, int64_t parts, const float* part, float* dw, float* db) {
    __shared__ float lds[64][17];
    const int cols = 2 * channels, c = blockIdx.x * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
    const int64_t lo = parts * slice / 64, hi = parts * (slice + 1) / 64;
    float s = 0.0f;
    if (c < cols)
        for (int64_t g = lo; g < hi; g += 8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = g + i < hi ? part[(g + i) * cols + c] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
    lds[slice][threadIdx.x % 16] = s;
    __syncthreads();
    if (threadIdx.x < 16 && c < cols) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i) s += lds[i][threadIdx.x];
        (c < channels ? dw[c] : db[c - channels]) = s;
    }
}

bool aligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// The shape of a pass: the threads of a workgroup and the tokens it holds.
struct Shape {
    int threads, held;
};

template <typename H>
Shape shape_of(GroupNormArgs& a) {
    const int per = a.channels / a.groups, es = a.dtype ? 2 : 4, hold = a.dtype ? Hold<bf16_t, H> : Hold<float, H>, most = H::THREADS;
    a.per = per;
    // whole groups, in whole vectors where a few groups give them
    int unit = per;
    while (unit % V && unit + per <= std::min(256, a.channels)) unit += per;
    if (unit % V) unit = per;
    // about 128 bytes of a row; 64 where a workgroup then holds the longest sequence
    auto with = [&](int bytes) {
        int block = unit;
        while (block * es < bytes && block + unit <= a.channels) block += unit;
        a.block = block;
        a.lanes = (block + V - 1) / V;
    };
    with(128);
    if (most / a.lanes * hold < a.seqs.longest) {
        with(64);
        if (most / a.lanes * hold < a.seqs.longest) with(128);
    }
    a.blocks = (a.channels + a.block - 1) / a.block;
    Shape s;
    s.threads = 256;
    while (s.threads < most && (s.threads < a.lanes || (int64_t)s.threads / a.lanes * hold < a.seqs.longest)) s.threads *= 2;
    s.held = s.threads / a.lanes * hold;
    a.seqs.seg = a.seqs.longest > s.held ? s.held : 0;
    a.seqs.slots = packed_slots(a.seqs, a.seqs.seg);
    a.parts = a.seqs.seg ? a.seqs.slots : std::min<int64_t>(a.seqs.slots, std::max(1, 4096 / a.blocks));
    return s;
}

int64_t align256(int64_t bytes) { return (bytes + 255) & ~(int64_t)255; }

struct Plan {
    int64_t sums, part, means, total;
};
Plan plan_of(const GroupNormArgs& a, bool backward) {
    Plan p{};
    p.sums = 0;
    p.part = p.sums + (a.seqs.seg ? align256(a.seqs.slots * a.groups * 8) : 0);
    p.means = p.part + (backward ? align256(a.parts * a.channels * 8) : 0);
    p.total = p.means + (backward && a.seqs.seg ? align256((int64_t)a.seqs.n * a.groups * 8) : 0);
    return p;
}

template <typename H>
hipError_t launch(const GroupNormArgs& in, hipStream_t s) {
    GroupNormArgs a = in;
    constexpr bool BACKWARD = H::BACKWARD;
    const Shape shape = shape_of<H>(a);
    const Plan p = plan_of(a, BACKWARD);
    char* ws = static_cast<char*>(a.ws);
    a.sums = reinterpret_cast<float*>(ws + p.sums);
    a.part = reinterpret_cast<float*>(ws + p.part);
    a.means = reinterpret_cast<float*>(ws + p.means);
    const int es = a.dtype ? 2 : 4;
    bool wide = a.channels % V == 0 && a.block % V == 0 && a.x.stride % V == 0 && aligned(a.x.p, V * es);
    if (BACKWARD)
        wide = wide && a.dy.stride % V == 0 && aligned(a.dy.p, V * es) && aligned(a.dx, V * es);
    else
        wide = wide && aligned(a.y, V * es);
    const bool whole = a.lanes <= 64 && 64 % a.lanes == 0;
    const int rows = whole ? shape.threads / 64 : shape.threads / a.lanes;
    const size_t sums = (size_t)2 * rows * a.lanes * V + 2 * (a.block / (a.channels / a.groups)), shares = (size_t)(shape.threads / a.lanes) * a.lanes * V;
    const size_t lds = std::max(sums, BACKWARD ? shares : (size_t)0) * 4;
    dim3 grid, again, join;
    if (!grid_of((BACKWARD ? a.parts : a.seqs.slots) * a.blocks, shape.threads, grid) || !grid_of(a.seqs.slots * a.blocks, shape.threads, again) ||
        !grid_of((int64_t)a.seqs.n * a.groups, 64, join))
        return hipErrorInvalidValue;
    auto run = [&](auto t, auto act, auto w) {
        typedef decltype(t) T;
        constexpr int ACT = act();
        constexpr bool W = w();
        hipError_t e = hipSuccess;
        if (a.seqs.n > 0) {
            if constexpr (BACKWARD)
                k_groupnorm_bwd<T, H, ACT, W, false><<<grid, shape.threads, lds, s>>>(a);
            else
                k_groupnorm_fwd<T, ACT, W, false><<<grid, shape.threads, lds, s>>>(a);
            e = hipGetLastError();
            if (e == hipSuccess && a.seqs.seg) {
                if constexpr (BACKWARD)
                    k_groupnorm_means<<<join, 64, 0, s>>>(a);
                else
                    k_groupnorm_join<<<join, 64, 0, s>>>(a);
                e = hipGetLastError();
                if (e != hipSuccess) return e;
                if constexpr (BACKWARD)
                    k_groupnorm_bwd<T, H, ACT, W, true><<<again, shape.threads, lds, s>>>(a);
                else
                    k_groupnorm_fwd<T, ACT, W, true><<<again, shape.threads, lds, s>>>(a);
                e = hipGetLastError();
            }
        }
        if (BACKWARD && e == hipSuccess) {
            k_groupnorm_dw<<<(2 * a.channels + 15) / 16, 1024, 0, s>>>(a.channels, a.seqs.n > 0 ? a.parts : 0, a.part, a.dw, a.db);
            e = hipGetLastError();
        }
        return e;
    };
    const std::true_type yes;
    const std::false_type no;
    auto with_act = [&](auto t) {
        const std::integral_constant<int, MDLSTM_NO_ACTIVATION> none;
        const std::integral_constant<int, MDLSTM_RELU> relu;
        const std::integral_constant<int, MDLSTM_SILU> silu;
        if (a.act == MDLSTM_SILU) return wide ? run(t, silu, yes) : run(t, silu, no);
        if (a.act == MDLSTM_RELU) return wide ? run(t, relu, yes) : run(t, relu, no);
        return wide ? run(t, none, yes) : run(t, none, no);
    };
    return a.dtype ? with_act(bf16_t()) : with_act(float());
}

bool wide_rows(const GroupNormArgs& a) { return a.channels / a.groups > V * Backward::THREADS; }

}  // namespace

size_t groupnorm_workspace_bytes(const GroupNormArgs& in, bool backward) {
    GroupNormArgs a = in;
    (void)(!backward ? shape_of<Forward>(a) : wide_rows(a) ? shape_of<BackwardOfWideRows>(a) : shape_of<Backward>(a));
    return (size_t)std::max<int64_t>(plan_of(a, backward).total, 16);
}

hipError_t launch_groupnorm_fwd(const GroupNormArgs& a, hipStream_t s) { return launch<Forward>(a, s); }
hipError_t launch_groupnorm_bwd(const GroupNormArgs& a, hipStream_t s) {
    return wide_rows(a) ? launch<BackwardOfWideRows>(a, s) : launch<Backward>(a, s);
}

}  // namespace mdl
