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

// Vectors of a tensor that a thread holds: 128 bytes forward, two tensors of 64 bytes backward.
template <typename T, bool BACKWARD>
constexpr int Hold = (BACKWARD ? 64 : 128) / (V * sizeof(T));

__device__ __forceinline__ float sigmoid(float u) { return 1.0f / (1.0f + expf(-u)); }

__device__ __forceinline__ float activate(float u, int act) {
    if (act == MDLSTM_SILU) return u * sigmoid(u);
    if (act == MDLSTM_RELU) return u < 0.0f ? 0.0f : u;  // a NaN stays one
    return u;
}
// dy act'(u)
__device__ __forceinline__ float activate_back(float dy, float u, int act) {
    if (act == MDLSTM_SILU) {
        const float s = sigmoid(u);
        return dy * (s * fmaf(u, 1.0f - s, 1.0f));
    }
    if (act == MDLSTM_RELU) return u > 0.0f ? dy : 0.0f;
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
        groups = width / (a.channels / a.groups);
        in_block = lane * V;
        valid = slice < slices ? max(0, min(V, width - in_block)) : 0;
        if (valid == 0) in_block = 0;
        c = block * a.block + in_block;
    }
};

// Sums over the workgroup's tokens and a group's channels of K values a channel, for each of a thread's channels the
// sum of its group. LDS: rows of `lanes` * V channels, a row a slice (or a wave, where waves hold whole rows), then the
// groups' sums. Waves take the groups in turn.
template <int K>
__device__ __forceinline__ void group_sums(const GroupNormArgs& a, const Place& me, const float (&v)[K][V], float* lds, float (&out)[K][V]) {
    const int per = a.channels / a.groups, row = a.lanes * V;
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
    __syncthreads();  // the sums of the call before have been read
    if (whole ? (threadIdx.x & 63) < a.lanes : me.slice < me.slices) {
        const int r = whole ? threadIdx.x / 64 : me.slice;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) lds[(k * rows + r) * row + me.lane * V + i] = t[k][i];
    }
    __syncthreads();
    const int wave = threadIdx.x / 64, in_wave = threadIdx.x & 63, waves = blockDim.x / 64;
    for (int g = wave; g < me.groups; g += waves) {
        float s[K] = {};
        for (int c = in_wave; c < per * rows; c += 64) {
            const int r = c / per, at = r * row + g * per + (c - r * per);
#pragma unroll
            for (int k = 0; k < K; ++k) s[k] += lds[k * rows * row + at];
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) s[k] += __shfl_xor(s[k], o);
            if (in_wave == 0) total[k * me.groups + g] = s[k];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = min((me.in_block + i) / per, me.groups - 1);
#pragma unroll
        for (int k = 0; k < K; ++k) out[k][i] = total[k * me.groups + g];
    }
}

// True for one thread and channel of each group of the block, to write what the group has.
__device__ __forceinline__ bool speaks(const GroupNormArgs& a, const Place& me, int i) {
    return me.slice == 0 && i < me.valid && (me.in_block + i) % (a.channels / a.groups) == 0;
}

// Forward. AGAIN: a segment of a long sequence whose mean and rstd are known; else
// a sequence that a workgroup holds, or a long one's segment for its sums alone.
template <typename T, bool WIDE, bool AGAIN>
__global__ __launch_bounds__(1024) void k_groupnorm_fwd(GroupNormArgs a) {
    constexpr int N = Hold<T, false>;
    extern __shared__ float lds[];
    const int64_t index = block_index(), slot = index / a.blocks;
    Unit u;
    if (slot >= a.seqs.slots || !unit_of(a.seqs, slot, u)) return;
    const bool part = u.from > 0 || u.to < u.len;
    if (AGAIN && !part) return;
    const int block = (int)(index - slot * a.blocks), per = a.channels / a.groups;
    const Place me(a, block);
    const T* x = static_cast<const T*>(a.x.p) + u.t0 * a.x.stride + me.c;
    const int64_t t = u.from + me.slice, stat = (int64_t)u.seq * a.groups;
    const bool mine = me.valid > 0;
    float mean[1][V] = {}, rstd[V];
    Raw<T> raw[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (mine && t + k * me.slices < u.to) raw[k] = load_raw<T, WIDE>(x + (t + (int64_t)k * me.slices) * a.x.stride, me.valid);
    if constexpr (!AGAIN) {
        const float count = (float)((u.to - u.from) * per);
        float sum[1][V] = {};
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (mine && t + k * me.slices < u.to) {
                float v[V];
                unpack(raw[k], v);
#pragma unroll
                for (int i = 0; i < V; ++i) sum[0][i] += v[i];
            }
        group_sums<1>(a, me, sum, lds, mean);
        float off[2][V] = {}, all[2][V];
#pragma unroll
        for (int i = 0; i < V; ++i) mean[0][i] = count > 0.0f ? mean[0][i] / count : 0.0f;
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (mine && t + k * me.slices < u.to) {
                float v[V];
                unpack(raw[k], v);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = v[i] - mean[0][i];
                    off[0][i] += d;
                    off[1][i] = fmaf(d, d, off[1][i]);
                }
            }
        group_sums<2>(a, me, off, lds, all);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = count > 0.0f ? all[0][i] / count : 0.0f;  // what rounding left of the mean
            mean[0][i] += d;
            const float squares = fmaxf(all[1][i] - count * d * d, 0.0f);
            if (all[1][i] != all[1][i]) mean[0][i] = all[1][i];
            const float var = count > 0.0f ? squares / count : 0.0f;
            rstd[i] = 1.0f / sqrtf(var + a.eps);
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
    if (!mine) return;
    float w[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = i < me.valid ? a.w[me.c + i] : 0.0f;
        b[i] = i < me.valid ? a.b[me.c + i] : 0.0f;
    }
    T* y = static_cast<T*>(a.y) + u.t0 * a.channels + me.c;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (t + k * me.slices < u.to) {
            float v[V];
            unpack(raw[k], v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activate(fmaf((v[i] - mean[0][i]) * rstd[i], w[i], b[i]), a.act);
            store_vec<T, WIDE>(y + (t + (int64_t)k * me.slices) * a.channels, me.valid, v);
        }
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
    const int per = a.channels / a.groups;
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
template <typename T, bool WIDE, bool AGAIN>
__global__ __launch_bounds__(1024) void k_groupnorm_bwd(GroupNormArgs a) {
    constexpr int N = Hold<T, true>;
    extern __shared__ float lds[];
    const int64_t index = block_index(), first = index / a.blocks;
    const int block = (int)(index - first * a.blocks), per = a.channels / a.groups;
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
        if (!unit_of(a.seqs, slot, u) || u.from >= u.to) continue;
        const bool part = u.from > 0 || u.to < u.len;
        if (AGAIN && !part) continue;
        const int64_t t = u.from + me.slice, stat = (int64_t)u.seq * a.groups;
        const T* x = static_cast<const T*>(a.x.p) + u.t0 * a.x.stride + me.c;
        const T* dy = static_cast<const T*>(a.dy.p) + u.t0 * a.dy.stride + me.c;
        Raw<T> rx[N], rg[N];
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (mine && t + k * me.slices < u.to) {
                rx[k] = load_raw<T, WIDE>(x + (t + (int64_t)k * me.slices) * a.x.stride, me.valid);
                rg[k] = load_raw<T, WIDE>(dy + (t + (int64_t)k * me.slices) * a.dy.stride, me.valid);
            }
        float mean[V], rstd[V], m[2][V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = min((me.c + i) / per, a.groups - 1);
            mean[i] = a.mean[stat + g];
            rstd[i] = a.rstd[stat + g];
        }
        // a token's c and e
        auto parts = [&](int k, float (&c)[V], float (&e)[V]) {
            unpack(rx[k], c);
            unpack(rg[k], e);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                c[i] = (c[i] - mean[i]) * rstd[i];
                e[i] = activate_back(e[i], fmaf(c[i], w[i], b[i]), a.act);
            }
        };
        if constexpr (!AGAIN) {
            float s[2][V] = {};
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (mine && t + k * me.slices < u.to) {
                    float c[V], e[V];
                    parts(k, c, e);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        s[0][i] += e[i];
                        s[1][i] = fmaf(e[i], c[i], s[1][i]);
                    }
                }
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
            const float count = (float)(u.len * per);
#pragma unroll
            for (int i = 0; i < V; ++i) m[0][i] /= count, m[1][i] /= count;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float* from = a.means + (stat + min((me.c + i) / per, a.groups - 1)) * 2;
                m[0][i] = from[0];
                m[1][i] = from[1];
            }
        }
        T* dx = static_cast<T*>(a.dx) + u.t0 * a.channels + me.c;
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (mine && t + k * me.slices < u.to) {
                float c[V], e[V];
                parts(k, c, e);
#pragma unroll
                for (int i = 0; i < V; ++i) e[i] = rstd[i] * (fmaf(e[i], w[i], -m[0][i]) - c[i] * m[1][i]);
                store_vec<T, WIDE>(dx + (t + (int64_t)k * me.slices) * a.channels, me.valid, e);
            }
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

// The shape of a pass: channels of a workgroup, its threads, the tokens it holds.
struct Shape {
    int threads, held;
};

Shape shape_of(GroupNormArgs& a, bool backward) {
    const int per = a.channels / a.groups, es = a.dtype ? 2 : 4;
    // whole groups of about 128 bytes of a row, in whole vectors where a few groups give them
    int unit = per;
    while (unit % V && unit + per <= std::min(256, a.channels)) unit += per;
    if (unit % V) unit = per;
    int block = unit;
    while (block * es < 128 && block + unit <= a.channels) block += unit;
    a.block = block;
    a.blocks = (a.channels + block - 1) / block;
    a.lanes = (block + V - 1) / V;
    const int hold = (backward ? 64 : 128) / (V * es);
    Shape s;
    s.threads = 256;
    while (s.threads < 1024 && (s.threads < a.lanes || (int64_t)s.threads / a.lanes * hold < a.seqs.longest)) s.threads *= 2;
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

template <bool BACKWARD>
hipError_t launch(const GroupNormArgs& in, hipStream_t s) {
    GroupNormArgs a = in;
    const Shape shape = shape_of(a, BACKWARD);
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
    auto run = [&](auto t, auto w) {
        typedef decltype(t) T;
        constexpr bool W = w();
        hipError_t e = hipSuccess;
        if (a.seqs.n > 0) {
            if constexpr (BACKWARD)
                k_groupnorm_bwd<T, W, false><<<grid, shape.threads, lds, s>>>(a);
            else
                k_groupnorm_fwd<T, W, false><<<grid, shape.threads, lds, s>>>(a);
            e = hipGetLastError();
            if (e == hipSuccess && a.seqs.seg) {
                if constexpr (BACKWARD)
                    k_groupnorm_means<<<join, 64, 0, s>>>(a);
                else
                    k_groupnorm_join<<<join, 64, 0, s>>>(a);
                e = hipGetLastError();
                if (e != hipSuccess) return e;
                if constexpr (BACKWARD)
                    k_groupnorm_bwd<T, W, true><<<again, shape.threads, lds, s>>>(a);
                else
                    k_groupnorm_fwd<T, W, true><<<again, shape.threads, lds, s>>>(a);
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
    if (a.dtype) return wide ? run(bf16_t(), yes) : run(bf16_t(), no);
    return wide ? run(float(), yes) : run(float(), no);
}

}  // namespace

size_t groupnorm_workspace_bytes(const GroupNormArgs& in, bool backward) {
    GroupNormArgs a = in;
    (void)shape_of(a, backward);
    return (size_t)std::max<int64_t>(plan_of(a, backward).total, 16);
}

hipError_t launch_groupnorm_fwd(const GroupNormArgs& a, hipStream_t s) { return launch<false>(a, s); }
hipError_t launch_groupnorm_bwd(const GroupNormArgs& a, hipStream_t s) { return launch<true>(a, s); }

}  // namespace mdl
