// Group norm with an activation over packed sequences, channels last: mean and
// variance over the tokens of a sequence and the channels of a group,
//     c = (x - mean) rstd        u = c w + b        y = act(u)
// and its gradients, with e = dy act'(u) and g = e w,
//     dx = rstd (g - mean(g) - c mean(g c))    dw = sum of e c    db = sum of e.
//
// HBM bounds it, so a workgroup keeps the tokens of a sequence in registers
// where they fit (a block of whole groups, `Hold` vectors of four channels a
// thread) between the sums and their use, and each input is read once. Longer
// sequences are cut into segments: a pass for the segments' sums, one that joins
// them in order, and a pass that reads the segments again. Measured, bf16 with silu:
// 128 sequences of 300 to 1200 tokens of 512 channels in 32 groups, forward held 66 us
// (196 MB, 3.0 TB/s), backward in segments 75 + 75 us (196 MB read, then 295 MB: 2.6 and
// 3.9 TB/s; held by 512 threads with 256 registers it took 175); eight pages of 60000
// to 70000 tokens of 320 channels, 102 + 161 us and 199 + 258 us (3.3, 4.2, 3.4 and 3.9
// TB/s). By the counters a number of the pages takes 9 and 18 vector instructions forward, 23
// and 23 backward: at four cycles each, sixteen for the exponential and the reciprocal,
// some 60% of the backward passes' time beside the memory's.
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

// What a pass does: all of a sequence that a workgroup holds; or a segment's sums; or a
// segment again, when its sequence's sums are known.
enum { WHOLE, SUMS, AGAIN };

// Threads of a workgroup at most, waves of a SIMD that its registers leave room for, the
// bytes of x that a thread holds (backward with dy's and, for a whole sequence, the
// fp32 numbers e beside them).
struct ForwardWhole {
    static constexpr int THREADS = 512, WAVES = 4, BYTES[2] = {160, 160}, LEAST = 64;  // bytes of fp32 and bf16; of a row at least
};
struct BackwardWhole {
    static constexpr int THREADS = 256, WAVES = 2, BYTES[2] = {160, 96}, LEAST = 64;
};
struct Segments {
    static constexpr int THREADS = 256, WAVES = 4, BYTES[2] = {64, 64}, LEAST = 128;
};
struct SegmentsOfWideRows {  // a row of a group needs more than 256 threads
    static constexpr int THREADS = 1024, WAVES = 4, BYTES[2] = {64, 64}, LEAST = 128;
};
template <typename T, typename H>
constexpr int Hold = H::BYTES[sizeof(T) == 2] / (V * sizeof(T));

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
    int64_t row, step;  // bytes
    uint32_t offset;
    int valid;
    __device__ __forceinline__ Rows(const void* p, int64_t stride, int64_t token, const Place& me)
        : base(static_cast<char*>(const_cast<void*>(p)) + token * stride * (int64_t)sizeof(T)), row(stride * (int64_t)sizeof(T)), step(me.slices * row),
          offset((uint32_t)me.slice * (uint32_t)stride * sizeof(T) + me.c * sizeof(T)), valid(me.valid) {}
    __device__ __forceinline__ void skip(int tokens) { base += tokens * row; }
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
// The slot and the block of channels of a workgroup: all blocks of a slot on one XCD
// (workgroups 8 apart) one after the other, as they share the rows' lines.
__device__ __forceinline__ void place(const GroupNormArgs& a, int64_t& slot, int& block) {
    const int64_t index = block_index(), at = index / 8;
    slot = uniform(at / a.blocks) * 8 + index % 8;
    block = __builtin_amdgcn_readfirstlane((int)(at % a.blocks));
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
    for (int c = threadIdx.x; c < K * me.width; c += (int)blockDim.x) {  // the rows, in order, into the first
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

template <typename T, typename H, int ACT, bool WIDE, int MODE>
__global__ __launch_bounds__(H::THREADS, H::WAVES) void k_groupnorm_fwd(GroupNormArgs a) {
    constexpr int N = Hold<T, H>;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    int64_t slot;
    int block;
    place(a, slot, block);
    Unit u;
    if (!find_unit(a, slot, u)) return;
    const int per = a.per, all = (int)(u.to - u.from);
    const Place me(a, block);
    Rows<T, WIDE> x(a.x.p, a.x.stride, u.t0 + u.from, me), y(a.y, a.channels, u.t0 + u.from, me);
    const int64_t stat = (int64_t)u.seq * a.groups;
    const bool mine = me.valid > 0;
    int left = all, n = min(left, a.held);  // tokens from here on, those held now
    float mean[1][V] = {}, rstd[V];
    Raw<T> raw[N];
    // f(k) for the thread's vectors; what no thread of the workgroup has is skipped as a whole
    auto each = [&](auto f) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k * me.slices < n)
                if (mine && me.slice + k * me.slices < n) f(k);
    };
    auto load = [&](int k) { raw[k] = x.load(k); };
    auto next = [&]() {  // the tokens behind those held; false behind the last
        x.skip(a.held);
        y.skip(a.held);
        left -= a.held;
        n = min(left, a.held);
        if (left > 0) each(load);
        return left > 0;
    };
    each(load);
    float w[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        w[i] = i < me.valid ? a.w[me.c + i] : 0.0f;
        b[i] = i < me.valid ? a.b[me.c + i] : 0.0f;
    }
    if constexpr (MODE != AGAIN) {
        float sum[1][V] = {};
        each([&](int k) {
            float v[V];
            unpack(raw[k], v);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[0][i] += v[i];
        });
        group_sums<1>(a, me, sum, lds, mean);
        float off[2][V] = {}, total[2][V];
#pragma unroll
        for (int i = 0; i < V; ++i) mean[0][i] *= n > 0 ? 1.0f / ((float)n * (float)per) : 0.0f;
        // distances from the mean of the tokens held first: those of a segment are not far from it beside their own spread
        do {
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
        } while (MODE == SUMS && next());
        group_sums<2>(a, me, off, lds, total);
        const float inv = all > 0 ? 1.0f / ((float)all * (float)per) : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = total[0][i] * inv;  // from there to the mean of all, and what rounding left
            mean[0][i] += d;
            const float squares = fmaxf(fmaf(-total[0][i], d, total[1][i]), 0.0f);
            if (total[1][i] != total[1][i]) mean[0][i] = total[1][i];
            rstd[i] = 1.0f / sqrtf(fmaf(squares, inv, a.eps));
            if (speaks(a, me, i)) {
                const int g = (me.c + i) / per;
                if (MODE == SUMS) {
                    float* s = a.sums + (u.slot * a.groups + g) * 2;
                    s[0] = mean[0][i];
                    s[1] = squares;
                } else {
                    a.mean[stat + g] = mean[0][i];
                    a.rstd[stat + g] = rstd[i];
                }
            }
        }
        if (MODE == SUMS) return;
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
    do {
        each([&](int k) {
            float v[V];
            unpack(raw[k], v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = activate<ACT, sizeof(T) == 4>(fmaf(v[i] - mean[0][i], rstd[i], b[i]));
            y.store(k, v);
        });
    } while (MODE == AGAIN && next());
}

// mean and rstd of the sequences from their segments': a wave a group.
__global__ __launch_bounds__(64) void k_groupnorm_join(GroupNormArgs a) {
    const int64_t index = block_index();
    const int seq = (int)(index / a.groups), g = (int)(index - (int64_t)seq * a.groups);
    if (seq >= a.seqs.n) return;
    Unit u;
    sequence_of(a.seqs, seq, u);
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
    const double mean = sum([](double n, double m, double) { return n * m; }) / (double)max(u.len, (int64_t)1);
    const double squares = sum([=](double n, double m, double q) { return q + n * per * (m - mean) * (m - mean); });
    if (threadIdx.x == 0) {
        a.mean[(int64_t)seq * a.groups + g] = (float)mean;
        a.rstd[(int64_t)seq * a.groups + g] = (float)(1.0 / sqrt(squares / ((double)max(u.len, (int64_t)1) * per) + (double)a.eps));
    }
}

template <typename T, typename H, int ACT, bool WIDE, int MODE>
__global__ __launch_bounds__(H::THREADS, H::WAVES) void k_groupnorm_bwd(GroupNormArgs a) {
    constexpr int N = Hold<T, H>;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    int64_t first;
    int block;
    place(a, first, block);
    if (first >= a.parts) return;
    const int per = a.per;
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
        const int all = (int)(u.to - u.from);
        int left = all, n = min(left, a.held);
        const int64_t stat = (int64_t)u.seq * a.groups, token = u.t0 + u.from;
        Rows<T, WIDE> x(a.x.p, a.x.stride, token, me), dy(a.dy.p, a.dy.stride, token, me), dx(a.dx, a.channels, token, me);
        auto each = [&](auto f) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k * me.slices < n)
                    if (mine && me.slice + k * me.slices < n) f(k);
        };
        Raw<T> rx[N], rg[N];
        auto load = [&](int k) { rx[k] = x.load(k), rg[k] = dy.load(k); };
        auto next = [&]() {
            x.skip(a.held);
            dy.skip(a.held);
            dx.skip(a.held);
            left -= a.held;
            n = min(left, a.held);
            if (left > 0) each(load);
            return left > 0;
        };
        each(load);
        float mean[V], rstd[V], m[2][V], s[2][V] = {}, e[N][V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = min((me.c + i) / per, a.groups - 1);
            mean[i] = a.mean[stat + g];
            rstd[i] = a.rstd[stat + g];
        }
        auto parts = [&](int k, float (&c)[V], float (&e)[V]) {
            unpack(rx[k], c);
            unpack(rg[k], e);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = c[i] - mean[i];
                c[i] = d * rstd[i];
                // where it decides, u has the forward pass's own roundings: relu lets through what it let through there
                const float u = ACT == MDLSTM_RELU ? fmaf(d, rstd[i] * w[i], b[i]) : fmaf(c[i], w[i], b[i]);
                e[i] = activate_back<ACT, sizeof(T) == 4>(e[i], u);
            }
        };
        if constexpr (MODE != AGAIN) {
            do {
                each([&](int k) {
                    float c[V], now[V];
                    parts(k, c, now);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        if (MODE == WHOLE) e[k][i] = now[i];
                        s[0][i] += now[i];
                        s[1][i] = fmaf(now[i], c[i], s[1][i]);
                    }
                });
            } while (MODE == SUMS && next());
        }
        if constexpr (MODE != AGAIN) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                db[i] += s[0][i];
                dw[i] += s[1][i];
                s[0][i] *= w[i];
                s[1][i] *= w[i];
            }
            group_sums<2>(a, me, s, lds, m);
            if (MODE == SUMS) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (speaks(a, me, i)) {
                        float* to = a.sums + (u.slot * a.groups + (me.c + i) / per) * 2;
                        to[0] = m[0][i];
                        to[1] = m[1][i];
                    }
                continue;
            }
            const float inv = 1.0f / ((float)all * (float)per);
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
        do {
            each([&](int k) {
                float c[V], now[V];
                if constexpr (MODE == AGAIN) {
                    parts(k, c, now);
                } else {
                    unpack(rx[k], c);
#pragma unroll
                    for (int i = 0; i < V; ++i) c[i] = (c[i] - mean[i]) * rstd[i], now[i] = e[k][i];
                }
#pragma unroll
                for (int i = 0; i < V; ++i) c[i] = rstd[i] * fmaf(-c[i], m[1][i], fmaf(now[i], w[i], -m[0][i]));
                dx.store(k, c);
            });
        } while (MODE == AGAIN && next());
    }
    if (MODE == AGAIN) return;
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

// The group means of g and g c of the sequences: a wave a group.
__global__ __launch_bounds__(64) void k_groupnorm_means(GroupNormArgs a) {
    const int64_t index = block_index();
    const int seq = (int)(index / a.groups), g = (int)(index - (int64_t)seq * a.groups);
    if (seq >= a.seqs.n) return;
    Unit u;
    sequence_of(a.seqs, seq, u);
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
        const double size = (double)max(u.len, (int64_t)1) * a.per;
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

// Chooses channels of a workgroup, its threads and whether it holds whole sequences
// (seqs.seg 0). A workgroup takes whole groups, about 128 bytes of a row; 64 where
// it then holds the longest sequence: forward of 128 sequences of 300 to 1200 tokens
// of 512 bf16 channels 59 us, in segments 82; backward of 256 of 100 to 300 78 us, 96
// in segments.
template <typename H>
int shape_of(GroupNormArgs& a) {
    const int es = a.dtype ? 2 : 4, hold = a.dtype ? Hold<bf16_t, H> : Hold<float, H>;
    a.per = a.channels / a.groups;
    // whole groups, in whole vectors where a few groups give them
    int unit = a.per;
    while (unit % V && unit + a.per <= std::min(256, a.channels)) unit += a.per;
    if (unit % V) unit = a.per;
    auto with = [&](int bytes) {
        int block = unit;
        while (block * es < bytes && block + unit <= a.channels) block += unit;
        a.block = block;
        a.lanes = (block + V - 1) / V;
        a.blocks = (a.channels + block - 1) / block;
        return a.lanes <= H::THREADS ? H::THREADS / a.lanes * hold : 0;
    };
    int held = 0;
    for (int bytes = 128; bytes >= H::LEAST; bytes /= 2)
        if ((held = with(bytes)) >= std::max<int64_t>(a.seqs.longest, 1)) break;
    const bool whole = held >= std::max<int64_t>(a.seqs.longest, 1);
    if (!whole) held = with(128);
    int threads = H::THREADS;
    while (whole && threads > 64 && threads / 2 >= a.lanes && (int64_t)threads / 2 / a.lanes * hold >= a.seqs.longest) threads /= 2;
    // segments of up to four times what a workgroup holds, where some 2048 of them are left: a workgroup's start (its
    // sequence, weights, sums) takes about as long as 32 KB. Forward / backward with one, two, four and eight times, of
    // 320 bf16 channels: 8 sequences of 65000 tokens 271 / 442, 252 / 405, 256 / 400, 255 / 418 us, one of 30000 28 / 42,
    // 28 / 40, 32 / 47, 41 / 61. With 1024 left 8 of 8000 took 40 / 65 instead of 44 / 72, and 128 of 300 to 1200 tokens
    // of 512 channels 12 us more, as their segments differ.
    const int64_t times = std::max<int64_t>(1, std::min<int64_t>(4, a.seqs.tokens * a.blocks / (std::max(held, 1) * (int64_t)2048)));
    a.held = whole ? (int)std::max<int64_t>(a.seqs.longest, 1) : held;
    a.seqs.seg = whole ? 0 : std::max<int64_t>(held * times, 1);
    a.seqs.slots = packed_slots(a.seqs, a.seqs.seg);
    // backward: each part has a row of dw and db, however many slots there are
    a.parts = std::min<int64_t>(a.seqs.slots, std::max(1, 4096 / a.blocks));
    return threads;
}

// The same for segments, whatever the longest sequence.
template <typename H>
int segments_of(GroupNormArgs& a) {
    const int64_t longest = a.seqs.longest;
    a.seqs.longest = (int64_t)1 << 40;
    const int threads = shape_of<H>(a);
    a.seqs.longest = longest;
    return threads;
}

// f with the way a pass holds its sequences (shape_of is done), and the threads of a workgroup. Whole where the
// longest fits: 512 sequences of 60 tokens of 256 channels in bf16 14 us forward and 30 backward, in segments 40
// and 62; of 200 tokens 32 and 81 against 61 and 106.
template <bool BACKWARD, typename F>
auto with_hold(GroupNormArgs& a, F&& f) {
    typedef std::conditional_t<BACKWARD, BackwardWhole, ForwardWhole> Whole;
    const int threads = shape_of<Whole>(a);
    if (!a.seqs.seg) return f(Whole(), threads);
    if (a.per > V * Segments::THREADS) return f(SegmentsOfWideRows(), segments_of<SegmentsOfWideRows>(a));
    return f(Segments(), segments_of<Segments>(a));
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

template <bool BACKWARD, typename H>
hipError_t launch(GroupNormArgs a, int threads, hipStream_t s) {
    constexpr bool SEG = std::is_same_v<H, Segments> || std::is_same_v<H, SegmentsOfWideRows>;
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
    const int rows = whole ? threads / 64 : threads / a.lanes;
    const size_t sums = (size_t)2 * rows * a.lanes * V + 2 * (a.block / a.per), slices = (size_t)(threads / a.lanes) * a.lanes * V;
    const int64_t shares = a.parts;
    const size_t lds = std::max(sums, BACKWARD ? slices : (size_t)0) * 4;
    dim3 grid, join;
    if (!grid_of(((BACKWARD ? a.parts : a.seqs.slots) + 7) / 8 * 8 * a.blocks, threads, grid) ||
        !grid_of((int64_t)a.seqs.n * a.groups, 64, join))
        return hipErrorInvalidValue;
    auto run = [&](auto t, auto act, auto w) {
        typedef decltype(t) T;
        constexpr int ACT = act();
        constexpr bool W = w();
        hipError_t e = hipSuccess;
        auto pass = [&](auto mode) {
            if constexpr (BACKWARD)
                k_groupnorm_bwd<T, H, ACT, W, mode()><<<grid, threads, lds, s>>>(a);
            else
                k_groupnorm_fwd<T, H, ACT, W, mode()><<<grid, threads, lds, s>>>(a);
            return hipGetLastError();
        };
        if (a.seqs.n > 0) {
            if constexpr (!SEG) {
                e = pass(std::integral_constant<int, WHOLE>());
            } else {
                e = pass(std::integral_constant<int, SUMS>());
                if (e != hipSuccess) return e;
                if constexpr (BACKWARD)
                    k_groupnorm_means<<<join, 64, 0, s>>>(a);
                else
                    k_groupnorm_join<<<join, 64, 0, s>>>(a);
                e = hipGetLastError();
                if (e != hipSuccess) return e;
                if (!BACKWARD) {  // segments of what a workgroup holds now (pages 156 us, 193 with longer ones; backward 281 against 270)
                    a.seqs.seg = a.held;
                    a.seqs.slots = packed_slots(a.seqs, a.held);
                }
                a.parts = a.seqs.slots;
                if (!grid_of((a.seqs.slots + 7) / 8 * 8 * a.blocks, threads, grid)) return hipErrorInvalidValue;
                e = pass(std::integral_constant<int, AGAIN>());
            }
        }
        if (BACKWARD && e == hipSuccess) {
            k_groupnorm_dw<<<(2 * a.channels + 15) / 16, 1024, 0, s>>>(a.channels, a.seqs.n > 0 ? shares : 0, a.part, a.dw, a.db);
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

}  // namespace

size_t groupnorm_workspace_bytes(const GroupNormArgs& in, bool backward) {
    GroupNormArgs a = in;
    auto plan = [&](auto, int) { return plan_of(a, backward).total; };
    return (size_t)std::max<int64_t>(backward ? with_hold<true>(a, plan) : with_hold<false>(a, plan), 16);
}

hipError_t launch_groupnorm_fwd(const GroupNormArgs& in, hipStream_t s) {
    GroupNormArgs a = in;
    return with_hold<false>(a, [&](auto hold, int threads) { return launch<false, decltype(hold)>(a, threads, s); });
}
hipError_t launch_groupnorm_bwd(const GroupNormArgs& in, hipStream_t s) {
    GroupNormArgs a = in;
    return with_hold<true>(a, [&](auto hold, int threads) { return launch<true, decltype(hold)>(a, threads, s); });
}

}  // namespace mdl
