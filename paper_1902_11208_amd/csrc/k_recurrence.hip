// Gated linear recurrence over packed sequences: for each channel
//     h_t = f_t h_(t-1) + u_t        f = sigmoid(z), u = (1 - f) x   (or f = z, u = x)
// and its gradients, with the adjoint s_t = f_t G_t, G_t = dh_t + s_(t+1):
//     dz = G (h_(t-1) - x) f (1 - f), dx = G (1 - f)   (or dz = G h_(t-1), dx = G).
//
// A run of tokens maps a state to A h + B (A the product of its f, B what it
// leaves of a zero state), and runs are joined by (A, B) then (A', B') ->
// (A' A, A' B + B'). A workgroup walks a sequence in tiles of 128 tokens: sixteen
// slices of eight tokens, a thread for a slice of two channels. A thread keeps
// its tokens' f and u in registers, the slices' sums meet in LDS, every thread
// finds the state its slice starts from and goes through its tokens once more.
// So each input is read once and each output written once, and HBM bounds it. The
// next tile is loaded while one is computed.
//
// The forward pass keeps the fp32 state at every tile's start (1/64 of bf16
// inputs), and the backward pass finds h again from it instead of from the
// rounded output: h - x is a difference, and a rounded h would leave it with
// an error of 2^-9 of h.
#include <algorithm>

#include "common.hpp"
#include "recurrence.hpp"
#include "sequence.hpp"

namespace mdl {
namespace {

constexpr int L = 8;        // tokens of a slice
constexpr int SLICES = 16;  // slices of a tile
static_assert(L * SLICES == kRecurrenceTile, "a tile is its slices");

constexpr int V = 2;  // channels of a thread

// The channels of a thread as they are in memory.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <typename T>
struct RawOf {
    typedef u32x2 type;
    typedef u32x2 anywhere __attribute__((aligned(1)));
};
template <>
struct RawOf<bf16_t> {
    typedef uint32_t type;
    typedef uint32_t anywhere __attribute__((aligned(1)));
};
template <typename T>
using Raw = typename RawOf<T>::type;

// `valid` of the two channels at p; the others read as 0. WIDE: p is aligned to
// both and both are valid; else two valid ones are moved by the same instruction at
// their elements' alignment.
template <typename T, bool WIDE>
__device__ __forceinline__ Raw<T> load_raw(const T* p, int valid) {
    if constexpr (WIDE) return *reinterpret_cast<const Raw<T>*>(p);
    if (valid == V) return *reinterpret_cast<const typename RawOf<T>::anywhere*>(p);
    if constexpr (sizeof(T) == 4)
        return u32x2{valid > 0 ? __float_as_uint(p[0]) : 0u, 0u};
    else
        return valid > 0 ? (uint32_t)p[0] : 0u;
}
__device__ __forceinline__ void unpack(u32x2 r, float (&v)[V]) {
    v[0] = __uint_as_float(r[0]);
    v[1] = __uint_as_float(r[1]);
}
__device__ __forceinline__ void unpack(uint32_t r, float (&v)[V]) {
    v[0] = __uint_as_float(r << 16);
    v[1] = __uint_as_float(r & 0xffff0000u);
}
template <typename T, bool WIDE>
__device__ __forceinline__ void store_vec(T* p, int valid, const float (&v)[V]) {
    Raw<T> r;
    if constexpr (sizeof(T) == 4)
        r = u32x2{__float_as_uint(v[0]), __float_as_uint(v[1])};
    else
        r = f2bf2(v[0], v[1]);
    if constexpr (WIDE) {
        *reinterpret_cast<Raw<T>*>(p) = r;
    } else if (valid == V) {
        *reinterpret_cast<typename RawOf<T>::anywhere*>(p) = r;
    } else if (valid > 0) {
        St<T>::st1(p, v[0]);
    }
}
__device__ __forceinline__ void load_f32(const float* p, int valid, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = i < valid ? p[i] : 0.0f;
}
__device__ __forceinline__ void store_f32(float* p, int valid, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < valid) p[i] = v[i];
}

// sigmoid(z) and 1 - sigmoid(z), both to a few ulp of themselves: the smaller one
// is e / (1 + e) and not a difference. The reciprocal takes one Newton step: an
// error of f is met again in every token that a state lives through.
__device__ __forceinline__ void sigmoids(float z, float& f, float& rest) {
    const float e = expf(-fabsf(z)), d = 1.0f + e;
    float r = __builtin_amdgcn_rcpf(d);
    r = fmaf(fmaf(-d, r, 1.0f), r, r);
    const float small = e * r;
    f = z < 0.0f ? small : r;
    rest = z < 0.0f ? r : small;
    if (z != z) f = rest = z;
}

template <bool SIG>
__device__ __forceinline__ void coefficients(float z, float x, float& f, float& u) {
    if constexpr (SIG) {
        float rest;
        sigmoids(z, f, rest);
        u = rest * x;
    } else {
        f = z;
        u = x;
    }
}

// States beyond this, and sums that are not finite, are not joined by A h + B
// (A may have fallen below fp32's range, 0 times infinity is no number, A and
// B may have overflowed where the recurrence does not): the tokens are walked.
constexpr float LARGE_STATE = 0x1p64f;

__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_huge_valf(); }

// (A, B) that a join can use, or NaN.
__device__ __forceinline__ void mark_unusable(float& A, float& B) {
    if (!(finite(A) && finite(B))) A = B = __builtin_nanf("");
}

// What a thread is: a slice of a tile and two channels.
template <typename T, int CL>
struct Place {
    int slice, lane, c, valid;
    __device__ __forceinline__ Place(const RecurrenceArgs& a, int block) {
        slice = threadIdx.x / CL;
        lane = threadIdx.x % CL;
        c = (block * CL + lane) * V;
        valid = max(0, min(V, a.channels - c));
        if (valid == 0) c = 0;
    }
};

template <typename T, bool WIDE>
struct Rows {
    const T* p;
    int64_t stride;
    int valid;
    __device__ __forceinline__ Rows(const RowView& v, int64_t t0, int c, int valid_)
        : p(static_cast<const T*>(v.p) + t0 * v.stride + c), stride(v.stride), valid(valid_) {}
    // eight tokens from t; those from `to` on repeat the last one (and are not used)
    __device__ __forceinline__ void load(int64_t t, int64_t to, Raw<T> (&r)[L]) const {
#pragma unroll
        for (int i = 0; i < L; ++i) r[i] = load_raw<T, WIDE>(p + min(t + i, to - 1) * stride, valid);
    }
    __device__ __forceinline__ void at(int64_t t, float (&v)[V]) const { unpack(load_raw<T, WIDE>(p + t * stride, valid), v); }
};

// A slice's sums in LDS, of one of two tiles in turn (one barrier a tile).
template <int CL, int N>
struct Sums {
    float v[2][N][SLICES][CL * V];
};

__device__ __forceinline__ void copy_in(float* to, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = v[i];
}

// The state that slice `mine` starts from and the one that the tile leaves, from
// the state `h` it starts from (REVERSE: slices from the last to the first). True
// where a channel's sums cannot be joined.
template <int CL, bool REVERSE>
__device__ __forceinline__ bool join_slices(const float (*A)[CL * V], const float (*B)[CL * V], int mine, int lane, float (&h)[V],
                                            float (&start)[V]) {
    float top[V], before[V];
#pragma unroll
    for (int i = 0; i < V; ++i) before[i] = h[i], top[i] = fabsf(h[i]), start[i] = h[i];
#pragma unroll
    for (int k = 0; k < SLICES; ++k) {
        const int s = REVERSE ? SLICES - 1 - k : k;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (s == mine) start[i] = h[i];
            h[i] = fmaf(A[s][lane * V + i], h[i], B[s][lane * V + i]);
            top[i] = fmaxf(top[i], fabsf(h[i]));
        }
    }
    bool bad = false;
#pragma unroll
    for (int i = 0; i < V; ++i) bad = bad || (before[i] == before[i] && (h[i] != h[i] || top[i] > LARGE_STATE));
    return bad;
}

// h through the tokens from .. to - 1, one by one; `start`: the state in front of token `at`.
template <typename T, bool SIG, bool WIDE>
__device__ __forceinline__ void walk_forward(Rows<T, WIDE> z, Rows<T, WIDE> x, int64_t from, int64_t to, int64_t at,
                                             float (&h)[V], float (&start)[V]) {
#pragma unroll 1
    for (int64_t t = from; t < to; ++t) {
        float vz[V], vx[V];
        z.at(t, vz);
        x.at(t, vx);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (t == at) start[i] = h[i];
            float f, u;
            coefficients<SIG>(vz[i], vx[i], f, u);
            h[i] = fmaf(f, h[i], u);
        }
    }
}

// The adjoint from token to - 1 down to `from`; `start`: the one that meets token at - 1.
template <typename T, bool SIG, bool WIDE>
__device__ __forceinline__ void walk_reverse(Rows<T, WIDE> z, Rows<T, WIDE> dh, int64_t from, int64_t to, int64_t at,
                                             float (&s)[V], float (&start)[V]) {
#pragma unroll 1
    for (int64_t t = to - 1; t >= from; --t) {
        float vz[V], vg[V];
        z.at(t, vz);
        dh.at(t, vg);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (t == at - 1) start[i] = s[i];
            float f, u;
            coefficients<SIG>(vz[i], 0.0f, f, u);
            s[i] = f * (vg[i] + s[i]);
        }
    }
}

template <int CL>
constexpr int threads_of() { return CL * SLICES; }

// Forward pass of a sequence or segment. SUMS: only what it maps a state to, for the join.
template <typename T, bool SIG, bool WIDE, int CL, bool SUMS>
__global__ __launch_bounds__(threads_of<CL>()) void k_recurrence_fwd(RecurrenceArgs a, int blocks) {
    __shared__ Sums<CL, 2> lds;
    const int64_t index = block_index();
    const int64_t slot = index / blocks;
    Unit u;
    if (slot >= a.seqs.slots || !unit_of(a.seqs, slot, u)) return;
    const Place<T, CL> me(a, (int)(index - slot * blocks));
    const Rows<T, WIDE> z(a.z, u.t0, me.c, me.valid), x(a.x, u.t0, me.c, me.valid);
    const int64_t row = (int64_t)u.seq * a.channels + me.c, slot_row = u.slot * a.channels + me.c;
    float carry[V], A[V];
#pragma unroll
    for (int i = 0; i < V; ++i) carry[i] = 0.0f, A[i] = 1.0f;
    if (!SUMS) {
        if (u.from > 0)
            load_f32(a.starts + slot_row, me.valid, carry);
        else if (a.state)
            load_f32(a.state + row, me.valid, carry);
    }
    Raw<T> rz[L], rx[L];
    int64_t t = u.from + me.slice * L;
    if (u.from < u.to) z.load(t, u.to, rz), x.load(t, u.to, rx);
    int parity = 0;
    for (int64_t tile = u.from; tile < u.to; tile += kRecurrenceTile, t += kRecurrenceTile, parity ^= 1) {
        float f[L][V], in[L][V], pa[V], pb[V];
#pragma unroll
        for (int i = 0; i < V; ++i) pa[i] = 1.0f, pb[i] = 0.0f;
#pragma unroll
        for (int l = 0; l < L; ++l) {
            float vz[V], vx[V];
            unpack(rz[l], vz);
            unpack(rx[l], vx);
            const bool real = t + l < u.to;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                coefficients<SIG>(vz[i], vx[i], f[l][i], in[l][i]);
                if (!real) f[l][i] = 1.0f, in[l][i] = 0.0f;
                pa[i] *= f[l][i];
                pb[i] = fmaf(f[l][i], pb[i], in[l][i]);
            }
        }
        if (tile + kRecurrenceTile < u.to) z.load(t + kRecurrenceTile, u.to, rz), x.load(t + kRecurrenceTile, u.to, rx);
#pragma unroll
        for (int i = 0; i < V; ++i) mark_unusable(pa[i], pb[i]);
        copy_in(&lds.v[parity][0][me.slice][me.lane * V], pa);
        copy_in(&lds.v[parity][1][me.slice][me.lane * V], pb);
        lds_barrier();
        float h[V];
        if constexpr (SUMS) {
#pragma unroll
            for (int s = 0; s < SLICES; ++s)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float fs = lds.v[parity][0][s][me.lane * V + i];
                    A[i] *= fs;
                    carry[i] = fmaf(fs, carry[i], lds.v[parity][1][s][me.lane * V + i]);
                    if (fabsf(carry[i]) > LARGE_STATE) A[i] = __builtin_nanf("");
                }
        } else {
            float before[V];
#pragma unroll
            for (int i = 0; i < V; ++i) before[i] = carry[i];
            if (join_slices<CL, false>(lds.v[parity][0], lds.v[parity][1], me.slice, me.lane, carry, h)) {
#pragma unroll
                for (int i = 0; i < V; ++i) carry[i] = before[i];
                walk_forward<T, SIG, WIDE>(z, x, tile, min(tile + kRecurrenceTile, u.to), t, carry, h);
            }
            if (a.marks && tile > 0 && me.slice == 0)
                store_f32(a.marks + (u.t0 / kRecurrenceTile + tile / kRecurrenceTile) * a.channels + me.c, me.valid, before);
            T* out = static_cast<T*>(a.h) + (u.t0 + t) * a.channels + me.c;
#pragma unroll
            for (int l = 0; l < L; ++l) {
#pragma unroll
                for (int i = 0; i < V; ++i) h[i] = fmaf(f[l][i], h[i], in[l][i]);
                if (t + l < u.to && me.valid) store_vec<T, WIDE>(out + (int64_t)l * a.channels, me.valid, h);
            }
        }
    }
    if (me.slice != 0) return;
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i) mark_unusable(A[i], carry[i]);
        store_f32(a.sums + slot_row, me.valid, A);
        store_f32(a.sums + a.seqs.slots * a.channels + slot_row, me.valid, carry);
    } else if (a.final_state && u.to == u.len) {
        store_f32(a.final_state + row, me.valid, carry);
    }
}

// Backward pass. SUMS: only what the unit maps the adjoint behind it to.
template <typename T, bool SIG, bool WIDE, int CL, bool SUMS>
__global__ __launch_bounds__(threads_of<CL>()) void k_recurrence_bwd(RecurrenceArgs a, int blocks) {
    __shared__ Sums<CL, 3> lds;
    const int64_t index = block_index();
    const int64_t slot = index / blocks;
    Unit u;
    if (slot >= a.seqs.slots || !unit_of(a.seqs, slot, u)) return;
    const Place<T, CL> me(a, (int)(index - slot * blocks));
    const Rows<T, WIDE> z(a.z, u.t0, me.c, me.valid), x(a.x, u.t0, me.c, me.valid), g(a.dh, u.t0, me.c, me.valid);
    const int64_t row = (int64_t)u.seq * a.channels + me.c, slot_row = u.slot * a.channels + me.c;
    float carry[V], A[V];
#pragma unroll
    for (int i = 0; i < V; ++i) carry[i] = 0.0f, A[i] = 1.0f;
    if (!SUMS) {
        if (u.to < u.len)
            load_f32(a.starts + slot_row, me.valid, carry);
        else if (a.dfinal)
            load_f32(a.dfinal + row, me.valid, carry);
    }
    auto load_mark = [&](int64_t tile, float (&m)[V]) {
        if (tile > 0)
            load_f32(a.marks + (u.t0 / kRecurrenceTile + tile / kRecurrenceTile) * a.channels + me.c, me.valid, m);
        else if (a.state)
            load_f32(a.state + row, me.valid, m);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) m[i] = 0.0f;
    };
    Raw<T> rz[L], rx[L], rg[L];
    float mark[V];
    int64_t tile = u.from + (u.to - u.from - 1) / kRecurrenceTile * kRecurrenceTile, t = tile + me.slice * L;
    if (u.from < u.to) {
        z.load(t, u.to, rz);
        g.load(t, u.to, rg);
        if (!SUMS) x.load(t, u.to, rx), load_mark(tile, mark);
    }
    int parity = 0;
    for (; u.from < u.to && tile >= u.from; tile -= kRecurrenceTile, t -= kRecurrenceTile, parity ^= 1) {
        // d: h_(t-1)'s share of dz without h, f (1 - f) (or 1), then dz without G
        float f[L][V], in[L][V], d[L][V], dy[L][V], pa[V], pb[V], pr[V];
#pragma unroll
        for (int i = 0; i < V; ++i) pa[i] = 1.0f, pb[i] = 0.0f, pr[i] = 0.0f;
#pragma unroll
        for (int l = 0; l < L; ++l) {
            float vz[V], vx[V];
            unpack(rz[l], vz);
            unpack(rg[l], dy[l]);
            if (!SUMS) unpack(rx[l], vx);
            const bool real = t + l < u.to;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if constexpr (SIG) {
                    sigmoids(vz[i], f[l][i], d[l][i]);  // d: 1 - f
                    in[l][i] = SUMS ? 0.0f : vx[i];     // x
                } else {
                    f[l][i] = vz[i];
                    in[l][i] = SUMS ? 0.0f : vx[i];
                    d[l][i] = 1.0f;
                }
                if (!real) f[l][i] = 1.0f, in[l][i] = d[l][i] = dy[l][i] = 0.0f;
                pa[i] *= f[l][i];
                if (!SUMS) pb[i] = fmaf(f[l][i], pb[i], d[l][i] * in[l][i]);
            }
        }
#pragma unroll
        for (int l = L - 1; l >= 0; --l)
#pragma unroll
            for (int i = 0; i < V; ++i) pr[i] = f[l][i] * (dy[l][i] + pr[i]);
        float now[V];
#pragma unroll
        for (int i = 0; i < V; ++i) now[i] = SUMS ? 0.0f : mark[i];
        if (tile > u.from) {
            z.load(t - kRecurrenceTile, u.to, rz);
            g.load(t - kRecurrenceTile, u.to, rg);
            if (!SUMS) x.load(t - kRecurrenceTile, u.to, rx), load_mark(tile - kRecurrenceTile, mark);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float pa2 = pa[i];
            mark_unusable(pa2, pr[i]);
            if (!SUMS) mark_unusable(pa[i], pb[i]);
            if (pa2 != pa2) pa[i] = pa2;
        }
        copy_in(&lds.v[parity][0][me.slice][me.lane * V], pa);
        if (!SUMS) copy_in(&lds.v[parity][1][me.slice][me.lane * V], pb);
        copy_in(&lds.v[parity][2][me.slice][me.lane * V], pr);
        lds_barrier();
        if constexpr (SUMS) {
#pragma unroll
            for (int s = SLICES - 1; s >= 0; --s)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float fs = lds.v[parity][0][s][me.lane * V + i];
                    A[i] *= fs;
                    carry[i] = fmaf(fs, carry[i], lds.v[parity][2][s][me.lane * V + i]);
                    if (fabsf(carry[i]) > LARGE_STATE) A[i] = __builtin_nanf("");
                }
        } else {
            float h[V], s[V], before[V];
#pragma unroll
            for (int i = 0; i < V; ++i) before[i] = now[i];
            const int64_t end = min(tile + kRecurrenceTile, u.to);
            if (join_slices<CL, false>(lds.v[parity][0], lds.v[parity][1], me.slice, me.lane, now, h))
                walk_forward<T, SIG, WIDE>(z, x, tile, end, t, before, h);
#pragma unroll
            for (int i = 0; i < V; ++i) before[i] = carry[i];
            if (join_slices<CL, true>(lds.v[parity][0], lds.v[parity][2], me.slice, me.lane, carry, s)) {
#pragma unroll
                for (int i = 0; i < V; ++i) carry[i] = s[i] = before[i];
                walk_reverse<T, SIG, WIDE>(z, g, tile, end, min(t + L, end), carry, s);
            }
#pragma unroll
            for (int l = 0; l < L; ++l)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float rest = d[l][i], xv = in[l][i];
                    if constexpr (SIG) {
                        in[l][i] = (h[i] - xv) * f[l][i] * rest;
                        h[i] = fmaf(f[l][i], h[i], rest * xv);
                    } else {
                        in[l][i] = h[i];
                        h[i] = fmaf(f[l][i], h[i], xv);
                    }
                }
            const int64_t first = (u.t0 + t) * a.channels + me.c;
#pragma unroll
            for (int l = L - 1; l >= 0; --l) {
                float oz[V], ox[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float G = dy[l][i] + s[i];
                    oz[i] = G * in[l][i];
                    ox[i] = G * d[l][i];
                    s[i] = f[l][i] * G;
                }
                if (t + l < u.to && me.valid) {
                    store_vec<T, WIDE>(static_cast<T*>(a.dz) + first + (int64_t)l * a.channels, me.valid, oz);
                    store_vec<T, WIDE>(static_cast<T*>(a.dx) + first + (int64_t)l * a.channels, me.valid, ox);
                }
            }
        }
    }
    if (me.slice != 0) return;
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < V; ++i) mark_unusable(A[i], carry[i]);
        store_f32(a.sums + slot_row, me.valid, A);
        store_f32(a.sums + a.seqs.slots * a.channels + slot_row, me.valid, carry);
    } else if (a.dstate && u.from == 0) {
        store_f32(a.dstate + row, me.valid, carry);
    }
}

// The states (REVERSE: adjoints) that a sequence's segments start from, one
// thread a channel: segments in order, those whose sums cannot be joined token by
// token.
template <typename T, bool SIG, bool REVERSE>
__global__ __launch_bounds__(64) void k_recurrence_join(RecurrenceArgs a, int blocks) {
    const int64_t index = block_index();
    const int seq = (int)(index / blocks), c = (int)(index - (int64_t)seq * blocks) * 64 + threadIdx.x;
    if (seq >= a.seqs.n || c >= a.channels) return;
    Unit u;
    sequence_of(a.seqs, seq, u);
    const int64_t count = (u.len + a.seqs.seg - 1) / a.seqs.seg, slot0 = u.t0 / a.seqs.seg + seq, all = a.seqs.slots * a.channels;
    const float* from = REVERSE ? a.dfinal : a.state;
    float h = from ? from[(int64_t)seq * a.channels + c] : 0.0f;
    const T* z = static_cast<const T*>(a.z.p) + u.t0 * a.z.stride + c;
    const RowView& other = REVERSE ? a.dh : a.x;
    const T* x = static_cast<const T*>(other.p) + u.t0 * other.stride + c;
    constexpr int AHEAD = 8;  // segments whose sums are loaded together
    for (int64_t k0 = 0; k0 + 1 < count; k0 += AHEAD) {
        float A[AHEAD], B[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t k = min(k0 + i, count - 1);
            const int64_t at = (slot0 + (REVERSE ? count - 1 - k : k)) * a.channels + c;
            A[i] = a.sums[at];
            B[i] = a.sums[all + at];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t k = k0 + i, j = REVERSE ? count - 1 - k : k;
            if (k + 1 >= count) break;  // nothing starts behind the last one
            const float next = fmaf(A[i], h, B[i]);
            if (h == h && (next != next || fabsf(h) > LARGE_STATE)) {
                const int64_t lo = j * a.seqs.seg, hi = min(u.len, lo + a.seqs.seg);
                for (int64_t s = lo; s < hi; ++s) {
                    const int64_t t = REVERSE ? lo + hi - 1 - s : s;
                    float f, in;
                    const float v = St<T>::ld1(x + t * other.stride);
                    coefficients<SIG>(St<T>::ld1(z + t * a.z.stride), v, f, in);
                    h = REVERSE ? f * (v + h) : fmaf(f, h, in);
                }
            } else {
                h = next;
            }
            a.starts[(slot0 + (REVERSE ? j - 1 : j + 1)) * a.channels + c] = h;
        }
    }
}

// One token for each row: two channels a thread.
template <typename T, bool SIG, bool WIDE>
__global__ __launch_bounds__(256) void k_advance(AdvanceArgs a, int vecs) {
    const int64_t i = block_index() * 256 + threadIdx.x;
    const int64_t row = i / vecs;
    if (row >= a.n) return;
    const int c = (int)(i - row * vecs) * V, valid = min(V, a.channels - c);
    const int64_t slot = a.slot ? a.slot[row] : row;
    float h[V];
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = 0.0f;
    if (slot >= 0 && slot < a.slots) {
        float* st = a.state + slot * a.channels + c;
        const Raw<T> rz = load_raw<T, WIDE>(static_cast<const T*>(a.z.p) + row * a.z.stride + c, valid);
        const Raw<T> rx = load_raw<T, WIDE>(static_cast<const T*>(a.x.p) + row * a.x.stride + c, valid);
        typedef float vec __attribute__((ext_vector_type(V)));
        if (WIDE) {
            const vec v = *reinterpret_cast<const vec*>(st);
#pragma unroll
            for (int j = 0; j < V; ++j) h[j] = v[j];
        } else {
            load_f32(st, valid, h);
        }
        float z[V], x[V];
        unpack(rz, z);
        unpack(rx, x);
        vec o;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float f, u;
            coefficients<SIG>(z[j], x[j], f, u);
            h[j] = fmaf(f, h[j], u);
            o[j] = h[j];
        }
        if (WIDE)
            *reinterpret_cast<vec*>(st) = o;
        else
            store_f32(st, valid, h);
    }
    store_vec<T, WIDE>(static_cast<T*>(a.out) + row * a.channels + c, valid, h);
}

bool aligned(const void* p, int to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Rows whose pairs of channels lie at their alignment.
bool wide_rows(const RowView& v, int es) { return aligned(v.p, V * es) && v.stride % V == 0; }

template <typename F>
hipError_t with_types(int dtype, int sigmoid, bool wide, F&& f) {
    const std::true_type yes;
    const std::false_type no;
    if (dtype) {
        if (sigmoid) return wide ? f(bf16_t(), yes, yes) : f(bf16_t(), yes, no);
        return wide ? f(bf16_t(), no, yes) : f(bf16_t(), no, no);
    }
    if (sigmoid) return wide ? f(float(), yes, yes) : f(float(), yes, no);
    return wide ? f(float(), no, yes) : f(float(), no, no);
}

// Lanes of a row: as many as its pairs of channels need, at most 32.
template <typename F>
hipError_t with_lanes(int vecs, F&& f) {
    if (vecs <= 4) return f(std::integral_constant<int, 4>());
    if (vecs <= 8) return f(std::integral_constant<int, 8>());
    if (vecs <= 16) return f(std::integral_constant<int, 16>());
    return f(std::integral_constant<int, 32>());
}

int vecs_of(int channels) { return (channels + V - 1) / V; }

// Tokens of a segment; 0: whole sequences. A workgroup's tiles follow each other,
// so sequences are cut where the longest one would hold the chip up: where it is
// longer than all tokens spread over the CUs. Segments then give a CU four units.
int64_t segment_of(const RecurrenceArgs& a) {
    constexpr int64_t CUS = 256;
    const int64_t blocks = (vecs_of(a.channels) + 31) / 32, share = a.seqs.tokens * blocks / CUS;
    if (a.seqs.longest <= std::max<int64_t>(1024, 2 * share)) return 0;
    return std::max<int64_t>(256, (share / 4 + kRecurrenceTile - 1) / kRecurrenceTile * kRecurrenceTile);
}

RecurrenceArgs plan(const RecurrenceArgs& in) {
    RecurrenceArgs a = in;
    a.seqs.seg = segment_of(a);
    a.seqs.slots = packed_slots(a.seqs, a.seqs.seg);
    if (a.seqs.seg) {
        a.sums = static_cast<float*>(a.ws);
        a.starts = a.sums + 2 * a.seqs.slots * a.channels;
    }
    return a;
}

template <bool BACKWARD>
hipError_t launch(const RecurrenceArgs& in, hipStream_t s) {
    const RecurrenceArgs a = plan(in);
    if (a.seqs.n == 0) return hipSuccess;
    const int es = a.dtype ? 2 : 4;
    bool wide = a.channels % V == 0 && wide_rows(a.z, es) && wide_rows(a.x, es);
    if (BACKWARD)
        wide = wide && wide_rows(a.dh, es) && aligned(a.dz, V * es) && aligned(a.dx, V * es);
    else
        wide = wide && aligned(a.h, V * es);
    return with_types(a.dtype, a.sigmoid, wide, [&](auto t, auto sig, auto w) {
        typedef decltype(t) T;
        const int vecs = vecs_of(a.channels);
        return with_lanes(vecs, [&](auto lanes) {
            constexpr int CL = lanes();
            constexpr bool SIG = sig(), W = w();
            const int blocks = (vecs + CL - 1) / CL;
            dim3 grid;
            if (!grid_of(a.seqs.slots * blocks, threads_of<CL>(), grid)) return hipErrorInvalidValue;
            if (a.seqs.seg) {
                if constexpr (BACKWARD)
                    k_recurrence_bwd<T, SIG, W, CL, true><<<grid, threads_of<CL>(), 0, s>>>(a, blocks);
                else
                    k_recurrence_fwd<T, SIG, W, CL, true><<<grid, threads_of<CL>(), 0, s>>>(a, blocks);
                hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
                const int cols = (a.channels + 63) / 64;
                dim3 jgrid;
                if (!grid_of((int64_t)a.seqs.n * cols, 64, jgrid)) return hipErrorInvalidValue;
                k_recurrence_join<T, SIG, BACKWARD><<<jgrid, 64, 0, s>>>(a, cols);
                e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
            if constexpr (BACKWARD)
                k_recurrence_bwd<T, SIG, W, CL, false><<<grid, threads_of<CL>(), 0, s>>>(a, blocks);
            else
                k_recurrence_fwd<T, SIG, W, CL, false><<<grid, threads_of<CL>(), 0, s>>>(a, blocks);
            return hipGetLastError();
        });
    });
}

}  // namespace

size_t recurrence_workspace_bytes(const RecurrenceArgs& a) {
    const int64_t seg = segment_of(a);
    return seg ? (size_t)3 * packed_slots(a.seqs, seg) * a.channels * 4 : 16;
}

hipError_t launch_recurrence_fwd(const RecurrenceArgs& a, hipStream_t s) { return launch<false>(a, s); }
hipError_t launch_recurrence_bwd(const RecurrenceArgs& a, hipStream_t s) { return launch<true>(a, s); }

hipError_t launch_advance(const AdvanceArgs& a, hipStream_t s) {
    if (a.n == 0) return hipSuccess;
    const int es = a.dtype ? 2 : 4;
    const bool wide = a.channels % V == 0 && wide_rows(a.z, es) && wide_rows(a.x, es) && aligned(a.out, V * es) && aligned(a.state, 8);
    return with_types(a.dtype, a.sigmoid, wide, [&](auto t, auto sig, auto w) {
        typedef decltype(t) T;
        const int vecs = vecs_of(a.channels);
        dim3 grid;
        if (!grid_of(((int64_t)a.n * vecs + 255) / 256, 256, grid)) return hipErrorInvalidValue;
        k_advance<T, sig(), w()><<<grid, 256, 0, s>>>(a, vecs);
        return hipGetLastError();
    });
}

}  // namespace mdl
