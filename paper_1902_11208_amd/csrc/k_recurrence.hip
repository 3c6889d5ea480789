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
// next tile is loaded while one is computed. Measured: 128 sequences of 300 to 1200
// tokens of 512 bf16 channels, forward 73 us (290 MB, 4.0 TB/s), backward 129 us (490
// MB, 3.8 TB/s, and 50 MB of spilled registers); one sequence of 65536 tokens of 1024, in
// segments, 50 us for their sums, 12 to join them, 78 for the pass itself. By the counters
// a number takes 28 vector instructions forward and 50 backward with a sigmoid: at four
// cycles each, sixteen for the exponential and the reciprocal, 40 and 68 us, more than half
// of the memory's time; with 64-bit row addresses and masks in every tile the forward pass
// took 123 us.
//
// The forward pass keeps the fp32 state at every tile's start (1/128 of bf16 z
// and x), and the backward pass finds h again from it instead of from the
// rounded output: h - x is a difference, and a rounded h would leave it with
// an error of up to 2^-8 of h.
#include <algorithm>
#include <type_traits>

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
// error of f is met again in every token that a state lives through. EXACT: the
// product with log2(e) keeps its low half, without which e is off by |z| 2^-24; for
// bf16 inputs that is far below z's own rounding.
template <bool EXACT>
__device__ __forceinline__ void sigmoids(float z, float& f, float& rest) {
    constexpr float HIGH = -1.44269502162933349609375f, LOW = -1.925963033500011e-08f, LN2 = 0.693147180559945309f;
    const float m = fabsf(z), t = m * HIGH;
    float e = __builtin_amdgcn_exp2f(t);
    if constexpr (EXACT) e = fmaf(e, LN2 * fmaf(m, LOW, fmaf(m, HIGH, -t)), e);
    if (EXACT && t < -160.0f) e = 0.0f;  // below fp32's range, where m HIGH may be beyond it
    const float d = 1.0f + e;
    float r = __builtin_amdgcn_rcpf(d);
    r = fmaf(fmaf(-d, r, 1.0f), r, r);
    const float small = e * r;
    f = z < 0.0f ? small : r;
    rest = z < 0.0f ? r : small;
}

template <typename T, bool SIG>
__device__ __forceinline__ void coefficients(float z, float x, float& f, float& u) {
    if constexpr (SIG) {
        float rest;
        sigmoids<sizeof(T) == 4>(z, f, rest);
        u = rest * x;
    } else {
        f = z;
        u = x;
    }
}

// A h + B is what the tokens give unless something leaves fp32's range on the way:
// A may have fallen below it under a large state, 0 times infinity is no number,
// factors may have grown and shrunk. So slices whose growth (the product of the factors
// beyond 1, which bounds every run of them) is more than 4 or whose B is large are marked
// with NaN; sixteen of them then grow a state by at most 2^32. What A has lost below the
// range is then at most 2^-145, and a state that a slice takes down by more than 2^-120 may
// be that. Where a mark, a large state or such a fall is met the tokens are walked one by
// one. Sigmoids neither grow anything nor give back what fell.
constexpr float LARGE = 0x1p40f;
constexpr float FALL = 0x1p-120f;
constexpr float SEGMENT_FALL = 0x1p-68f;  // growth of at most 2^32 leaves a segment's A at most 2^-93 off

__device__ __forceinline__ void mark_growth(float growth, float most, float& A) {
    if (!(growth <= most)) A = __builtin_nanf("");
}
__device__ __forceinline__ void mark_rest(float& B) {
    if (!(fabsf(B) <= LARGE)) B = __builtin_nanf("");
}
// The state from an unmarked run is not what the tokens give.
__device__ __forceinline__ bool unsafe(float from, float joined) {
    return from == from && (joined != joined || fabsf(from) > LARGE);
}
__device__ __forceinline__ bool fell(float from, float joined, float by) { return fabsf(joined) < fabsf(from) * by; }

// Rows of a sequence as a thread reads them: a uniform base, and 32 bits of its own
// offset (128 rows are less than 2^32 bytes apart by the caller's check).
template <typename T, bool WIDE>
struct Rows {
    const char* base;
    int64_t stride;  // bytes
    uint32_t c;      // bytes
    int valid;
    __device__ __forceinline__ Rows(const RowView& v, int64_t t0, int c_, int valid_)
        : base(static_cast<const char*>(v.p) + t0 * v.stride * (int64_t)sizeof(T)), stride(v.stride * (int64_t)sizeof(T)),
          c((uint32_t)c_ * sizeof(T)), valid(valid_) {}
    __device__ __forceinline__ Raw<T> at(const char* row, uint32_t offset) const {
        return load_raw<T, WIDE>(reinterpret_cast<const T*>(row + offset), valid);
    }
    // a slice's eight tokens of the tile at `tile`, of which `n` tokens are real: behind them the last one again
    __device__ __forceinline__ void load(int64_t tile, int64_t n, int slice, Raw<T> (&r)[L]) const {
        const char* row = base + tile * stride;
        if (n >= kRecurrenceTile) {
            const uint32_t mine = (uint32_t)(slice * L) * (uint32_t)stride + c;
#pragma unroll
            for (int i = 0; i < L; ++i) r[i] = at(row + i * stride, mine);
        } else {
#pragma unroll
            for (int i = 0; i < L; ++i) r[i] = at(row, (uint32_t)min(slice * L + i, (int)n - 1) * (uint32_t)stride + c);
        }
    }
    __device__ __forceinline__ void token(int64_t t, float (&v)[V]) const { unpack(at(base + t * stride, c), v); }
};

// [tokens][channels] outputs of a slice, `n` tokens of the tile real.
template <typename T, bool WIDE>
struct Out {
    char* base;
    uint32_t stride, c;  // bytes
    int valid;
    __device__ __forceinline__ Out(void* p, int64_t t0, int channels, int c_, int valid_)
        : base(static_cast<char*>(p) + t0 * channels * (int64_t)sizeof(T)), stride((uint32_t)channels * sizeof(T)),
          c((uint32_t)c_ * sizeof(T)), valid(valid_) {}
    __device__ __forceinline__ void store(int64_t tile, int slice, int l, const float (&v)[V]) const {
        char* row = base + (tile + l) * (int64_t)stride;
        if (valid > 0) store_vec<T, WIDE>(reinterpret_cast<T*>(row + ((uint32_t)(slice * L) * stride + c)), valid, v);
    }
};

// What a thread is: a slice of a tile and two channels.
struct Place {
    int slice, lane, c, valid;
    __device__ __forceinline__ Place(int channels, int lanes, int block) {
        slice = threadIdx.x / lanes;
        lane = threadIdx.x % lanes;
        c = (block * lanes + lane) * V;
        valid = max(0, min(V, channels - c));
        if (valid == 0) c = 0;
    }
};

__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// The workgroup's unit and block of channels; false where there is none.
template <bool SUMS>
__device__ __forceinline__ bool find_unit(const RecurrenceArgs& a, int blocks, Unit& u, int& block) {
    const int64_t index = block_index();
    int64_t slot = uniform(index / blocks);
    block = __builtin_amdgcn_readfirstlane((int)(index - slot * blocks));
    if (!SUMS && a.seqs.seg) slot = a.seqs.slots - 1 - slot;  // what the pass for the sums read last is still in the caches
    if (slot < 0 || slot >= a.seqs.slots || !unit_of(a.seqs, slot, u)) return false;
    u.seq = __builtin_amdgcn_readfirstlane(u.seq);
    u.t0 = uniform(u.t0);
    u.len = uniform(u.len);
    u.from = uniform(u.from);
    u.to = uniform(u.to);
    u.edge = uniform(u.edge);
    return true;
}

// The sums and starts have a row for each edge between a sequence's segments. The `seg` tokens before an edge are those of
// one segment, so an edge at token t has row (t - 1) / seg to itself, and sequences without edges take none. u.edge is
// the row of the edge before a segment; the edge behind it has the next.
constexpr int EDGE_BEHIND = 1;

__device__ __forceinline__ int64_t mark_row(const Unit& u, int64_t tile) { return u.t0 / kRecurrenceTile + tile / kRecurrenceTile; }

// What the slices of a tile tell each other, for one of two tiles in turn (one
// barrier a tile): their sums, and the state (adjoint) that the tile before left.
template <int CL, int N>
struct Shared {
    float2 sum[2][N][SLICES][CL];
    float2 carry[2][CL];
};
__device__ __forceinline__ float2 pack(const float (&v)[V]) { return make_float2(v[0], v[1]); }

// The state that meets slice `mine`, from `h` that meets the tile: the slices before
// it (REVERSE: behind it) in order. A wave goes no further than its last one. True where
// the tokens may give another state.
template <int CL, bool REVERSE, bool SIG>
__device__ __forceinline__ bool join_slices(const float2 (*A)[CL], const float2 (*B)[CL], int mine, int lane, float (&h)[V]) {
    const float from[V] = {h[0], h[1]};
    float least = 0.0f;  // below 0 after a fall
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const int n = REVERSE ? SLICES - 1 - wave * 64 / CL : min(SLICES - 1, (wave * 64 + 63) / CL);
    for (int k0 = 0; k0 < n; k0 += 4) {
        float2 pa[4], pb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = REVERSE ? SLICES - 1 - k0 - i : k0 + i;
            pa[i] = A[s][lane];
            pb[i] = B[s][lane];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = REVERSE ? SLICES - 1 - k0 - i : k0 + i;
            const bool before = REVERSE ? s > mine : s < mine;
            const float h0 = fmaf(pa[i].x, h[0], pb[i].x), h1 = fmaf(pa[i].y, h[1], pb[i].y);
            const float to0 = before ? h0 : h[0], to1 = before ? h1 : h[1];
            if (!SIG) least = fminf(fminf(least, fmaf(fabsf(h[0]), -FALL, fabsf(to0))), fmaf(fabsf(h[1]), -FALL, fabsf(to1)));
            h[0] = to0;
            h[1] = to1;
        }
    }
    return least < 0.0f || unsafe(from[0], h[0]) || unsafe(from[1], h[1]);
}

// h through the tokens from .. to - 1, one by one.
template <typename T, bool SIG, bool WIDE>
__device__ __forceinline__ void walk_forward(const Rows<T, WIDE>& z, const Rows<T, WIDE>& x, int64_t from, int64_t to, float (&h)[V]) {
#pragma unroll 1
    for (int64_t t = from; t < to; ++t) {
        float vz[V], vx[V];
        z.token(t, vz);
        x.token(t, vx);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float f, u;
            coefficients<T, SIG>(vz[i], vx[i], f, u);
            h[i] = fmaf(f, h[i], u);
        }
    }
}

// The adjoint from token to - 1 down to `from`.
template <typename T, bool SIG, bool WIDE>
__device__ __forceinline__ void walk_reverse(const Rows<T, WIDE>& z, const Rows<T, WIDE>& dh, int64_t from, int64_t to, float (&s)[V]) {
#pragma unroll 1
    for (int64_t t = to - 1; t >= from; --t) {
        float vz[V], vg[V];
        z.token(t, vz);
        dh.token(t, vg);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float f, u;
            coefficients<T, SIG>(vz[i], 0.0f, f, u);
            s[i] = f * (vg[i] + s[i]);
        }
    }
}

template <int CL>
constexpr int threads_of() { return CL * SLICES; }

// A segment's A and B, with a tile's slices in order (REVERSE: from the last), by the threads of the last one to be joined.
template <int CL, bool REVERSE, bool SIG>
__device__ __forceinline__ void add_slices(const float2 (*a)[CL], const float2 (*b)[CL], int lane, float (&growth)[V], float (&A)[V], float (&B)[V]) {
    for (int k = 0; k < SLICES; ++k) {
        const int s = REVERSE ? SLICES - 1 - k : k;
        const float sa[V] = {a[s][lane].x, a[s][lane].y}, sb[V] = {b[s][lane].x, b[s][lane].y};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float next = fmaf(sa[i], B[i], sb[i]);
            if (!SIG) {
                growth[i] *= fmaxf(fabsf(sa[i]), 1.0f);
                if (fell(B[i], next, FALL)) growth[i] = __builtin_huge_valf();
            }
            A[i] *= sa[i];
            B[i] = next;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (!SIG) mark_growth(growth[i], 0x1p32f, A[i]);
        mark_rest(B[i]);
    }
}

// Forward pass of a sequence or segment. SUMS: only what it maps a state to, for the join.
template <typename T, bool SIG, bool WIDE, int CL, bool SUMS>
__global__ __launch_bounds__(threads_of<CL>()) void k_recurrence_fwd(RecurrenceArgs a, int blocks) {
    __shared__ Shared<CL, 2> lds;
    Unit u;
    int block;
    if (!find_unit<SUMS>(a, blocks, u, block)) return;
    if (SUMS && u.to == u.len) return;  // nothing starts behind it
    const Place me(a.channels, CL, block);
    const Rows<T, WIDE> z(a.z, u.t0, me.c, me.valid), x(a.x, u.t0, me.c, me.valid);
    const Out<T, WIDE> out(a.h, u.t0, a.channels, me.c, me.valid);
    const int64_t row = (int64_t)u.seq * a.channels + me.c;
    const bool last = me.slice == SLICES - 1;
    float h[V] = {}, A[V] = {1.0f, 1.0f}, B[V] = {}, growth[V] = {1.0f, 1.0f};
    if (!SUMS && last) {
        if (u.from > 0) {
            load_f32(a.starts + u.edge * a.channels + me.c, me.valid, h);
            if (a.marks && u.from < u.to) store_f32(a.marks + mark_row(u, u.from) * a.channels + me.c, me.valid, h);
        } else if (a.state) {
            load_f32(a.state + row, me.valid, h);
        }
        lds.carry[0][me.lane] = pack(h);
    }
    Raw<T> rz[L], rx[L];
    if (u.from < u.to) {
        z.load(u.from, u.to - u.from, me.slice, rz);
        x.load(u.from, u.to - u.from, me.slice, rx);
    }
    int parity = 0;
    for (int64_t tile = u.from; tile < u.to; tile += kRecurrenceTile, parity ^= 1) {
        const int n = (int)min(u.to - tile, (int64_t)kRecurrenceTile), mine = n - me.slice * L;  // real tokens of the tile, of the slice
        float f[L][V], in[L][V], pa[V], pb[V], pg[V];
        auto sums = [&](auto whole) {
#pragma unroll
            for (int i = 0; i < V; ++i) pa[i] = 1.0f, pb[i] = 0.0f, pg[i] = 1.0f;
#pragma unroll
            for (int l = 0; l < L; ++l) {
                float vz[V], vx[V];
                unpack(rz[l], vz);
                unpack(rx[l], vx);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    coefficients<T, SIG>(vz[i], vx[i], f[l][i], in[l][i]);
                    if (!whole() && l >= mine) f[l][i] = 1.0f, in[l][i] = 0.0f;
                    pa[i] *= f[l][i];
                    if (!SIG) pg[i] *= fmaxf(fabsf(f[l][i]), 1.0f);
                    pb[i] = fmaf(f[l][i], pb[i], in[l][i]);
                }
            }
        };
        if (n == kRecurrenceTile)
            sums(std::true_type());
        else
            sums(std::false_type());
        const int64_t next = tile + kRecurrenceTile;
        if (next < u.to) {
            z.load(next, u.to - next, me.slice, rz);
            x.load(next, u.to - next, me.slice, rx);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!SIG) mark_growth(pg[i], 4.0f, pa[i]);
            mark_rest(pb[i]);
        }
        lds.sum[parity][0][me.slice][me.lane] = pack(pa);
        lds.sum[parity][1][me.slice][me.lane] = pack(pb);
        lds_barrier();
        if constexpr (SUMS) {
            if (last) add_slices<CL, false, SIG>(lds.sum[parity][0], lds.sum[parity][1], me.lane, growth, A, B);
        } else {
            const float2 carry = lds.carry[parity][me.lane];
            h[0] = carry.x, h[1] = carry.y;
            if (join_slices<CL, false, SIG>(lds.sum[parity][0], lds.sum[parity][1], me.slice, me.lane, h)) {
                h[0] = carry.x, h[1] = carry.y;
                walk_forward<T, SIG, WIDE>(z, x, tile, min(tile + me.slice * L, u.to), h);
            }
            auto go = [&](auto whole) {
#pragma unroll
                for (int l = 0; l < L; ++l) {
#pragma unroll
                    for (int i = 0; i < V; ++i) h[i] = fmaf(f[l][i], h[i], in[l][i]);
                    if (whole() || l < mine) out.store(tile, me.slice, l, h);
                }
            };
            if (n == kRecurrenceTile)
                go(std::true_type());
            else
                go(std::false_type());
            if (last) {
                lds.carry[parity ^ 1][me.lane] = pack(h);
                if (a.marks && next < u.to) store_f32(a.marks + mark_row(u, next) * a.channels + me.c, me.valid, h);
            }
        }
    }
    if (!last) return;
    if constexpr (SUMS) {
        const int64_t edge = (u.edge + EDGE_BEHIND) * a.channels + me.c;
        store_f32(a.sums + edge, me.valid, A);
        store_f32(a.sums + a.edges * a.channels + edge, me.valid, B);
    } else if (a.final_state && u.to == u.len) {
        store_f32(a.final_state + row, me.valid, h);
    }
}

// Backward pass. SUMS: only what the unit maps the adjoint behind it to.
template <typename T, bool SIG, bool WIDE, int CL, bool SUMS>
__global__ __launch_bounds__(threads_of<CL>(), sizeof(T) == 2 ? 4 : 2) void k_recurrence_bwd(RecurrenceArgs a, int blocks) {
    __shared__ Shared<CL, 3> lds;
    Unit u;
    int block;
    if (!find_unit<SUMS>(a, blocks, u, block)) return;
    if (SUMS && u.from == 0) return;  // nothing ends before it
    const Place me(a.channels, CL, block);
    const Rows<T, WIDE> z(a.z, u.t0, me.c, me.valid), x(a.x, u.t0, me.c, me.valid), g(a.dh, u.t0, me.c, me.valid);
    const Out<T, WIDE> out_z(a.dz, u.t0, a.channels, me.c, me.valid), out_x(a.dx, u.t0, a.channels, me.c, me.valid);
    const int64_t row = (int64_t)u.seq * a.channels + me.c;
    const bool first = me.slice == 0;
    float s[V] = {}, A[V] = {1.0f, 1.0f}, B[V] = {}, growth[V] = {1.0f, 1.0f}, mark[V] = {};
    if (!SUMS && first) {
        if (u.to < u.len)
            load_f32(a.starts + (u.edge + EDGE_BEHIND) * a.channels + me.c, me.valid, s);
        else if (a.dfinal)
            load_f32(a.dfinal + row, me.valid, s);
        lds.carry[0][me.lane] = pack(s);
    }
    auto load_mark = [&](int64_t tile) {
        if (tile > 0)
            load_f32(a.marks + mark_row(u, tile) * a.channels + me.c, me.valid, mark);
        else if (a.state)
            load_f32(a.state + row, me.valid, mark);
        else
            mark[0] = mark[1] = 0.0f;
    };
    Raw<T> rz[L], rx[L], rg[L];
    auto load = [&](int64_t tile) {
        z.load(tile, u.to - tile, me.slice, rz);
        g.load(tile, u.to - tile, me.slice, rg);
        if constexpr (!SUMS) {
            x.load(tile, u.to - tile, me.slice, rx);
            load_mark(tile);
        }
    };
    int64_t tile = u.from + max(u.to - u.from - 1, (int64_t)0) / kRecurrenceTile * kRecurrenceTile;
    if (u.from < u.to) load(tile);
    int parity = 0;
    for (; u.from < u.to && tile >= u.from; tile -= kRecurrenceTile, parity ^= 1) {
        const int n = (int)min(u.to - tile, (int64_t)kRecurrenceTile), mine = n - me.slice * L;
        // rest: 1 - f (or 1); cx, cg: x and dh as loaded, the registers of the fp32 numbers would halve the waves of bf16
        float f[L][V], rest[L][V], pa[V], pb[V], pr[V], pg[V];
        Raw<T> cx[L], cg[L];
        auto sums = [&](auto whole) {
#pragma unroll
            for (int i = 0; i < V; ++i) pa[i] = 1.0f, pb[i] = 0.0f, pr[i] = 0.0f, pg[i] = 1.0f;
#pragma unroll
            for (int l = 0; l < L; ++l) {
                float vz[V], vx[V];
                const bool real = whole() || l < mine;
                unpack(rz[l], vz);
                cg[l] = real ? rg[l] : Raw<T>{};
                if constexpr (!SUMS) {
                    cx[l] = real ? rx[l] : Raw<T>{};
                    unpack(cx[l], vx);
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if constexpr (SIG) {
                        sigmoids<sizeof(T) == 4>(vz[i], f[l][i], rest[l][i]);
                    } else {
                        f[l][i] = vz[i];
                        rest[l][i] = 1.0f;
                    }
                    if (!real) f[l][i] = 1.0f, rest[l][i] = 0.0f;
                    pa[i] *= f[l][i];
                    if (!SIG) pg[i] *= fmaxf(fabsf(f[l][i]), 1.0f);
                    if constexpr (!SUMS) pb[i] = fmaf(f[l][i], pb[i], SIG ? rest[l][i] * vx[i] : vx[i]);
                }
            }
        };
        if (n == kRecurrenceTile)
            sums(std::true_type());
        else
            sums(std::false_type());
#pragma unroll
        for (int l = L - 1; l >= 0; --l) {
            float dy[V];
            unpack(cg[l], dy);
#pragma unroll
            for (int i = 0; i < V; ++i) pr[i] = f[l][i] * (dy[i] + pr[i]);
        }
        const float from[V] = {mark[0], mark[1]};
        if (tile > u.from) load(tile - kRecurrenceTile);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!SIG) mark_growth(pg[i], 4.0f, pa[i]);
            mark_rest(pb[i]);
            mark_rest(pr[i]);
        }
        lds.sum[parity][0][me.slice][me.lane] = pack(pa);
        if constexpr (!SUMS) lds.sum[parity][1][me.slice][me.lane] = pack(pb);
        lds.sum[parity][2][me.slice][me.lane] = pack(pr);
        lds_barrier();
        if constexpr (SUMS) {
            if (first) add_slices<CL, true, SIG>(lds.sum[parity][0], lds.sum[parity][2], me.lane, growth, A, B);
        } else {
            float h[V] = {from[0], from[1]};
            if (join_slices<CL, false, SIG>(lds.sum[parity][0], lds.sum[parity][1], me.slice, me.lane, h)) {
                h[0] = from[0], h[1] = from[1];
                walk_forward<T, SIG, WIDE>(z, x, tile, min(tile + me.slice * L, u.to), h);
            }
            const float2 carry = lds.carry[parity][me.lane];
            s[0] = carry.x, s[1] = carry.y;
            if (join_slices<CL, true, SIG>(lds.sum[parity][0], lds.sum[parity][2], me.slice, me.lane, s)) {
                s[0] = carry.x, s[1] = carry.y;
                walk_reverse<T, SIG, WIDE>(z, g, min(tile + (me.slice + 1) * L, tile + n), tile + n, s);
            }
            float in[L][V];  // dz without G
#pragma unroll
            for (int l = 0; l < L; ++l) {
                float vx[V];
                unpack(cx[l], vx);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if constexpr (SIG) {
                        in[l][i] = (h[i] - vx[i]) * (f[l][i] * rest[l][i]);
                        h[i] = fmaf(f[l][i], h[i], rest[l][i] * vx[i]);
                    } else {
                        in[l][i] = h[i];
                        h[i] = fmaf(f[l][i], h[i], vx[i]);
                    }
                }
            }
            auto go = [&](auto whole) {
#pragma unroll
                for (int l = L - 1; l >= 0; --l) {
                    float oz[V], ox[V], dy[V];
                    unpack(cg[l], dy);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float G = dy[i] + s[i];
                        oz[i] = G * in[l][i];
                        ox[i] = SIG ? G * rest[l][i] : G;
                        s[i] = f[l][i] * G;
                    }
                    if (whole() || l < mine) {
                        out_z.store(tile, me.slice, l, oz);
                        out_x.store(tile, me.slice, l, ox);
                    }
                }
            };
            if (n == kRecurrenceTile)
                go(std::true_type());
            else
                go(std::false_type());
            if (first) lds.carry[parity ^ 1][me.lane] = pack(s);
        }
    }
    if (!first) return;
    if constexpr (SUMS) {
        const int64_t edge = u.edge * a.channels + me.c;
        store_f32(a.sums + edge, me.valid, A);
        store_f32(a.sums + a.edges * a.channels + edge, me.valid, B);
    } else if (a.dstate && u.from == 0) {
        store_f32(a.dstate + row, me.valid, s);
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
    const int64_t count = (u.len + a.seqs.seg - 1) / a.seqs.seg, all = a.edges * a.channels;
    if (count < 2) return;
    // the edge behind (REVERSE: before) the k-th segment that the pass meets
    const int64_t edge0 = (u.t0 + a.seqs.seg - 1) / a.seqs.seg + (REVERSE ? count - 2 : 0);
    auto edge = [&](int64_t k) { return (edge0 + (REVERSE ? -k : k)) * a.channels + c; };
    const float* from = REVERSE ? a.dfinal : a.state;
    float h = from ? from[(int64_t)seq * a.channels + c] : 0.0f;
    const T* z = static_cast<const T*>(a.z.p) + u.t0 * a.z.stride + c;
    const RowView& other = REVERSE ? a.dh : a.x;
    const T* x = static_cast<const T*>(other.p) + u.t0 * other.stride + c;
    constexpr int AHEAD = 16;  // segments together: loaded ahead, and joined without a branch where none is unsafe
    float next_a[AHEAD], next_b[AHEAD];
    auto load = [&](int64_t k0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int64_t at = edge(min(k0 + i, count - 2));
            next_a[i] = a.sums[at];
            next_b[i] = a.sums[all + at];
        }
    };
    load(0);
    for (int64_t k0 = 0; k0 + 1 < count; k0 += AHEAD) {
        const int n = (int)min(count - 1 - k0, (int64_t)AHEAD);  // nothing starts behind the last one
        float A[AHEAD], B[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) A[i] = next_a[i], B[i] = next_b[i];
        if (k0 + AHEAD + 1 < count) load(k0 + AHEAD);
        const float from = h;
        bool walk = false;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (i < n) {
                const float next = fmaf(A[i], h, B[i]);
                walk = walk || unsafe(h, next) || (!SIG && fell(h, next, SEGMENT_FALL));
                h = next;
                a.starts[edge(k0 + i)] = h;
            }
        if (!walk) continue;
        h = from;
        for (int i = 0; i < n; ++i) {  // each from its sums if that is safe, else token by token
            const int64_t j = REVERSE ? count - 1 - k0 - i : k0 + i, at = edge(k0 + i);
            const float next = fmaf(a.sums[at], h, a.sums[all + at]);
            if (unsafe(h, next) || (!SIG && fell(h, next, SEGMENT_FALL))) {
                const int64_t lo = j * a.seqs.seg, hi = min(u.len, lo + a.seqs.seg);
                for (int64_t s = lo; s < hi; ++s) {
                    const int64_t t = REVERSE ? lo + hi - 1 - s : s;
                    float f, in;
                    const float v = St<T>::ld1(x + t * other.stride);
                    coefficients<T, SIG>(St<T>::ld1(z + t * a.z.stride), v, f, in);
                    h = REVERSE ? f * (v + h) : fmaf(f, h, in);
                }
            } else {
                h = next;
            }
            a.starts[at] = h;
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
            coefficients<T, SIG>(z[j], x[j], f, u);
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
// Forward and backward in bf16 at 512 channels, whole against in segments: one
// sequence of 600 tokens 14 / 21 against 16 / 20 us, of 800 19 / 28 against 17 / 20, of
// 4000 75 / 114 against 19 / 22, 8 of 2000 40 / 66 against 28 / 35; 32 of 2000 42 / 83
// against 69 / 97, 64 of 6000 281 / 412 against 473 / 667.
int64_t segment_of(const RecurrenceArgs& a) {
    constexpr int64_t CUS = 256;
    const int64_t blocks = (vecs_of(a.channels) + 31) / 32, share = a.seqs.tokens * blocks / CUS;
    if (a.seqs.longest <= std::max<int64_t>(768, 2 * share)) return 0;
    return std::max<int64_t>(256, (share / 4 + kRecurrenceTile - 1) / kRecurrenceTile * kRecurrenceTile);
}

int64_t edges_of(const RecurrenceArgs& a, int64_t seg) { return a.seqs.tokens / seg + 1; }

RecurrenceArgs plan(const RecurrenceArgs& in) {
    RecurrenceArgs a = in;
    a.seqs.seg = segment_of(a);
    a.seqs.slots = packed_slots(a.seqs, a.seqs.seg);
    if (a.seqs.seg) {
        a.edges = edges_of(a, a.seqs.seg);
        a.sums = static_cast<float*>(a.ws);
        a.starts = a.sums + 2 * a.edges * a.channels;
    }
    return a;
}

template <bool BACKWARD>
hipError_t launch(const RecurrenceArgs& in, hipStream_t s) {
    RecurrenceArgs a = plan(in);
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
    return seg ? (size_t)3 * edges_of(a, seg) * a.channels * 4 : 16;
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
