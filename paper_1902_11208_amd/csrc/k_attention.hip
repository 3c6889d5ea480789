// Linear attention with a decay for each head: the scan over packed sequences,
// the sum over shared heads, and the single-token step.
#include <algorithm>
#include <type_traits>

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

// ---------------------------------------------------------------------------
// The scan in chunks of C = 32 tokens, on matrix instructions. With the state S
// [dk][dv] before a chunk and g the decay, for tokens i, j of the chunk
//     o_i = g^(i+1) q_i S + sum_(j<=i) g^(i-j) (q_i . k_j) v_j
//     S'  = g^C S + sum_j g^(C-1-j) k_j v_j^T
// so a chunk costs products of 32-row tiles instead of 32 dependent steps.
//
// A wave keeps its columns of one head's state in MFMA accumulators for the whole
// sequence; the waves of a workgroup share the chunk's q, k and v rows in LDS
// (double buffers: one barrier a chunk, two where P is shared). All products are
// computed transposed, O^T = S^T Q^T + V^T P^T with P^T = K Q^T: a tile's
// accumulators hold, in lane 16 g + n, rows 4 g .. 4 g + 3 of column n, and a
// reduction may run in any order, so S and P^T are operands of the next product
// as they stand, with the reduction slots of lane group g taken as rows 4 g + r
// (and 16 + 4 g + r). The state never passes through LDS.
//
// bf16: q, k and v are operands as they are stored; P and S, fp32 sums, enter as
// two bf16 pieces each, the rounded number and what that leaves out (2^-17 of it
// is dropped), so an output carries the error of its own rounding only: 1.66e-3
// of the outputs. One piece each would leave 2.35e-3 and take 103 instead of
// 127 us for the wide batch's forward pass, 212 instead of 266 for its gradients.
// The state's sum takes g^(C-1-j) v_j in PIECES pieces (2, or 3 where the state is
// a result of the call: 2^-25 of a term is left out).
//
// What bounds it: memory at 64 columns where units are many (1024 units of 1024
// tokens, bf16, 0.54 GB: 115 us, 4.7 TB/s, where a copy reaches 5.5); at 128 bf16
// columns the waits between a chunk's products, which two workgroups a CU cannot
// fill (1024 units of 1024 tokens, 1.07 GB: 294 us, 3.7 TB/s; matrix instructions
// take 19% of the time, vector instructions 30%); the fp32 MFMA at 128 fp32 columns
// (694 us, 3.1 TB/s); the latency of a chunk where units are few (a unit alone: 1.0
// us a chunk at 64 bf16 columns, 2.1 at 128, 1.05 at 32 fp32). C = 32 and not 64: the
// products inside a chunk grow with C, the state's do not, and a chunk of 64 rows
// would leave one workgroup a CU at 128 columns.
// ---------------------------------------------------------------------------
constexpr int C = 32;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <typename T>
struct Mx;
template <>
struct Mx<float> {
    typedef floatx4 Frag;  // reduction over 16: slots 4 g + r
    static constexpr int KB = 16, PAD_Q = 4, PAD = 4;
    static __device__ __forceinline__ floatx4 mma(Frag a, Frag b, floatx4 c) {
#pragma unroll
        for (int r = 0; r < 4; ++r) c = mfma_f32(a[r], b[r], c);
        return c;
    }
    // row `row` of a staged tile, reduction along it; of a q tile, whose slots lie together
    static __device__ __forceinline__ Frag along(const float* tile, int pitch, int row, int k, int g) {
        return *reinterpret_cast<const floatx4*>(tile + row * pitch + k + 4 * g);
    }
    static __device__ __forceinline__ Frag along_q(const float* tile, int pitch, int row, int k, int g) {
        return along(tile, pitch, row, k, g);
    }
    static __device__ __forceinline__ void put_q(float* row, int col, u32x4 v) { *reinterpret_cast<u32x4*>(row + col) = v; }
    // column `col0 + n`, reduction down the rows
    static __device__ __forceinline__ Frag down(const float* tile, int pitch, int row0, int col0, int g, int n) {
        Frag f;
#pragma unroll
        for (int r = 0; r < 4; ++r) f[r] = tile[(row0 + 4 * g + r) * pitch + col0 + n];
        return f;
    }
    // fp32 numbers as operands of a product
    static constexpr int OPERANDS = 1;
    template <int N>
    static __device__ __forceinline__ void split(const floatx4* t, Frag (&f)[N]) {
        f[0] = t[0];
    }
};
template <>
struct Mx<bf16_t> {
    typedef bf16x8 Frag;  // reduction over 32: slots 4 g + r, then 16 + 4 g + r
    static constexpr int KB = 32, PAD_Q = 8, PAD = 16;
    typedef short s4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ floatx4 mma(Frag a, Frag b, floatx4 c) { return mfma_bf16(a, b, c); }
    static __device__ __forceinline__ Frag along(const bf16_t* tile, int pitch, int row, int k, int g) {
        const uint2 lo = *reinterpret_cast<const uint2*>(tile + row * pitch + k + 4 * g);
        const uint2 hi = *reinterpret_cast<const uint2*>(tile + row * pitch + k + 16 + 4 * g);
        return as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y));
    }
    // q rows are only read along, so a lane group's eight slots of 32 columns are staged side by side
    static __device__ __forceinline__ Frag along_q(const bf16_t* tile, int pitch, int row, int k, int g) {
        return as_bf16x8(*reinterpret_cast<const uint4*>(tile + row * pitch + k + 8 * g));
    }
    static __device__ __forceinline__ void put_q(bf16_t* row, int col, u32x4 v) {
        bf16_t* p = row + (col & ~31) + (col & 15) * 2 + ((col >> 4) & 1) * 4;
        *reinterpret_cast<u32x2*>(p) = u32x2{v[0], v[1]};
        *reinterpret_cast<u32x2*>(p + 8) = u32x2{v[2], v[3]};
    }
    // The LDS transpose read: in each sixteen lanes, lane 4 j + c points at four
    // consecutive values of row j, and lane n receives column n of the four rows.
    static __device__ __forceinline__ uint2 tr(const bf16_t* p) {
        const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(p));
        uint2 r;
        __builtin_memcpy(&r, &v, 8);
        return r;
    }
    static __device__ __forceinline__ Frag down(const bf16_t* tile, int pitch, int row0, int col0, int g, int n) {
        const bf16_t* p = tile + (row0 + 4 * g + (n >> 2)) * pitch + col0 + 4 * (n & 3);
        const uint2 lo = tr(p), hi = tr(p + 16 * pitch);
        return as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y));
    }
    static __device__ __forceinline__ Frag from(const floatx4* t) {
        return as_bf16x8(make_uint4(f2bf2(t[0][0], t[0][1]), f2bf2(t[0][2], t[0][3]), f2bf2(t[1][0], t[1][1]),
                                    f2bf2(t[1][2], t[1][3])));
    }
    // fp32 numbers as N bf16 operands: rounded, what that leaves out rounded, ...
    static constexpr int OPERANDS = 2;
    template <int N>
    static __device__ __forceinline__ void split(const floatx4* t, Frag (&f)[N]) {
        floatx4 x[2] = {t[0], t[1]};
#pragma unroll
        for (int c = 0; c < N; ++c) {
            f[c] = from(x);
            if (c + 1 < N)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[h][r] -= (float)f[c][4 * h + r];
        }
    }
};

// exp(-rate n) for n >= 0; 1 at n = 0 for every rate.
__device__ __forceinline__ float power(float l2, int n) { return n == 0 ? 1.0f : __builtin_amdgcn_exp2f(l2 * (float)n); }

// Sequences are cut into segments of `seg` tokens that are scanned side by
// side where there are too few sequences to fill the chip. Segment j of
// sequence i has slot i + offsets[i] / seg + j; slots in between stay empty.
__device__ __forceinline__ int find_sequence(const int64_t* offsets, int n, int64_t tokens, int64_t seg, int64_t slot) {
    int lo = 0, hi = n;  // the last sequence whose first slot is at most `slot`
    const int lane = threadIdx.x & 63;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, i = lo + lane * step;
        const bool in = i < hi && i + min(max(offsets[i], (int64_t)0), tokens) / seg <= slot;
        const int below = __popcll(__ballot(in));
        if (below == 0) break;
        lo += (below - 1) * step;
        hi = min(hi, lo + step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

struct Unit {
    int role, head, seq;
    int64_t slot, j;  // slot and segment; without segments slot = seq, j = 0
};

// Units in launch order: workgroup b runs on XCD b % 8, which takes the roles
// and `together` heads of one slot one after the other: they read the same
// tokens, and the heads of a token share cache lines where they are narrow (1024
// units of 32 bf16 columns, 32 chunks each: 78 us by (slot, key head), 49 by slot).
// False: no unit.
__device__ __forceinline__ bool unit_of(const ScanArgs& a, Unit& u) {
    const int group = a.together, kv = a.heads / group, inner = a.n_roles * group;
    const int64_t b = block_index(), i = b >> 3, rest = i / inner * 8 + (b & 7);
    const int in = (int)(i % inner);
    u.slot = rest / kv;
    if (u.slot >= a.slots) return false;
    u.role = in % a.n_roles;
    u.head = (int)(rest % kv) * group + in / a.n_roles;
    u.j = 0;
    u.seq = (int)u.slot;
    if (!a.seg && a.order) {  // longest first: the wide batch's gradients 269 us, 295 as numbered
        u.seq = __builtin_amdgcn_readfirstlane(a.order[u.slot]);
        if (u.seq < 0 || u.seq >= a.n) return false;
    }
    if (a.seg) {
        u.seq = find_sequence(a.offsets, a.n, a.tokens, a.seg, u.slot);
        u.j = u.slot - u.seq - min(max(a.offsets[u.seq], (int64_t)0), a.tokens) / a.seg;
    }
    return u.j >= 0;  // negative only where the offsets do not ascend
}

// 32 rows of a tensor as a buffer: row r of a chunk lies r `stride` bytes from
// its row 0, backwards in a scan from the end. Offsets count from the row at
// the lowest address; OUT is outside the buffer: such loads give 0 and such
// stores write nothing, without a branch.
constexpr int OUT = 0x7fffffff;
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer(const char* row_0, int64_t stride) {
    const char* p = stride < 0 ? row_0 + (C - 1) * stride : row_0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p), 0, 0x7ffffff0, 0x00027000);
}
__device__ __forceinline__ int row_offset(int row, int stride) { return stride < 0 ? (row - (C - 1)) * stride : row * stride; }

// A thread's share of a chunk's q, k or v rows, on its way from memory to LDS:
// rows first, first + STEP, ... of it, 16 bytes each. Rows before row0 and
// columns from dim on are zero. WIDE: rows are whole aligned 16-byte vectors
// and a chunk spans less than 2^31 bytes.
template <typename T, int D, int THREADS, bool WIDE>
struct Stage {
    static constexpr int EPV = 16 / sizeof(T), VPR = D / EPV, N = C * VPR / THREADS, STEP = THREADS / VPR;
    static_assert(N * THREADS == C * VPR, "every thread has the same number of vectors");
    u32x4 v[N];
    int offset;  // of the first vector
    __device__ __forceinline__ void init(int64_t stride, int dim) {
        const int first = threadIdx.x / VPR, col = threadIdx.x % VPR * EPV;
        offset = col < dim ? row_offset(first, (int)stride) + col * (int)sizeof(T) : OUT;
    }
    __device__ __forceinline__ void load(const char* base, int64_t stride, int dim, int row0) {
        const int first = threadIdx.x / VPR, col = threadIdx.x % VPR * EPV;
        if constexpr (WIDE) {
            const Buffer b = buffer(base, stride);
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = __builtin_amdgcn_raw_buffer_load_b128(
                    b, first + i * STEP >= row0 && offset != OUT ? offset + i * STEP * (int)stride : OUT, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = u32x4{0, 0, 0, 0};
                if (first + i * STEP >= row0) {
                    const T* p = reinterpret_cast<const T*>(base + (first + i * STEP) * stride) + col;
                    T e[EPV];
#pragma unroll
                    for (int j = 0; j < EPV; ++j) e[j] = col + j < dim ? p[j] : T(0);
                    __builtin_memcpy(&v[i], e, 16);
                }
            }
        }
    }
    template <bool IS_Q>
    __device__ __forceinline__ void store(T* tile, int pitch) const {
        T* p = tile + threadIdx.x / VPR * pitch;
        const int col = threadIdx.x % VPR * EPV;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (IS_Q)
                Mx<T>::put_q(p + i * STEP * pitch, col, v[i]);
            else
                *reinterpret_cast<u32x4*>(p + i * STEP * pitch + col) = v[i];
        }
    }
};

__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                     (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// Has a value computed here, not again or later on.
template <typename V>
__device__ __forceinline__ void keep(V& x) {
    asm volatile("" : "+v"(x));
}

// exp(x) to about 2^-48 as a sum of two positive numbers, so that an infinite
// state times it stays infinite.
struct Decay {
    float hi, lo;
};
__device__ __forceinline__ Decay decay_of(double x) {
    constexpr float least = 0x1p-149f;
    const double e = exp(x);
    float hi = (float)e;
    if ((double)hi > e) hi = __uint_as_float(__float_as_uint(hi) - 1);
    if (hi < least) hi = least;
    const float lo = (float)(e - (double)hi);
    return Decay{hi, lo < least ? least : lo};
}

__device__ __forceinline__ bool not_finite(float x) { return !(x - x == 0.0f); }

// Outputs and states of a wave that came out infinite or NaN, taken again one
// token at a time. In a chunk's products a value that is not finite reaches
// other tokens and rows as 0 v = NaN, and a bf16 operand's pieces as v - v; a
// state beyond 2^120 overflows in registers that hold up to 2^8 times of it.
// What came out finite stays as it is.
template <typename T, int KT, int NT, bool LOCAL, typename Init>
__device__ __forceinline__ void scan_plain(const ScanArgs& a, const ScanRole& R, int head, int64_t t0, int64_t len, int64_t from,
                                        int64_t to, int slab, float* to_state, bool transposed, Init init) {
    const int l = threadIdx.x & 63, g = l >> 4, n = l & 15, dk = R.q.dim, dv = R.v.dim;
    const Decay once = decay_of(-(double)a.rates[head]), none = decay_of(0.0);
    floatx4 S[KT][NT];
    init(S, 0);  // in reverse, also that of a later segment has decayed up to its first token
    for (int64_t pos = from; pos < to; ++pos) {
        const int64_t t = R.reverse ? t0 + len - 1 - pos : t0 + pos;
        const T *q = at<T>(R.q, t, head), *k = at<T>(R.k, t, head), *v = at<T>(R.v, t, head);
        const Decay f = R.reverse && pos == from ? none : once;
        float o[NT], x[NT];
#pragma unroll
        for (int m = 0; m < NT; ++m) {
            const int c = slab + 16 * m + n;
            o[m] = 0.0f;
            x[m] = c < dv ? St<T>::ld1(v + c) * R.in_scale : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + 4 * g + r;
                const float kr = row < dk ? St<T>::ld1(k + row) : 0.0f, qr = !LOCAL && row < dk ? St<T>::ld1(q + row) : 0.0f;
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    S[i][m][r] = row < dk ? fmaf(S[i][m][r], f.hi, fmaf(S[i][m][r], f.lo, kr * x[m])) : 0.0f;
                    o[m] = fmaf(qr, S[i][m][r], o[m]);
                }
            }
#pragma unroll
        for (int m = 0; m < NT && !LOCAL; ++m) {
            o[m] += __shfl_xor(o[m], 16);
            o[m] += __shfl_xor(o[m], 32);
            const int c = slab + 16 * m + n;
            if (g == 0 && c < dv) {
                const int64_t at_o = (t * a.heads + head) * dv + c;
                if (R.out_f32) {
                    float* d = static_cast<float*>(R.out) + at_o;
                    if (not_finite(*d)) *d = o[m] * R.out_scale;
                } else {
                    T* d = static_cast<T*>(R.out) + at_o;
                    if (not_finite(St<T>::ld1(d))) St<T>::st1(d, o[m] * R.out_scale);
                }
            }
        }
    }
    if (!to_state) return;
    const Decay f = R.reverse && to > from ? once : none;
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * i + 4 * g + r, c = slab + 16 * m + n;
                if (row < dk && c < dv) {
                    float* d = to_state + (transposed ? c * dk + row : row * dv + c);
                    if (not_finite(*d)) *d = fmaf(S[i][m][r], f.hi, S[i][m][r] * f.lo);
                }
            }
}

// A workgroup's waves share a unit's chunk. A wave has NT column tiles of the
// state and TI of the chunk's two token tiles. With TI 2 each wave's columns are
// its own, and from four waves on P^T comes from three of them through LDS. With
// TI 1 two waves share columns: of 32 by 32 states (SPLIT) each keeps 16 of the
// rows, multiplies both token tiles by them and passes on the tile that is the
// other's; of 16 by 16 ones both keep the state, and each computes its part of P.
//
// WIDE: rows of q, k, v are whole 16-byte vectors. LOCAL: only the state that
// a segment adds to zero; of a sequence's last segment where the final state is
// asked for.
//
// The scan's length need not be a multiple of C: its first chunk starts before
// the first token, with rows of zeros, so that distances to a chunk's end are
// the same in every chunk.
template <int D, int NT, int TI>
constexpr int scan_threads() { return 64 * (D / 16 / NT) * (2 / TI); }

template <typename T, int D, int NT, int TI, bool WIDE, int PIECES, bool LOCAL>
__global__ __launch_bounds__((scan_threads<D, NT, TI>()), 2) void k_scan(ScanArgs a) {
    typedef Mx<T> M;
    typedef typename M::Frag Frag;
    constexpr int THREADS = scan_threads<D, NT, TI>(), TPF = M::KB / 16, COLS = D / 16 / NT;
    constexpr bool SPLIT = TI == 1 && D == 32;
    constexpr int KT = SPLIT ? 1 : D / 16, OT = SPLIT ? 2 : TI;  // state tiles of a column tile, token tiles they meet
    static_assert(!SPLIT || (TPF == 1 && NT == 1), "a split state is built for fp32");
    constexpr int PQ = D + M::PAD_Q, PK = D + M::PAD;
    constexpr int NP = sizeof(T) == 4 ? 1 : PIECES, NO = M::OPERANDS;
    constexpr bool SHARE = SPLIT || (TI == 2 && !LOCAL && THREADS >= 192);
    constexpr int AT_K = LOCAL ? 0 : C * PQ, AT_V = AT_K + C * PK, BUF = AT_V + C * PK;
    constexpr int BUFS = 2 * BUF * sizeof(T) <= 60 * 1024 ? 2 : 1;
    __shared__ __align__(16) T lds[BUFS * BUF];
    // bf16 outputs pass through LDS, to leave as whole rows a chunk later: a wave's
    // own stores are 32 bytes of a row (wide batch forward 128 us, 171 with those)
    constexpr bool ROWS_OUT = sizeof(T) == 2 && WIDE && !LOCAL;
    constexpr int PO = D + 8, OUT_PIECES = C * D / 8, OBUFS = SHARE ? 1 : 2;
    __shared__ __align__(16) T out_rows[ROWS_OUT ? OBUFS * C * PO : 8];
    typedef T Tile[64][4];  // P^T tile, four values of a lane together
    __shared__ __align__(16) Tile shared_p[NO][SHARE ? 3 : 1];
    __shared__ __align__(16) float passed[SPLIT ? 4 : 1][64][4];
    Unit u;
    if (!unit_of(a, u)) return;
    const ScanRole& R = a.role[u.role];
    int64_t t0, len;
    sequence(a.offsets, u.seq, a.tokens, a.longest, t0, len);
    t0 = uniform(t0);
    len = uniform(len);
    const int64_t from = u.j * a.seg, to = a.seg ? min(len, from + a.seg) : len;
    if (u.j > 0 && from >= len) return;
    if (LOCAL && to >= len && !R.final_state) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l = threadIdx.x & 63, g = l >> 4, n = l & 15, slab = wave % COLS * NT * 16, i0 = TI == 2 ? 0 : wave / COLS;
    const int dk = R.q.dim, dv = R.v.dim, head = u.head, e = R.reverse;
    const float l2 = -1.4426950408889634f * a.rates[head];  // log2 g

    // Decays inside a chunk; a token j beyond i meets it with 0. SHARE: of the tile
    // that this wave computes, (j, i) = (0, 0), (0, 1) or (1, 1); else of those of
    // its token tiles.
    float same[4], lower[4], w[2][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = n, j = 4 * g + r;
        const float ps = R.in_scale * R.out_scale;
        same[r] = j <= i ? ps * power(l2, i - j) : 0.0f;
        lower[r] = ps * power(l2, 16 + i - j);
        if (SHARE && wave == 1) same[r] = lower[r];
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h][r] = R.in_scale * power(l2, C - 1 - (16 * h + j) + e);
        keep(same[r]);
        keep(lower[r]);
        keep(w[0][r]);
        keep(w[1][r]);
    }
    // The state in registers is S / g^age: what it has decayed by since it was
    // last scaled is left out until that reaches 2^-8 (a multiplication a chunk
    // and element less; beyond, exponents would cost precision). late: weight of
    // the registers' state at the chunk's tokens.
    const int skip = (int)(-(to - from) & (C - 1));  // rows of zeros in the first chunk
    const int oldest = __builtin_amdgcn_readfirstlane((int)fminf(8.0f / fabsf(l2), 1e9f));
    int age = 0;
    float full[OT], late[OT];
#pragma unroll
    for (int h = 0; h < OT; ++h) {
        const int i = 16 * ((SPLIT ? 0 : i0) + h) + n;
        full[h] = R.out_scale * power(l2, i + 1 - e);
        late[h] = R.out_scale * power(l2, max(i - skip, 0) + 1 - e);
        keep(full[h]);
    }

    auto init = [&](auto& S, int tile0) {
        const float* from_state = nullptr;
        const int64_t size = (int64_t)dk * dv;
        bool transposed = false;
        if (LOCAL) {
        } else if (u.j > 0) {  // the slot before holds the state that this segment starts from
            from_state = a.states + (((int64_t)u.role * a.heads + head) * a.slots + u.slot - 1) * size;
        } else if (R.state) {
            from_state = R.state + ((int64_t)u.seq * a.heads + head) * size;
            transposed = R.state_t;
        }
#pragma unroll
        for (int t = 0; t < (int)std::extent<std::remove_reference_t<decltype(S)>>(); ++t)
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * (tile0 + t) + 4 * g + r, c = slab + 16 * m + n;
                    S[t][m][r] = from_state && i < dk && c < dv ? from_state[transposed ? c * dk + i : i * dv + c] : 0.0f;
                }
    };
    const int tile0 = SPLIT ? i0 : 0;
    floatx4 S[KT][NT];  // S[t][m][r] = state[16 (tile0 + t) + 4 g + r][slab + 16 m + n]
    init(S, tile0);

    // bytes between rows and from a chunk to the next; the chunk's row 0 is scan position pos
    const int dir = R.reverse ? -1 : 1;
    const int64_t first = (R.reverse ? t0 + len - 1 : t0) + dir * (from - skip);
    const int64_t qs = dir * R.q.token_stride * (int64_t)sizeof(T), ks = dir * R.k.token_stride * (int64_t)sizeof(T),
                  vs = dir * R.v.token_stride * (int64_t)sizeof(T);
    const char* qp = reinterpret_cast<const char*>(at<T>(R.q, 0, head)) + first * dir * qs;
    const char* kp = reinterpret_cast<const char*>(at<T>(R.k, 0, head)) + first * dir * ks;
    const char* vp = reinterpret_cast<const char*>(at<T>(R.v, 0, head)) + first * dir * vs;
    const bool f32 = sizeof(T) == 4 || R.out_f32;
    const int osize = f32 ? 4 : (int)sizeof(T), os = dir * a.heads * dv * osize;  // bytes between output rows
    char* out = static_cast<char*>(R.out) + (first * a.heads + head) * dv * osize;
    Stage<T, D, THREADS, WIDE> sq, sk, sv;
    if (!LOCAL) sq.init(qs, dk);
    sk.init(ks, dk);
    sv.init(vs, dv);
    auto fetch = [&](int skip) {
        if (!LOCAL) sq.load(qp, qs, dk, skip);
        sk.load(kp, ks, dk, skip);
        sv.load(vp, vs, dv, skip);
        qp += C * qs;
        kp += C * ks;
        vp += C * vs;
    };
    auto put = [&](T* buf) {
        if (!LOCAL) sq.template store<true>(buf, PQ);
        sk.template store<false>(buf + AT_K, PK);
        sv.template store<false>(buf + AT_V, PK);
    };
    // rows of the chunk at `row`, from row0 on, as staged in out_rows
    auto flush = [&](const T* staged, char* row, int row0) {
        const Buffer to_out = buffer(row, os);
#pragma unroll
        for (int x = threadIdx.x; x < (OUT_PIECES + THREADS - 1) / THREADS * THREADS; x += THREADS) {
            const int i = x / (D / 8), c = x % (D / 8) * 8;
            const bool in = x < OUT_PIECES && i >= row0 && c < dv;
            const u32x4 v = *reinterpret_cast<const u32x4*>(staged + (x < OUT_PIECES ? i * PO + c : 0));
            __builtin_amdgcn_raw_buffer_store_b128(v, to_out, in ? row_offset(i, os) + c * 2 : OUT, 0, 2);
        }
    };
    const int chunks = (int)((to - from + C - 1) / C);
    const floatx4 zero = {0, 0, 0, 0};
    floatx4 bad = zero;  // NaN once an output was not finite
    int row0 = skip, flush0 = skip;
    if (chunks > 0) {
        fetch(skip);
        put(lds);
    }
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const T* Q = lds + (BUFS == 2 ? (chunk & 1) * BUF : 0);
        const T *K = Q + AT_K, *V = Q + AT_V;
        lds_barrier();  // this chunk's rows are there; with two buffers no wave reads the other one any more
        if (chunk + 1 < chunks) fetch(0);
        floatx4 o[NT][OT];
        Frag vf[NT][2 / TPF];
        if (!LOCAL) {
            floatx4 p[3] = {zero, zero, zero};  // (j tile, i tile) (0, 0), (0, 1), (1, 1)
            if (SHARE && wave < 3) {
                const int j0 = wave == 2 ? 16 : 0, q0 = wave == 0 ? 0 : 16;
#pragma unroll
                for (int k = 0; k < D / M::KB; ++k)
                    p[0] = M::mma(M::along(K, PK, j0 + n, k * M::KB, g), M::along_q(Q, PQ, q0 + n, k * M::KB, g), p[0]);
                // a select: what lies beyond i may be infinite
                if (wave == 1) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[0][r] *= same[r];
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[0][r] = 4 * g + r <= n ? p[0][r] * same[r] : 0.0f;
                }
                const floatx4 t[2] = {p[0], zero};
                Frag f[NO];
                M::split(t, f);
#pragma unroll
                for (int c = 0; c < NO; ++c) __builtin_memcpy(shared_p[c][wave][l], &f[c], sizeof(shared_p[c][wave][l]));
            }
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int h = 0; h < OT; ++h) o[m][h] = zero;
#pragma unroll
            for (int k = 0; k < KT / TPF; ++k) {
                Frag q[OT];
#pragma unroll
                for (int h = 0; h < OT; ++h)
                    q[h] = M::along_q(Q, PQ, 16 * ((SPLIT ? 0 : i0) + h) + n, k * M::KB + 16 * tile0, g);
                if (!SHARE) {
                    const Frag k0 = M::along(K, PK, n, k * M::KB, g);
                    if (TI == 2) {
                        p[0] = M::mma(k0, q[0], p[0]);
                        p[1] = M::mma(k0, q[TI - 1], p[1]);
                        p[2] = M::mma(M::along(K, PK, 16 + n, k * M::KB, g), q[TI - 1], p[2]);
                    } else if (i0 == 0) {
                        p[0] = M::mma(k0, q[0], p[0]);
                    } else {
                        p[1] = M::mma(k0, q[0], p[1]);
                        p[2] = M::mma(M::along(K, PK, 16 + n, k * M::KB, g), q[0], p[2]);
                    }
                }
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    floatx4 t[TPF];
#pragma unroll
                    for (int x = 0; x < TPF; ++x) t[x] = S[k * TPF + x][m];
                    Frag s[NO];
                    M::split(t, s);
#pragma unroll
                    for (int c = 0; c < NO; ++c)
#pragma unroll
                        for (int h = 0; h < OT; ++h) o[m][h] = M::mma(s[c], q[h], o[m][h]);
                }
            }
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int h = 0; h < 2 / TPF; ++h) vf[m][h] = M::down(V, PK, h * M::KB, slab + 16 * m, g, n);
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int h = 0; h < OT; ++h) {
                    o[m][h] *= late[h];
                    keep(o[m][h]);  // beyond the branch below it was read before the matrix instruction had written it
                }
            if (SPLIT) St<float>::st4(passed[wave][l], i0 == 0 ? o[0][OT - 1] : o[0][0]);
            if (ROWS_OUT && !f32 && chunk > 0) {  // the outputs of the chunk before
                flush(out_rows + (OBUFS == 2 ? ((chunk - 1) & 1) * C * PO : 0), out, flush0);
                out += (int64_t)C * os;
                flush0 = 0;
            }
            Frag f0[2 / TPF][NO], f1[2 / TPF][NO];  // P^T for the token tiles 0 and 1
            if (SHARE) {
                lds_barrier();
                if constexpr (sizeof(T) == 2) {
#pragma unroll
                    for (int c = 0; c < NO; ++c) {
                        const uint2 x = *reinterpret_cast<const uint2*>(shared_p[c][0][l]),
                                    y = *reinterpret_cast<const uint2*>(shared_p[c][1][l]),
                                    z = *reinterpret_cast<const uint2*>(shared_p[c][2][l]);
                        f0[0][c] = as_bf16x8(make_uint4(x.x, x.y, 0, 0));
                        f1[0][c] = as_bf16x8(make_uint4(y.x, y.y, z.x, z.y));
                    }
                } else {
                    f0[0][0] = St<T>::ld4(shared_p[0][0][l]);
                    f1[0][0] = St<T>::ld4(shared_p[0][1][l]);
                    f1[1][0] = St<T>::ld4(shared_p[0][2][l]);
                    if (SPLIT) o[0][0] = (i0 == 0 ? o[0][0] : o[0][OT - 1]) + St<float>::ld4(passed[wave ^ COLS][l]);
                }
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    p[0][r] = 4 * g + r <= n ? p[0][r] * same[r] : 0.0f;
                    p[2][r] = 4 * g + r <= n ? p[2][r] * same[r] : 0.0f;
                    p[1][r] *= lower[r];
                }
                const floatx4 b0[2] = {p[0], zero}, b1[2] = {p[1], p[2]};
#pragma unroll
                for (int h = 0; h < 2 / TPF; ++h) {
                    M::split(b0 + h, f0[h]);
                    M::split(b1 + h, f1[h]);
                }
            }
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int c = 0; c < NO; ++c) {
                    if (TI == 2 || i0 == 0) o[m][0] = M::mma(vf[m][0], f0[0][c], o[m][0]);
                    if (TI == 2 || i0 == 1) {
#pragma unroll
                        for (int h = 0; h < 2 / TPF; ++h) o[m][TI - 1] = M::mma(vf[m][h], f1[h][c], o[m][TI - 1]);
                    }
                }
        } else {
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int h = 0; h < 2 / TPF; ++h) vf[m][h] = M::down(V, PK, h * M::KB, slab + 16 * m, g, n);
        }
        // S = g^C S + K^T (w V)
        float fresh = 1.0f;
        age += C - row0;
        if (age > oldest) {
            const float f = power(l2, age);
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int m = 0; m < NT; ++m) S[t][m] *= f;
            age = 0;
        } else {
            fresh = __builtin_amdgcn_exp2f(-l2 * (float)age);
        }
#pragma unroll
        for (int h = 0; h < OT; ++h) late[h] = full[h] * power(l2, age);
        Frag wv[NT][2 / TPF][NP];
#pragma unroll
        for (int m = 0; m < NT; ++m) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) wv[m][h][0][r] = vf[m][h][r] * (w[h][r] * fresh);
            } else {
                floatx4 x[2];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[h][r] = (float)vf[m][0][4 * h + r] * (w[h][r] * fresh);
                M::split(x, wv[m][0]);
            }
        }
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int h = 0; h < 2 / TPF; ++h) {
                const Frag kt = M::down(K, PK, h * M::KB, 16 * (tile0 + t), g, n);
#pragma unroll
                for (int c = NP - 1; c >= 0; --c)
#pragma unroll
                    for (int m = 0; m < NT; ++m) S[t][m] = M::mma(kt, wv[m][h][c], S[t][m]);
            }
        // the next chunk's rows before the outputs: a wait for them would wait for those too
        if (BUFS == 1) lds_barrier();
        if (chunk + 1 < chunks) put(lds + (BUFS == 2 ? ((chunk + 1) & 1) * BUF : 0));
        if (!LOCAL) {
            const Buffer to_out = buffer(out, os);
#pragma unroll
            for (int h = 0; h < TI; ++h) {
                const int i = 16 * (i0 + h) + n;
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    const int c = slab + 16 * m + 4 * g;
                    if (ROWS_OUT && !f32) {
                        St<T>::st4(out_rows + (OBUFS == 2 ? (chunk & 1) * C * PO : 0) + i * PO + c, o[m][h]);
                    } else if (WIDE) {
                        u32x4 x;
                        __builtin_memcpy(&x, &o[m][h], 16);
                        __builtin_amdgcn_raw_buffer_store_b128(x, to_out, i >= row0 && c < dv ? row_offset(i, os) + c * 4 : OUT, 0, 2);
                    } else if (i >= row0) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (c + r < dv) {
                                if (f32)
                                    reinterpret_cast<float*>(out + i * os)[c + r] = o[m][h][r];
                                else
                                    St<T>::st1(reinterpret_cast<T*>(out + i * os) + c + r, o[m][h][r]);
                            }
                    }
                }
            }
            // An output that is not finite leaves 0 o = NaN.
            if constexpr (sizeof(T) == 2) {
                const Frag none = {};
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    const floatx4 out2[2] = {o[m][0], o[m][OT - 1]};
                    bad = M::mma(M::from(out2), none, bad);
                }
            } else {
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int h = 0; h < TI; ++h)
#pragma unroll
                        for (int r = 0; r < 4; ++r) bad[r] = fmaf(o[m][h][r], 0.0f, bad[r]);
            }
            if (!ROWS_OUT || f32) out += (int64_t)C * os;
        }
        row0 = 0;
    }
    if (ROWS_OUT && !f32 && chunks > 0) {
        lds_barrier();
        flush(out_rows + (OBUFS == 2 ? ((chunks - 1) & 1) * C * PO : 0), out, flush0);
    }
    {
        const float f = power(l2, age);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int m = 0; m < NT; ++m) S[t][m] *= f;
    }

    const int64_t size = (int64_t)dk * dv;
    float* to_state = nullptr;
    bool transposed = false;
    if (LOCAL) {
        to_state = a.states + (((int64_t)u.role * a.heads + head) * a.slots + u.slot) * size;
    } else if (R.final_state && !a.seg) {  // with segments it comes from k_join_segments
        to_state = R.final_state + ((int64_t)u.seq * a.heads + head) * size;
        transposed = R.state_t;
    }
    if (to_state && (SPLIT || i0 == 0)) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int m = 0; m < NT; ++m)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * (tile0 + t) + 4 * g + r, c = slab + 16 * m + n;
                    if (i < dk && c < dv) to_state[transposed ? c * dk + i : i * dv + c] = S[t][m][r];
                }
    }
    // A state that was not finite once is so at the end.
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int r = 0; r < 4; ++r) bad[r] = fmaf(S[t][m][r], 0.0f, bad[r]);
    if (__syncthreads_or(not_finite(bad[0] + bad[1] + bad[2] + bad[3]))) {
        __threadfence();  // outputs and states as written, also by the waves that share this one's columns
        __syncthreads();
        if (i0 == 0) scan_plain<T, D / 16, NT, LOCAL>(a, R, head, t0, len, from, to, slab, to_state, transposed, init);
    }
}

// The states that segments start from: for every sequence, head and element of
// the state, over its segments in order. Slot j holds what segment j adds to
// zero and receives the state that segment j + 1 starts from; the last one's
// goes to the final states.
__global__ __launch_bounds__(256) void k_join_segments(ScanArgs a) {
    const int role = blockIdx.z % a.n_roles;
    const ScanRole& R = a.role[role];
    const int64_t unit = block_index();
    if (unit >= (int64_t)a.n * a.heads) return;
    const int seq = (int)(unit / a.heads), head = (int)(unit % a.heads), size = R.q.dim * R.v.dim;
    const int x = blockIdx.z / a.n_roles * 256 + threadIdx.x;
    int64_t t0, len;
    sequence(a.offsets, seq, a.tokens, a.longest, t0, len);
    t0 = uniform(t0);
    len = uniform(len);
    if (x >= size || (len <= a.seg && !R.final_state)) return;
    const double rate = a.rates[head];
    const Decay gs = decay_of(-rate * (double)a.seg);
    const int64_t outside = ((int64_t)seq * a.heads + head) * size + (R.state_t ? x % R.v.dim * R.q.dim + x / R.v.dim : x);
    float s = R.state ? R.state[outside] : 0.0f;
    const int64_t slot0 = seq + t0 / a.seg;
    float* p = a.states + (((int64_t)role * a.heads + head) * a.slots + slot0) * size + x;
    const int64_t step = size;
    const int joins = len > 0 ? (int)((len - 1) / a.seg) : 0;
    // Latency bounds it: N loads are in flight while the N before are joined, and
    // the last ones read a slot again rather than branch (128 segments of 8 heads of
    // 64 x 64, 34 MB: 10.4 us, 13.0 with rounds of 32 one after the other).
    constexpr int N = 16;
    float v[N], next[N];
    auto load = [&](float(&to)[N], int j) {
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = p[min(j + i, joins - 1) * step];
    };
    if (joins > 0) load(v, 0);
    int j = 0;
    for (; j + N < joins; j += N) {
        load(next, j + N);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            s = fmaf(s, gs.hi, fmaf(s, gs.lo, v[i]));
            p[(j + i) * step] = s;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = next[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (j + i < joins) {
            s = fmaf(s, gs.hi, fmaf(s, gs.lo, v[i]));
            p[(j + i) * step] = s;
        }
    if (R.final_state) {
        const float last = a.states[(((int64_t)role * a.heads + head) * a.slots + slot0 + joins) * size + x];
        const double g = fmax(exp(-rate * (double)(len - joins * a.seg)), 0x1p-1074);  // not 0: s may be infinite
        R.final_state[outside] = len > 0 ? (float)(g * (double)s + (double)last) : s;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_sum_heads(int64_t n, int group, int dim, const float* src, T* dst) {
    const int64_t i = block_index() * 256 + threadIdx.x;  // (token, kv head, element)
    if (i >= n) return;
    const int64_t th = i / dim;
    const float* p = src + th * group * dim + (i - th * dim);
    float s = 0.0f;
    for (int c = 0; c < group; ++c) s += p[(int64_t)c * dim];
    St<T>::st1(dst + i, s);
}

// ---------------------------------------------------------------------------
// One token: the state is read and written once and nothing else counts, so a
// workgroup per (row, head) issues all its loads of the state at once. CG
// threads share a row of it, V columns each; the workgroup's other threads take
// other rows, and their sums for o meet by shuffles and in LDS. 509 rows of 16 heads
// of 128 x 128: 204 us for 1.07 GB, 5.3 TB/s; few rows: the launch (3.2 us). 4 heads of
// 32 x 32 fp32, 16384 rows: 4.6 TB/s. Narrower states leave most of the 256 threads
// without one (16 x 16 and 65536 rows: 427 us, 1.4 TB/s, 1.6 ns a workgroup), and
// states whose rows are not 16-byte vectors move by 4 bytes a lane (61 x 61, 4096
// rows: 143 us, 3.5 TB/s).
// ---------------------------------------------------------------------------
template <int V>
struct Cols {
    float x[V];
};

template <typename T, int V, int CG>
__global__ __launch_bounds__(256) void k_step(StepArgs a) {
    constexpr int RG = 256 / CG, N = (128 + RG - 1) / RG;  // rows at once, rows of a thread
    __shared__ float q[128], k[128], part[4][CG * V];
    const int64_t row = block_index();
    if (row >= a.n) return;
    const int head = blockIdx.z, dk = a.q.dim, dv = a.v.dim;
    const int c = threadIdx.x % CG * V, r0 = threadIdx.x / CG;
    const int64_t slot = a.slot ? a.slot[row] : row;
    T* out = static_cast<T*>(a.out) + (row * a.heads + head) * dv;
    if (slot < 0 || slot >= a.slots) {
        if ((int)threadIdx.x < dv) St<T>::st1(out + threadIdx.x, 0.0f);
        return;
    }
    float* S = a.state + (slot * a.heads + head) * dk * dv + c;
    Cols<V> s[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (r0 + i * RG < dk && c < dv) {
            if constexpr (V == 4) {
                const floatx4 t = __builtin_nontemporal_load(reinterpret_cast<const floatx4*>(S + (r0 + i * RG) * dv));
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i].x[j] = t[j];
            } else {
                s[i].x[0] = S[(r0 + i * RG) * dv];
            }
        }
    if ((int)threadIdx.x < dk)
        q[threadIdx.x] = St<T>::ld1(at<T>(a.q, row, head) + threadIdx.x);
    else if (threadIdx.x >= 128 && (int)threadIdx.x - 128 < dk)
        k[threadIdx.x - 128] = St<T>::ld1(at<T>(a.k, row, head) + threadIdx.x - 128);
    float v[V], o[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        v[j] = c < dv ? St<T>::ld1(at<T>(a.v, row, head) + c + j) : 0.0f;
        o[j] = 0.0f;
    }
    const float g = expf(-a.rates[head]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (r0 + i * RG < dk && c < dv) {
            const float ki = k[r0 + i * RG], qi = q[r0 + i * RG];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[i].x[j] = fmaf(ki, v[j], s[i].x[j] * g);
                o[j] = fmaf(qi, s[i].x[j], o[j]);
            }
            if constexpr (V == 4)
                __builtin_nontemporal_store(floatx4{s[i].x[0], s[i].x[1], s[i].x[2], s[i].x[3]},
                                            reinterpret_cast<floatx4*>(S + (r0 + i * RG) * dv));
            else
                S[(r0 + i * RG) * dv] = s[i].x[0];
        }
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int d = CG; d < 64; d *= 2) o[j] += __shfl_xor(o[j], d);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // a wave's columns: all CG threads' where they fit in it, else its half of them
    if constexpr (CG <= 64) {
        if (lane < CG)
#pragma unroll
            for (int j = 0; j < V; ++j) part[wave][lane * V + j] = o[j];
        __syncthreads();
        if ((int)threadIdx.x < dv) {
            const int x = threadIdx.x;
            St<T>::st1(out + x, (part[0][x] + part[1][x] + part[2][x] + part[3][x]) * a.scale);
        }
    } else {
        part[wave >> 1][threadIdx.x % CG] = o[0];
        __syncthreads();
        if ((int)threadIdx.x < dv) St<T>::st1(out + threadIdx.x, (part[0][threadIdx.x] + part[1][threadIdx.x]) * a.scale);
    }
}

}  // namespace

// Tokens of a segment, 0: sequences are scanned whole. Segments cost a second
// pass over k and v, the states between them and two more launches, so the
// longest sequence has to leave most of the chip idle for long: `idle` is how
// many times the chip could run all workgroups while it runs. Equal sequences,
// us whole and in segments, forward (gradients):
//     tokens  heads          idle       whole          segments
//      512    4 x 32 fp32    256 (85)   21.4 (21.5)    17.9 (18.0)
//                            32 (10.7)  21.6 (22.2)    18.8 (23.2)
//                            16 (5.3)   21.7 (22.6)    22.4 (30.1)
//     1024    8 x 64 bf16    32 (10.7)  37.3 (38.1)    23.0 (34.5)
//                            8 (2.7)    37.9 (51.3)    39.9 (81.0)
//     2048    8 x 64 bf16    8 (2.7)    70.3 (97.1)    55.4 (128)
//                            4 (1.3)    73.2 (141)     85.2 (245)
//     2048    4 x 128 bf16   16 (5.3)   146 (146)      51.9 (105)
//                            8 (2.7)    147 (148)      71.8 (205)
// One sequence of 384 tokens gains little (8 x 64 bf16: 17.1 and 18.6; 4 x 128
// 31.7 and 29.0; 4 x 64 fp32 29.3 and 23.9).
// They are as long as fills the chip once: four workgroups a CU, two above 64
// columns (one sequence of 32768, 8 heads of 128 bf16: 109 us with two, 144 with
// four, 157 with one; of 65536, 8 heads of 64: 78 us with four, 91 with eight, 95
// with one and a half).
static int64_t segment_of(const ScanArgs& a) {
    const int64_t resident = std::max(a.role[0].q.dim, a.role[0].v.dim) > 64 ? 512 : 1024, lanes = (int64_t)a.heads * a.n_roles;
    if (a.longest <= 384) return 0;
    const double idle = (double)a.longest * resident / ((double)a.tokens * lanes);
    if (idle < 6.0 || (double)a.longest * idle <= 8192.0) return 0;
    const int64_t want = resident / lanes + 1;  // slots
    return std::max<int64_t>((a.tokens / want + C - 1) / C * C, 128);
}

static int64_t slots_of(const ScanArgs& a, int64_t seg) { return seg ? a.n + a.tokens / seg : a.n; }

size_t scan_workspace_bytes(const ScanArgs& a) {
    const int64_t seg = segment_of(a);
    return seg ? (size_t)a.n_roles * slots_of(a, seg) * a.heads * a.role[0].q.dim * a.role[0].v.dim * 4 : 16;
}

template <typename T, int D, int NT, int TI, bool WIDE, int PIECES>
static hipError_t scan(const ScanArgs& a, hipStream_t s) {
    const int inner = a.n_roles * a.together;
    const int64_t rest = (a.slots * (a.heads / a.together) + 7) / 8, blocks = rest * 8 * inner;
    dim3 grid;
    if (a.seg) {
        if (!grid_of(blocks, scan_threads<D, NT, 2>(), grid)) return hipErrorInvalidValue;
        k_scan<T, D, NT, 2, WIDE, 3, true><<<grid, scan_threads<D, NT, 2>(), 0, s>>>(a);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int size = a.role[0].q.dim * a.role[0].v.dim;
        if (!grid_of((int64_t)a.n * a.heads, 256, grid)) return hipErrorInvalidValue;
        grid.z = (size + 255) / 256 * a.n_roles;
        k_join_segments<<<grid, 256, 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (!grid_of(blocks, scan_threads<D, NT, TI>(), grid)) return hipErrorInvalidValue;
    k_scan<T, D, NT, TI, WIDE, PIECES, false><<<grid, scan_threads<D, NT, TI>(), 0, s>>>(a);
    return hipGetLastError();
}

template <typename T, int D, int NT, int TI>
static hipError_t scan_any(const ScanArgs& a, hipStream_t s) {
    bool wide = true, state = false;
    constexpr int V = 16 / sizeof(T);
    for (int r = 0; r < a.n_roles; ++r) {
        for (const HeadView* v : {&a.role[r].q, &a.role[r].k, &a.role[r].v})
            wide = wide && (reinterpret_cast<uintptr_t>(v->p) & 15) == 0 && v->dim % V == 0 && v->token_stride % V == 0 &&
                   v->head_stride % V == 0 && v->token_stride < (1 << 22);
        state = state || (a.role[r].final_state && !a.seg);
    }
    if constexpr (sizeof(T) == 4) {
        return wide ? scan<T, D, NT, TI, true, 1>(a, s) : scan<T, D, NT, TI, false, 1>(a, s);
    } else {
        if (state) return wide ? scan<T, D, NT, TI, true, 3>(a, s) : scan<T, D, NT, TI, false, 3>(a, s);
        return wide ? scan<T, D, NT, TI, true, 2>(a, s) : scan<T, D, NT, TI, false, 2>(a, s);
    }
}

hipError_t launch_scan(const ScanArgs& in, hipStream_t s) {
    ScanArgs a = in;
    a.seg = segment_of(a);
    a.slots = slots_of(a, a.seg);
    a.states = static_cast<float*>(a.ws);
    a.together = a.slots >= 64 ? a.heads : a.group;  // fewer slots would leave XCDs idle
    const int d = std::max(a.role[0].q.dim, a.role[0].v.dim);
    if (a.dtype) {
        if (d <= 32) return scan_any<bf16_t, 32, 1, 2>(a, s);
        if (d <= 64) return scan_any<bf16_t, 64, 1, 2>(a, s);
        return scan_any<bf16_t, 128, 2, 2>(a, s);
    }
    // The fp32 MFMA takes longest, so up to 32 columns a wave takes one token tile:
    // at 32 with half of the state (2048 units of 16 chunks 121 us, 139 with whole
    // states and both tiles; 256 units 24 and 29), at 16 only up to a unit a SIMD
    // (32 units 18 us against 22; 1024 units of 8 to 400 tokens, log-normal about 100,
    // 16.4 against 19.0, of 200 each 13.7 against 13.8; gradients as 1536 units of 50
    // tokens 11.1 against 8.6). bf16 gained nothing from it (2048 units 61 against 57).
    if (d <= 16)
        return a.slots * a.heads * a.n_roles <= 1024 ? scan_any<float, 16, 1, 1>(a, s) : scan_any<float, 16, 1, 2>(a, s);
    if (d <= 32) return scan_any<float, 32, 1, 1>(a, s);
    if (d <= 64) return scan_any<float, 64, 1, 2>(a, s);
    return scan_any<float, 128, 2, 2>(a, s);
}

hipError_t launch_sum_heads(int64_t tokens, int kv_heads, int group, int dim, int dtype, const float* src, void* dst,
                            hipStream_t s) {
    const int64_t n = tokens * kv_heads * dim;
    dim3 grid;
    if (!grid_of((n + 255) / 256, 256, grid)) return hipErrorInvalidValue;
    if (dtype)
        k_sum_heads<<<grid, 256, 0, s>>>(n, group, dim, src, static_cast<bf16_t*>(dst));
    else
        k_sum_heads<<<grid, 256, 0, s>>>(n, group, dim, src, static_cast<float*>(dst));
    return hipGetLastError();
}

template <typename T>
static hipError_t step(const StepArgs& a, hipStream_t s) {
    dim3 grid;
    if (!grid_of(a.n, 256, grid)) return hipErrorInvalidValue;
    grid.z = a.heads;
    const int dv = a.v.dim;
    if (dv % 4 == 0) {  // rows of the state are whole 16-byte vectors
        if (dv <= 16)
            k_step<T, 4, 4><<<grid, 256, 0, s>>>(a);
        else if (dv <= 32)
            k_step<T, 4, 8><<<grid, 256, 0, s>>>(a);
        else if (dv <= 64)
            k_step<T, 4, 16><<<grid, 256, 0, s>>>(a);
        else
            k_step<T, 4, 32><<<grid, 256, 0, s>>>(a);
    } else if (dv <= 32) {
        k_step<T, 1, 32><<<grid, 256, 0, s>>>(a);
    } else {
        k_step<T, 1, 128><<<grid, 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

hipError_t launch_step(const StepArgs& a, hipStream_t s) { return a.dtype ? step<bf16_t>(a, s) : step<float>(a, s); }

}  // namespace mdl
