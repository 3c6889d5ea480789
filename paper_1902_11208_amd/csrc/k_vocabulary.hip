// Softmax cross entropy of rows over a vocabulary, from the rows x [rows][dim] and
// the vocabulary's weights W [vocab][dim], without stored logits l = x W^T. With
// the sum over the others, o = log(sum over v != target of exp(l_v)),
//     loss = log(1 + exp(o - l_target))            1 - p_target = sigmoid(o - l_target)
//     dl_v = c q_v,  c = dloss (1 - p_target),  q_v = exp(l_v - o),  q_target = -1
//     dx = c (q W)        dW = (c q)^T x
// Written so, neither the loss nor the gradient of a row whose target is nearly
// certain is a difference of numbers near 1, and the target's share of dx enters its
// product without rounding.
//
// Everything is a product of two operands whose rows run along the summed
// dimension, C = A B^T on the matrix units (k_product): tiles of both operands go
// straight to LDS in pieces of 64 of that dimension, two buffers in turn, and
// products of 16 x 16 x 32 take them from there. The forward pass keeps of a tile of
// logits each row's maximum and sum. The backward pass takes the vocabulary in
// pieces: a piece's logits again, q in bf16 both ways round (q for dx, c q
// transposed for dW), and two products with the transposed W and x.
//
// fp32 operands are three bf16 numbers each (split.hpp), the six largest products
// kept. With x and W in bf16, q and c q are two bf16 numbers each, 2^-16 of
// themselves off. One would be 2^-8 off, and the sum of q over the vocabulary is 0:
// what W's rows have in common falls out of dx, and is left of it in proportion if
// q is rounded (2000 rows of 128 with a common part of 10 beside a spread of 0.18 a
// coordinate: dx 2.8e-3 off, in two pieces 1.7e-3, which is the result's own rounding).
//
// Matrix instructions bound it: 256 x 256 tiles in eight waves of 128 x 64 read 192 KB
// of operands from LDS a step of 64 and write 64, beside 2048 cycles of products, without
// bank conflicts. Measured, 16383 rows of 1024 in bf16 over 50021: dW's products 1370
// TFLOP/s (sums of 2 x 16384, the matrix units busy 68% of the cycles), dx's 1260 (60%),
// the logits 1000 (48%; a tile's prologue and its sums of exponentials take 10 of 33 us),
// the logits again with q written both ways round in two pieces 600 (28%; 2.1 GB of q for
// 16384 of the vocabulary in 920 us). 128 x 128 tiles, two workgroups a CU, reach 600 to 700:
// they read twice as much LDS a product.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "sequence.hpp"
#include "split.hpp"
#include "vocabulary.hpp"

namespace mdl {
namespace {

constexpr int BK = 64;           // summed elements of a step
constexpr float LOG2E = 1.4426950408889634f;

// An operand: `pieces` planes of [rows][ld] bf16, ld a multiple of BK or enough elements for whole steps.
struct Operand {
    const bf16_t* p;
    int64_t plane, ld;
    int64_t rows;
};

// What of a row the epilogues need.
struct RowInfo {
    float most, share;  // q = 2^(l log2(e) - most) share
    float scale;        // c
    int target;         // -1: the row is left out
};

enum { LOGSUM, GRADIENT, PLANES, RESULT };

// The tiles of a gradient's product and the parts of its sum (cut_of).
struct Cut {
    bool large = false;
    int parts = 1;
};

struct Product {
    Operand a, b;
    int steps;          // steps of one pair of pieces
    int pairs;          // 1; 2 of a's two pieces with b; 6 of the three pieces of each
    Cut cut;            // PLANES, RESULT: the tiles and the parts of the sum (one where nothing is set, or for a result)
    int tiles_m, tiles_n;
    // LOGSUM
    const int64_t* targets;
    float2* part;       // [tiles_n][a.rows] of the tile's columns but the target (join_sums)
    float* logit;       // [a.rows] the target's logit
    int64_t first;      // vocabulary index of b's first row
    // GRADIENT
    const RowInfo* info;
    bf16_t* q;          // planes of [a.rows][ldq], columns b.rows to ldq are zeroed
    bf16_t* qt;         // planes of [b.rows][ldt], columns a.rows to ldt are zeroed
    int64_t ldq, ldt, q_plane, qt_plane;
    // PLANES
    float* out;         // [cut.parts][a.rows][ldo]
    int64_t ldo;
    int add;            // to what is there
    // RESULT: [a.rows][ldo] as stored, times the rows' scale (k_finish)
    void* result;
    const RowInfo* rows;
};

// A tile of a product: BM x BN, waves of WM x WN.
template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, WAVES = BM / WM * (BN / WN), THREADS = WAVES * 64, MI = WM / 16,
                         NI = WN / 16, LOADS = (BM + BN) / 8 / WAVES, A_LOADS = BM / 8 / WAVES;
    static_assert(BM / 8 % WAVES == 0 && BN / 8 % WAVES == 0, "whole loads of a wave");
};

// Which pieces a pair of them multiplies, two bits each, the smallest products first:
// (2, 0) (0, 2) (1, 1) (0, 1) (1, 0) (0, 0) of three; (1, 0) (0, 0) where a has two.
constexpr uint32_t PIECES_A = 2 | 0 << 2 | 1 << 4 | 0 << 6 | 1 << 8, PIECES_B = 0 | 2 << 2 | 1 << 4 | 1 << 6 | 0 << 8;

typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer_at(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7ffffff0, 0x00027000);
}

// A tile's rows in LDS: 64 elements (128 bytes) each, their eight 16-byte chunks
// exchanged by the row's index (chunk c of row r lies at c ^ (r & 7)), so that
// the sixteen rows a matrix operand takes at once lie in different banks.
template <class S>
struct Tile {
    bf16_t a[S::BM * BK], b[S::BN * BK];
};

template <class S>
struct Loader {
    uint32_t offset[S::LOADS];  // bytes from the tile's first row
    __device__ __forceinline__ Loader(const Product& g, int64_t m0, int64_t n0) {
        const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < S::LOADS; ++i) {
            const bool a = i < S::A_LOADS;
            const int r = (a ? i : i - S::A_LOADS) * S::WAVES * 8 + wave * 8 + lane / 8;
            const Operand& o = a ? g.a : g.b;
            const int64_t last = o.rows - 1 - (a ? m0 : n0);  // rows behind the last one repeat it
            offset[i] = (uint32_t)((min((int64_t)r, last) * o.ld + ((lane & 7) ^ (lane / 8)) * 8) * 2);
        }
    }
    __device__ __forceinline__ void load(Tile<S>& t, Buffer a, Buffer b) const {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
#pragma unroll
        for (int i = 0; i < S::LOADS; ++i) {
            const bool is_a = i < S::A_LOADS;
            bf16_t* to = (is_a ? t.a + i * S::WAVES * 8 * BK : t.b + (i - S::A_LOADS) * S::WAVES * 8 * BK) + wave * 8 * BK;
#ifdef __HIP_DEVICE_COMPILE__  // the host's pass over this file has no such builtin
            __builtin_amdgcn_raw_ptr_buffer_load_lds(is_a ? a : b, (__attribute__((address_space(3))) void*)to, 16, offset[i], 0, 0, 0);
#endif
        }
    }
};

// Operands of half a step (32 summed elements) from a tile: N sixteens of rows from the wave's `first`.
template <int N>
__device__ __forceinline__ void read_rows(const bf16_t* tile, int first, int half, bf16x8 (&v)[N]) {
    const int lane = threadIdx.x & 63, row = lane & 15, chunk = ((lane / 16 + half * 4) ^ (row & 7)) * 8;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const bf16x8*>(tile + (first + i * 16 + row) * BK + chunk);
}

// Everything this wave asked of memory and LDS has come (vmcnt and lgkmcnt 0).
__device__ __forceinline__ void all_arrived() { __builtin_amdgcn_s_waitcnt(0x0070); }

// READS reads of LDS spread among PRODUCTS products, and nothing moved across.
template <int READS, int PRODUCTS>
__device__ __forceinline__ void interleave() {
#pragma unroll
    for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                  // a read of LDS
        __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS / READS, 0);  // products
    }
    __builtin_amdgcn_sched_barrier(0);
}

// over the sixteen lanes of a row of a matrix result
template <bool MAX>
__device__ __forceinline__ float over16(float v) {
    auto with = [&](auto turn) {
        const float o = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), turn(), 0xf, 0xf, false));
        v = MAX ? fmaxf(v, o) : v + o;
    };
    with(std::integral_constant<int, 0x128>());
    with(std::integral_constant<int, 0x124>());
    with(std::integral_constant<int, 0x122>());
    with(std::integral_constant<int, 0x121>());
    return v;
}

// Tiles in an order that keeps those of an XCD (workgroups 8 apart) near each
// other: runs of the list per XCD, the list in blocks of 8 rows of tiles.
__device__ __forceinline__ void place(const Product& g, int index, int& tm, int& tn) {
    const int total = g.tiles_m * g.tiles_n, each = total / 8, more = total % 8, xcd = index % 8, at = index / 8;
    const int k = xcd * each + min(xcd, more) + at;
    const int band = 8 * g.tiles_n, first = k / band * 8, high = min(8, g.tiles_m - first), in = k % band;
    tm = first + in % high;
    tn = in / high;
}

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// Sums of exponentials as (m, sum of 2^(l log2(e) - m)), m the rounded product of
// the largest l with log2(e): the same m is taken from every term, so its rounding does
// not matter. No columns: (-infinity, 0).
__device__ __forceinline__ float finite_or_0(float m) { return m == -__builtin_huge_valf() ? 0.0f : m; }
__device__ __forceinline__ float2 join_sums(float2 s, float2 n) {
    const float top = fmaxf(s.x, n.x), base = finite_or_0(top);
    return make_float2(top, s.y * exp2_of(s.x - base) + n.y * exp2_of(n.x - base));
}

// Piece k of a number.
__device__ __forceinline__ float piece(float v, int k) {
    for (int i = 0; i < k; ++i) v -= bf2f(f2bf(v));
    return v;
}

// To the compiler, other numbers than before.
template <class S>
__device__ __forceinline__ void as_new(floatx4 (&acc)[S::MI][S::NI]) {
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) asm volatile("" : "+v"(acc[i][j]));
}

// A tile's q as rows, and c q as columns, through LDS, so that whole lines leave.
// A half of the tile lies in each of two buffers, in rows of whole 16-byte chunks that
// are exchanged by the row's index, so that the lanes of a write meet different banks.
template <class S>
__device__ __forceinline__ void store_rows(const Product& g, bf16_t* b0, bf16_t* b1, const floatx4 (&acc)[S::MI][S::NI], int k, int64_t m0,
                                           int64_t n0) {
    constexpr int ROW = S::BN / 2, CHUNKS = S::BN / 8;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wm = wave / (S::BN / S::WN), wn = wave % (S::BN / S::WN);
    const int quad = lane / 16, col = lane & 15;
    bf16_t* to = wn * S::WN < ROW ? b0 : b1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = wn * S::WN % ROW + j * 16 + col, m = wm * S::WM + i * 16 + quad * 4;
            bf16_t* at = to + m * ROW + ((n / 8) ^ (quad << 1)) * 8 + n % 8;
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                const uint32_t two = f2bf2(piece(acc[i][j][r], k), piece(acc[i][j][r + 1], k));
                at[r * ROW] = (bf16_t)two;
                at[(r + 1) * ROW] = (bf16_t)(two >> 16);
            }
        }
    __syncthreads();
    bf16_t* q = g.q + k * g.q_plane;
    for (int x = threadIdx.x; x < S::BM * CHUNKS; x += S::THREADS) {
        const int m = x / CHUNKS, c = x % CHUNKS;
        const bf16_t* from = (c < CHUNKS / 2 ? b0 : b1) + m * ROW + ((c % (CHUNKS / 2)) ^ ((m / 4 & 3) << 1)) * 8;
        const u32x4 v = *reinterpret_cast<const u32x4*>(from);
        if (m0 + m < g.a.rows && n0 + c * 8 < g.ldq) *reinterpret_cast<u32x4*>(q + (m0 + m) * g.ldq + n0 + c * 8) = v;
    }
}

template <class S>
__device__ __forceinline__ void store_columns(const Product& g, bf16_t* b0, bf16_t* b1, const floatx4 (&acc)[S::MI][S::NI],
                                              const float (&scale)[S::MI][4], int k, int64_t m0, int64_t n0) {
    constexpr int ROW = S::BM, CHUNKS = S::BM / 8, HALF = S::BN / 2, MASK = S::BM / 16 - 1;
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wm = wave / (S::BN / S::WN), wn = wave % (S::BN / S::WN);
    const int quad = lane / 16, col = lane & 15;
    bf16_t* to = wn * S::WN < HALF ? b0 : b1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) {
            const int n = wn * S::WN % HALF + j * 16 + col, m = wm * S::WM + i * 16 + quad * 4;
            uint32_t two[2];
#pragma unroll
            for (int r = 0; r < 4; r += 2)
                two[r / 2] = f2bf2(piece(acc[i][j][r] * scale[i][r], k), piece(acc[i][j][r + 1] * scale[i][r + 1], k));
            *reinterpret_cast<uint2*>(to + n * ROW + ((m / 8) ^ ((n & MASK) << 1)) * 8 + m % 8) = make_uint2(two[0], two[1]);
        }
    __syncthreads();
    bf16_t* qt = g.qt + k * g.qt_plane;
    for (int x = threadIdx.x; x < S::BN * CHUNKS; x += S::THREADS) {
        const int n = x / CHUNKS, c = x % CHUNKS;
        const bf16_t* from = (n < HALF ? b0 : b1) + n % HALF * ROW + (c ^ ((n & MASK) << 1)) * 8;
        const u32x4 v = *reinterpret_cast<const u32x4*>(from);
        if (n0 + n < g.b.rows && m0 + c * 8 < g.ldt) *reinterpret_cast<u32x4*>(qt + (n0 + n) * g.ldt + m0 + c * 8) = v;
    }
}

template <class S, int WHAT, int PIECES>
__global__ __launch_bounds__(S::THREADS) void k_product(Product g) {
    __shared__ Tile<S> t0;
    __shared__ Tile<S> t1;
    int tm, tn;
    place(g, blockIdx.x, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const int64_t m0 = (int64_t)tm * S::BM, n0 = (int64_t)tn * S::BN;
    const int all = g.steps * g.pairs, split = blockIdx.y;
    const int from = __builtin_amdgcn_readfirstlane((int)((int64_t)all * split / g.cut.parts)),
              to = __builtin_amdgcn_readfirstlane((int)((int64_t)all * (split + 1) / g.cut.parts));
    const Loader<S> load(g, m0, n0);
    const bf16_t *pa = g.a.p + m0 * g.a.ld, *pb = g.b.p + n0 * g.b.ld;
    int pair = __builtin_amdgcn_readfirstlane(g.steps ? from / g.steps : 0), step = from - pair * g.steps, left = to - from;  // of the next fetch
    const uint32_t pieces_a = g.pairs == 6 ? PIECES_A : g.pairs - 1, pieces_b = g.pairs == 6 ? PIECES_B : 0;
    auto fetch = [&](Tile<S>& t) {  // behind the last step: that one again
        const int64_t a = (pieces_a >> 2 * pair & 3) * g.a.plane, b = (pieces_b >> 2 * pair & 3) * g.b.plane;
        load.load(t, buffer_at(pa + a + (int64_t)step * BK), buffer_at(pb + b + (int64_t)step * BK));
        const int more = --left > 0, wrap = more & (step + 1 == g.steps);
        pair += wrap;
        step = wrap ? 0 : step + more;
    };
    floatx4 acc[S::MI][S::NI];
#pragma unroll
    for (int i = 0; i < S::MI; ++i)
#pragma unroll
        for (int j = 0; j < S::NI; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    // A step's tile is asked for a whole step before it is read, and a quarter step's
    // operands are read while the quarter before multiplies. Before the last quarter,
    // one barrier: the next tile has arrived, and all waves have read this one, whose
    // place the tile after the next takes.
    constexpr int MH = S::MI / 2, NI = S::NI;
    const int wm0 = threadIdx.x / 64 / (S::BN / S::WN) * S::WM, wn0 = threadIdx.x / 64 % (S::BN / S::WN) * S::WN;
    bf16x8 a0[MH], a1[MH], b0[NI], b1[NI];
    auto multiply = [&](const bf16x8(&a)[MH], const bf16x8(&b)[NI], auto high) {
#pragma unroll
        for (int i = 0; i < MH; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[high() * MH + i][j] = mfma_bf16(a[i], b[j], acc[high() * MH + i][j]);
    };
    const std::integral_constant<int, 0> low;
    const std::integral_constant<int, 1> high;
    auto one = [&](Tile<S>& now, Tile<S>& next) {
        read_rows(now.a, wm0 + MH * 16, 0, a1);
        multiply(a0, b0, low);
        interleave<MH, MH * NI>();
        read_rows(now.a, wm0 + MH * 16, 1, a0);
        read_rows(now.b, wn0, 1, b1);
        multiply(a1, b0, high);
        interleave<MH + NI, MH * NI>();
        read_rows(now.a, wm0, 1, a1);
        multiply(a0, b1, high);
        interleave<MH, MH * NI>();
        all_arrived();
        __builtin_amdgcn_s_barrier();
        fetch(now);
        read_rows(next.a, wm0, 0, a0);
        read_rows(next.b, wn0, 0, b0);
        multiply(a1, b1, low);
        interleave<MH + NI, MH * NI>();
    };
    if (from < to) {
        fetch(t0);
        all_arrived();
        __builtin_amdgcn_s_barrier();
        fetch(t1);
        read_rows(t0.a, wm0, 0, a0);
        read_rows(t0.b, wn0, 0, b0);
        int k = from;
        for (; k + 2 <= to; k += 2) {
            one(t0, t1);
            one(t1, t0);
        }
        if (k < to) one(t0, t1);
    }
    __syncthreads();
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63, wm = wave / (S::BN / S::WN), wn = wave % (S::BN / S::WN);
    const int quad = lane / 16, col = lane & 15;
    const int64_t rows = g.a.rows, cols = g.b.rows;
    if constexpr (WHAT == PLANES) {
        float* out = g.out + (int64_t)split * rows * g.ldo;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t m = m0 + wm * S::WM + i * 16 + quad * 4 + r;
#pragma unroll
                for (int j = 0; j < S::NI; ++j) {
                    const int64_t n = n0 + wn * S::WN + j * 16 + col;
                    if (m < rows && n < cols) {
                        float* p = out + m * g.ldo + n;
                        *p = g.add ? *p + acc[i][j][r] : acc[i][j][r];
                    }
                }
            }
    } else if constexpr (WHAT == RESULT) {
        typedef std::conditional_t<PIECES == 1, bf16_t, float> T;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t m = m0 + wm * S::WM + i * 16 + quad * 4 + r;
                if (m >= rows) continue;
                RowInfo f = {0.0f, 0.0f, 1.0f, 0};
                if (g.rows) f = g.rows[m];
#pragma unroll
                for (int j = 0; j < S::NI; ++j) {
                    const int64_t n = n0 + wn * S::WN + j * 16 + col;
                    if (n >= cols) continue;
                    float v = acc[i][j][r];
                    if (g.rows) v = f.target < 0 ? 0.0f : v * f.scale;
                    St<T>::st1(static_cast<T*>(g.result) + m * g.ldo + n, v);
                }
            }
    } else if constexpr (WHAT == LOGSUM) {
        int* target = reinterpret_cast<int*>(t0.a);  // of the tile's rows, counted from the tile's first column
        float2* sums = reinterpret_cast<float2*>(t1.a);  // [BN / WN][BM]
        for (int r = threadIdx.x; r < S::BM; r += S::THREADS) {
            const int64_t t = m0 + r < rows ? g.targets[m0 + r] : -1, at = t < 0 ? -1 : t - g.first - n0;
            target[r] = at >= 0 && at < S::BN && at < cols - n0 ? (int)at : -(1 << 20);
        }
        __syncthreads();
        const bool ragged = n0 + S::BN > cols;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = wm * S::WM + i * 16 + quad * 4 + r, t = target[row] - wn * S::WN - col;
                float v[S::NI], top = -__builtin_huge_valf(), sum = 0.0f;
#pragma unroll
                for (int j = 0; j < S::NI; ++j) v[j] = acc[i][j][r];
                // rows whose target is in the wave's columns, and columns behind the last, are rare
                if (ragged || __any(t > -16 && t < S::WN)) {
#pragma unroll
                    for (int j = 0; j < S::NI; ++j) {
                        if (t == j * 16) g.logit[m0 + row] = v[j];
                        if (t == j * 16 || n0 + wn * S::WN + j * 16 + col >= cols) v[j] = -__builtin_huge_valf();
                    }
                }
#pragma unroll
                for (int j = 0; j < S::NI; ++j) top = fmaxf(top, v[j]);
                top = over16<true>(top) * LOG2E;
                const float base = finite_or_0(top);
#pragma unroll
                for (int j = 0; j < S::NI; ++j) sum += exp2_of(fmaf(v[j], LOG2E, -base));
                sum = over16<false>(sum);
                if (col == 0) sums[wn * S::BM + row] = make_float2(top, sum);
            }
        __syncthreads();
        for (int r = threadIdx.x; r < S::BM; r += S::THREADS) {
            if (m0 + r >= rows) break;
            float2 s = sums[r];
#pragma unroll
            for (int w = 1; w < S::BN / S::WN; ++w) {
                s = join_sums(s, sums[w * S::BM + r]);
            }
            g.part[(int64_t)tn * rows + m0 + r] = s;
        }
    } else {
        RowInfo* info = reinterpret_cast<RowInfo*>(t0.a);
        for (int r = threadIdx.x; r < S::BM; r += S::THREADS) {
            info[r] = g.info[min(m0 + r, rows - 1)];
            if (m0 + r >= rows) info[r].target = -1;
        }
        __syncthreads();
        // q into the accumulators' place
        const bool ragged = n0 + S::BN > cols;
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const RowInfo f = info[wm * S::WM + i * 16 + quad * 4 + r];
                const int t = f.target < 0 ? -(1 << 20) : (int)min(max(f.target - g.first - n0 - wn * S::WN - col, (int64_t)-1024), (int64_t)1024);
#pragma unroll
                for (int j = 0; j < S::NI; ++j) acc[i][j][r] = exp2_of(fmaf(acc[i][j][r], LOG2E, -f.most)) * f.share;
                if (ragged || __any(t == -(1 << 20) || (t > -16 && t < S::WN))) {
#pragma unroll
                    for (int j = 0; j < S::NI; ++j) {
                        if (t == j * 16) acc[i][j][r] = -1.0f;
                        if (t == -(1 << 20) || n0 + wn * S::WN + j * 16 + col >= cols) acc[i][j][r] = 0.0f;
                    }
                }
            }
        float scale[S::MI][4];
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const RowInfo f = info[wm * S::WM + i * 16 + quad * 4 + r];
                scale[i][r] = f.target < 0 ? 0.0f : f.scale;
            }
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            // each pass takes its pieces from q again: kept from the pass before they would not fit the registers
            as_new<S>(acc);
            store_rows<S>(g, t0.a, t1.a, acc, k, m0, n0);
            as_new<S>(acc);
            store_columns<S>(g, t0.a, t1.a, acc, scale, k, m0, n0);
        }
    }
}

// o - l_target of a row, from the sum over the others (m, sum). m is rounded at its own
// size, and stays apart: every term has met the same m, and here it meets the target's logit
// before anything smaller. In one number with the sum's logarithm, at logits of 1000,
// losses and all q of a row were up to 4e-5 off.
__device__ __forceinline__ float sum_minus(float m, float sum, float logit) {
    return (fmaf(-logit, LOG2E, m) + log2f(sum)) * 0.693147180559945309f;
}

// A row's parts together: the sum over the others and the loss. Sixteen rows a
// workgroup, 64 slices of the parts, joined in a fixed order.
__global__ __launch_bounds__(1024) void k_losses(VocabularyArgs a, const float2* part, int64_t parts) {
    __shared__ float2 lds[64][16];
    const int in = threadIdx.x % 16, slice = threadIdx.x / 16;
    const int64_t r = (int64_t)blockIdx.x * 16 + in;
    float2 s = make_float2(-__builtin_huge_valf(), 0.0f);
    if (r < a.rows)
        for (int64_t k = slice; k < parts; k += 64) s = join_sums(s, part[k * a.rows + r]);
    lds[slice][in] = s;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        __syncthreads();
        if (slice < o) lds[slice][in] = s = join_sums(s, lds[slice + o][in]);
    }
    if (slice != 0 || r >= a.rows) return;
    const int64_t t = a.targets[r];
    const bool counts = t >= 0 && t < a.vocab;
    const float d = sum_minus(s.x, s.y, a.stats[a.rows + r]);  // no others: -infinity
    a.stats[r] = s.x;
    a.stats[a.rows + r] = s.y;
    a.losses[r] = !counts ? 0.0f : d > 0.0f ? d + log1pf(expf(-d)) : log1pf(expf(d));
}

// What the products need of row r, by a wave. The target's logit again: the forward pass leaves the sum's two numbers.
template <typename T>
__device__ __forceinline__ void find_row_info(const VocabularyArgs& a, int64_t r, RowInfo* info) {
    const int lane = threadIdx.x & 63;
    const int64_t t = a.targets[r];
    RowInfo v = {0.0f, 0.0f, 0.0f, -1};
    if (t >= 0 && t < a.vocab) {
        const T *x = static_cast<const T*>(a.x.p) + r * a.x.stride, *w = static_cast<const T*>(a.w.p) + t * a.w.stride;
        float logit = 0.0f;
#pragma unroll 4
        for (int c = lane; c < a.dim; c += 64) logit = fmaf(St<T>::ld1(x + c), St<T>::ld1(w + c), logit);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) logit += __shfl_xor(logit, o);
        const float m = a.stats[r], sum = a.stats[a.rows + r], d = sum_minus(m, sum, logit);
        v.most = finite_or_0(m);  // no others: there is no q
        v.share = sum == 0.0f ? 0.0f : 1.0f / sum;
        v.scale = a.dloss[r] * (d < 0.0f ? expf(d) / (1.0f + expf(d)) : 1.0f / (1.0f + expf(-d)));
        v.target = (int)t;
    }
    if (lane == 0) info[r] = v;
}

// The pieces of eight numbers at p, p + plane, ..., 16-byte aligned.
template <typename T>
__device__ __forceinline__ void put(bf16_t* p, int64_t plane, float (&v)[8]) {
#pragma unroll
    for (int n = 0; n < Pieces<T>::N; ++n) {
        uint32_t two[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            two[i] = f2bf2(v[2 * i], v[2 * i + 1]);
            v[2 * i] -= __uint_as_float(two[i] << 16);
            v[2 * i + 1] -= __uint_as_float(two[i] & 0xffff0000u);
        }
        *reinterpret_cast<u32x4*>(p + n * plane) = u32x4{two[0], two[1], two[2], two[3]};
    }
}

// Rows as an operand: fp32 in three pieces, [rows][ld] padded with zeros (NULL: not
// wanted); and transposed, [cols][ldt], ldt >= rows a multiple of 64, where rows that
// `targets` leaves out are zero (NULL: not wanted).
struct Copy {
    RowView src;
    int64_t rows;
    int cols;
    bf16_t* dst;
    int64_t plane, ld;
    bf16_t* dst_t;
    int64_t plane_t, ldt;
    const int64_t* targets;
    int vocab;
};

template <typename T>
__device__ __forceinline__ void pack(const Copy& p, int64_t chunk) {  // eight elements
    const int64_t r = chunk * 8 / p.ld, c = chunk * 8 - r * p.ld;
    if (r >= p.rows) return;
    const T* from = static_cast<const T*>(p.src.p) + r * p.src.stride + c;
    float v[8];
    if (c + 8 <= p.cols && (reinterpret_cast<uintptr_t>(from) & (4 * sizeof(T) - 1)) == 0) {
        const floatx4 a = St<T>::ld4(from), b = St<T>::ld4(from + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < p.cols ? St<T>::ld1(from + i) : 0.0f;
    }
    put<T>(p.dst + chunk * 8, p.plane, v);
}

template <typename T>
__device__ __forceinline__ void pack_transposed(const Copy& p, int64_t index, float (*lds)[65]) {  // 64 rows of 64 columns
    const int blocks = (p.cols + 63) / 64, c0 = (int)(index % blocks) * 64;
    const int64_t r0 = index / blocks * 64;
#pragma unroll 4
    for (int k = threadIdx.x; k < 64 * 64; k += 256) {
        const int64_t r = r0 + k / 64;
        const int c = c0 + k % 64;
        bool there = r < p.rows && c < p.cols;
        if (there && p.targets) there = p.targets[r] >= 0 && p.targets[r] < p.vocab;
        lds[k / 64][k % 64] = there ? St<T>::ld1(static_cast<const T*>(p.src.p) + r * p.src.stride + c) : 0.0f;
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 64 * 8; k += 256) {  // eight rows of the source a chunk
        const int r = k % 8 * 8, c = k / 8;
        if (c0 + c >= p.cols) break;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lds[r + i][c];
        put<T>(p.dst_t + (c0 + c) * p.ldt + r0 + r, p.plane_t, v);
    }
}

// What a product needs first, side by side in one launch: x and W as operands, the rows'
// info.
struct Prepare {
    Copy copy[2];
    VocabularyArgs a;
    RowInfo* info;          // or NULL
    int64_t end[5];         // workgroups up to the end of each part
};
template <typename T>
__global__ __launch_bounds__(256) void k_prepare(Prepare p) {
    __shared__ float lds[64][65];
    const int64_t block = block_index();
    int part = 0;
    while (part < 5 && block >= p.end[part]) ++part;
    if (part == 5) return;
    const int64_t index = block - (part ? p.end[part - 1] : 0);
    if (part < 2) {
        pack_transposed<T>(p.copy[part], index, lds);
    } else if (part < 4) {
        pack<T>(p.copy[part - 2], index * 256 + threadIdx.x);
    } else {
        const int64_t r = index * 4 + threadIdx.x / 64;
        if (r < p.a.rows) find_row_info<T>(p.a, r, p.info);
    }
}

// The planes of a product together, in order, times the row's scale (info), as
// stored. Rows without a scale come as one.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_finish(const float* planes, int splits, int64_t rows, int64_t cols, int blocks, const RowInfo* info,
                                                T* out) {
    const int64_t index = block_index(), r = index / blocks, c = ((index - r * blocks) * 256 + threadIdx.x) * 4;
    if (r >= rows || c >= cols) return;
    floatx4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    const int n = (int)min(cols - c, (int64_t)4);
#pragma unroll 4
    for (int k = 0; k < splits; ++k) {
        const float* p = planes + (k * rows + r) * cols + c;
        if (VEC) {
            s += *reinterpret_cast<const floatx4*>(p);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) s[i] += p[i];
        }
    }
    if (info) {
        const RowInfo f = info[r];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = f.target < 0 ? 0.0f : s[i] * f.scale;
    }
    T* to = out + r * cols + c;
    if (VEC) {
        St<T>::st4(to, s);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) St<T>::st1(to + i, s[i]);
    }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

typedef Shape<256, 256, 128, 64> Large;
typedef Shape<128, 128, 64, 64> Middle;
typedef Shape<64, 128, 64, 32> Low;

// The logits' tiles: Low where the rows fill half a middle one at most, Large where they
// still give most CUs a tile. Forward at 64 rows, 1024 channels and 50000 words:
// Low 26 us, Middle 31, Large 44. Forward and backward at 4000 rows: 4000 words of
// 1024 channels (256 large tiles) Large 44 / 220, Middle 49 / 221 us; at 2000 rows
// and 5000 words of 512 channels (160) Middle 32 / 126, Large 34 / 134.
template <bool ANY = true, typename F>
auto with_shape(int64_t m, int64_t n, F&& f) {
    if (m <= 64) return f(Low());
    if constexpr (ANY)
        if ((m + 255) / 256 * ((n + 255) / 256) >= 192) return f(Large());
    return f(Middle());
}

// The tiles of a gradient's product and the parts of its sum, with which it fills the
// chip: those that take the least time by a model of it. A round of workgroups takes as
// long as their steps (1.9 us of a large tile alone on its CU; 1.5 and 0.8 us of the
// others, two on a CU) and two more to start and end; every part's plane is written and
// read once, at 5 TB/s. Backward with large tiles from 192 of them on, whatever the
// parts, against this, in bf16: 4000 rows of 512 over 12000 448 and 399 us, 20000 of 256
// over 2000 307 and 289, 5000 of 1000 over 30000 1834 and 1695, 4000 of 512 over 3000 138
// and 141, 1000 of 256 over 100000 722 and 737.
template <class S>
double time_of(int64_t m, int64_t n, int64_t steps, int& parts) {
    const int64_t tiles = (m + S::BM - 1) / S::BM * ((n + S::BN - 1) / S::BN), slots = S::BM == 256 ? 256 : 512;
    const double step = S::BM == 256 ? 1.9 : S::BM == 128 ? 1.5 : 0.8, plane = (double)m * n * 8 / 5e6;
    double least = 1e300;
    for (int64_t k = 1; k <= std::max<int64_t>(1, std::min<int64_t>(64, steps / 4)); ++k) {
        const double time = (double)((tiles * k + slots - 1) / slots) * ((steps + k - 1) / k + 2) * step + k * plane;
        if (time < least) least = time, parts = (int)k;
    }
    return least;
}
Cut cut_of(int64_t m, int64_t n, int64_t steps) {
    Cut large{true, 1}, small{false, 1};
    if (m <= 64) {
        (void)time_of<Low>(m, n, steps, small.parts);
        return small;
    }
    return time_of<Large>(m, n, steps, large.parts) < time_of<Middle>(m, n, steps, small.parts) ? large : small;
}

template <int WHAT, int PIECES = 1>
hipError_t product(Product g, hipStream_t s) {
    auto launch = [&](auto shape) {
        typedef decltype(shape) S;
        g.tiles_m = (int)((g.a.rows + S::BM - 1) / S::BM);
        g.tiles_n = (int)((g.b.rows + S::BN - 1) / S::BN);
        k_product<S, WHAT, PIECES><<<dim3((unsigned)(g.tiles_m * g.tiles_n), (unsigned)g.cut.parts), S::THREADS, 0, s>>>(g);
        return hipGetLastError();
    };
    if constexpr (WHAT == PLANES || WHAT == RESULT) return g.a.rows <= 64 ? launch(Low()) : g.cut.large ? launch(Large()) : launch(Middle());
    // three pieces of q leave middle tiles no slower than large ones: backward of 1537 rows of 256 over 7003 in fp32 201
    // against 212 us, of 4000 rows of 512 over 12000 1151 against 1138
    return with_shape<WHAT != GRADIENT || PIECES != 3>(g.a.rows, g.b.rows, launch);
}

int64_t column_tile(int64_t m, int64_t n) {
    return with_shape(m, n, [](auto shape) { return (int64_t)decltype(shape)::BN; });
}

// Where everything lies in a call's workspace, and how the vocabulary is cut.
struct Plan {
    int64_t piece, dimp, rowsp;   // vocabulary rows of a piece, dim and rows in whole steps
    int pieces, q_pieces;         // of an operand's numbers, of q's
    int64_t x, w, part, info, xt, wt, q, qt, dx, dw, total;  // offsets
    int pairs() const { return pieces == 1 ? 1 : 6; }
    int q_pairs() const { return pieces == 1 ? 2 : 6; }
    Cut cut_dx(const VocabularyArgs& a) const { return cut_of(a.rows, a.dim, piece / BK * q_pairs()); }
    Cut cut_dw(const VocabularyArgs& a, int64_t n) const { return cut_of(n, a.dim, rowsp / BK * q_pairs()); }
};

bool direct(const VocabularyArgs& a, const RowView& v) {
    return a.dtype && a.dim % BK == 0 && v.stride % 8 == 0 && v.stride < (1 << 22) && (reinterpret_cast<uintptr_t>(v.p) & 15) == 0;
}

Plan plan_of(const VocabularyArgs& a, bool backward) {
    Plan p{};
    p.pieces = a.dtype ? 1 : 3;
    p.q_pieces = a.dtype ? 2 : 3;
    p.dimp = up(a.dim, BK);
    p.rowsp = up(std::max<int64_t>(a.rows, 1), BK);
    // Pieces of at most 2^28 logits and 2^16 weights; where there are several, with
    // as many rows of large tiles as make dW's tiles a multiple of the 256 CUs.
    int64_t most = std::max<int64_t>(256, std::min<int64_t>(65536, ((int64_t)1 << 28) / p.rowsp / 256 * 256)), even = 256;
    while (even / 256 * ((a.dim + 255) / 256) % 256 && even < most) even *= 2;
    if (even <= most) most = most / even * even;
    p.piece = std::min<int64_t>(up(a.vocab, BK), most);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t from = at;
        at += up(bytes, 256);
        return from;
    };
    // whether the operands lie as products want them is known at the call only
    p.x = take(p.rowsp * p.dimp * 2 * p.pieces);
    p.w = take(p.piece * p.dimp * 2 * p.pieces);
    if (!backward) {
        p.part = take((a.vocab / 128 + 2 + (a.vocab + p.piece - 1) / p.piece) * a.rows * 8);
    } else {
        p.info = take(a.rows * (int64_t)sizeof(RowInfo));
        p.xt = take(a.dim * p.rowsp * 2 * p.pieces);
        p.wt = take(a.dim * p.piece * 2 * p.pieces);
        p.q = take(p.rowsp * p.piece * 2 * p.q_pieces);
        p.qt = take(p.rowsp * p.piece * 2 * p.q_pieces);
        const int64_t rest = a.vocab % p.piece;
        p.dx = take(p.cut_dx(a).parts * a.rows * a.dim * 4);
        p.dw = take(std::max(p.cut_dw(a, std::min<int64_t>(p.piece, a.vocab)).parts * p.piece, rest ? p.cut_dw(a, rest).parts * rest : 0) * a.dim * 4);
    }
    p.total = std::max<int64_t>(at, 16);
    return p;
}

#define OK_OR_RETURN(expr)                     \
    do {                                       \
        const hipError_t _e = (expr);          \
        if (_e != hipSuccess) return _e;       \
    } while (0)

template <typename T>
hipError_t finish(const float* planes, int splits, int64_t rows, int64_t cols, const RowInfo* info, T* out, hipStream_t s) {
    const int64_t blocks = (cols + 1023) / 1024;
    dim3 grid;
    if (blocks > 0x7fffffff || !grid_of(rows * blocks, 256, grid)) return hipErrorInvalidValue;
    // a piece's rows of dW start anywhere in dW where dim is odd
    if (cols % 4 == 0 && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(T) - 1)) == 0)
        k_finish<T, true><<<grid, 256, 0, s>>>(planes, splits, rows, cols, (int)blocks, info, out);
    else
        k_finish<T, false><<<grid, 256, 0, s>>>(planes, splits, rows, cols, (int)blocks, info, out);
    return hipGetLastError();
}

template <typename T>
hipError_t prepare(Prepare p, hipStream_t s) {
    int64_t at = 0;
    for (int k = 0; k < 2; ++k) {
        const Copy& c = p.copy[k];
        if (c.dst_t) at += c.ldt / 64 * ((c.cols + 63) / 64);
        p.end[k] = at;
    }
    for (int k = 0; k < 2; ++k) {
        const Copy& c = p.copy[k];
        if (c.dst) at += (c.rows * c.ld / 8 + 255) / 256;
        p.end[2 + k] = at;
    }
    if (p.info) at += (p.a.rows + 3) / 4;
    p.end[4] = at;
    if (at == 0) return hipSuccess;
    dim3 grid;
    if (!grid_of(at, 256, grid)) return hipErrorInvalidValue;
    k_prepare<T><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
}

// x, and vocabulary rows first .. first + n - 1, as operands of the logits: as they are, or a copy in the workspace.
template <typename T>
Operand x_operand(const VocabularyArgs& a, const Plan& p, Copy& c) {
    c.src = a.x;
    c.rows = a.rows;
    c.cols = a.dim;
    if (direct(a, a.x)) return Operand{static_cast<const bf16_t*>(a.x.p), 0, a.x.stride, a.rows};
    c.dst = reinterpret_cast<bf16_t*>(static_cast<char*>(a.ws) + p.x);
    c.plane = p.rowsp * p.dimp;
    c.ld = p.dimp;
    return Operand{c.dst, c.plane, c.ld, a.rows};
}
template <typename T>
Operand w_operand(const VocabularyArgs& a, const Plan& p, int64_t first, int64_t n, Copy& c) {
    c.src = RowView{static_cast<const T*>(a.w.p) + first * a.w.stride, a.w.stride};
    c.rows = n;
    c.cols = a.dim;
    if (direct(a, a.w)) return Operand{static_cast<const bf16_t*>(c.src.p), 0, a.w.stride, n};
    c.dst = reinterpret_cast<bf16_t*>(static_cast<char*>(a.ws) + p.w);
    c.plane = p.piece * p.dimp;
    c.ld = p.dimp;
    return Operand{c.dst, c.plane, c.ld, n};
}

template <typename T>
hipError_t forward(const VocabularyArgs& a, hipStream_t s) {
    const Plan p = plan_of(a, false);
    char* ws = static_cast<char*>(a.ws);
    Prepare prep{};
    Product g{};
    g.a = x_operand<T>(a, p, prep.copy[0]);
    g.steps = (int)(p.dimp / BK);
    g.pairs = p.pairs();
    g.targets = a.targets;
    g.logit = a.stats + a.rows;
    float2* part = reinterpret_cast<float2*>(ws + p.part);
    // without a copy nothing cuts the vocabulary but the size of a launch
    const int64_t piece = direct(a, a.w) ? std::max(p.piece, ((int64_t)1 << 22) / ((a.rows + 63) / 64) * 128) : p.piece;
    int64_t parts = 0;
    for (int64_t first = 0; first < a.vocab; first += piece) {
        const int64_t n = std::min<int64_t>(piece, a.vocab - first);
        g.b = w_operand<T>(a, p, first, n, prep.copy[1]);
        OK_OR_RETURN(prepare<T>(prep, s));
        prep = Prepare{};
        g.first = first;
        g.part = part + parts * a.rows;
        OK_OR_RETURN(product<LOGSUM>(g, s));
        const int64_t tile = column_tile(a.rows, n);
        parts += (n + tile - 1) / tile;
    }
    k_losses<<<(unsigned)((a.rows + 15) / 16), 1024, 0, s>>>(a, part, parts);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const VocabularyArgs& a, hipStream_t s) {
    const Plan p = plan_of(a, true);
    char* ws = static_cast<char*>(a.ws);
    auto bf = [&](int64_t at) { return reinterpret_cast<bf16_t*>(ws + at); };
    auto f32 = [&](int64_t at) { return reinterpret_cast<float*>(ws + at); };
    RowInfo* info = reinterpret_cast<RowInfo*>(ws + p.info);
    T *dx = static_cast<T*>(a.dx), *dw = static_cast<T*>(a.dw);
    const int64_t xt_plane = a.dim * p.rowsp, wt_plane = a.dim * p.piece;
    for (int64_t first = 0; first < a.vocab; first += p.piece) {
        const int64_t n = std::min<int64_t>(p.piece, a.vocab - first), np = up(n, BK);
        Prepare prep{};
        Product g{};
        g.a = x_operand<T>(a, p, prep.copy[0]);
        g.b = w_operand<T>(a, p, first, n, prep.copy[1]);
        if (first == 0) {
            Copy& c = prep.copy[0];
            c.dst_t = bf(p.xt);
            c.plane_t = xt_plane;
            c.ldt = p.rowsp;
            c.targets = a.targets;
            c.vocab = a.vocab;
            prep.a = a;
            prep.info = a.rows > 0 ? info : nullptr;
        } else {
            prep.copy[0] = Copy{};  // is there
        }
        if (a.rows > 0) {
            Copy& c = prep.copy[1];
            c.dst_t = bf(p.wt);
            c.plane_t = wt_plane;
            c.ldt = np;
        } else {
            prep.copy[1] = Copy{};
        }
        OK_OR_RETURN(prepare<T>(prep, s));
        if (a.rows > 0) {
            g.steps = (int)(p.dimp / BK);
            g.pairs = p.pairs();
            g.first = first;
            g.info = info;
            g.q = bf(p.q);
            g.qt = bf(p.qt);
            g.ldq = np;
            g.ldt = p.rowsp;
            g.q_plane = g.qt_plane = p.rowsp * p.piece;
            OK_OR_RETURN((product<GRADIENT, sizeof(T) == 2 ? 2 : 3>(g, s)));
            Product x{};
            x.a = Operand{g.q, g.q_plane, np, a.rows};
            x.b = Operand{bf(p.wt), wt_plane, np, a.dim};
            x.steps = (int)(np / BK);
            x.pairs = p.q_pairs();
            x.cut = p.cut_dx(a);
            x.out = f32(p.dx);
            x.ldo = a.dim;
            x.add = first > 0;
            if (x.cut.parts == 1 && p.piece >= a.vocab) {
                x.result = dx;
                x.rows = info;
                OK_OR_RETURN((product<RESULT, Pieces<T>::N>(x, s)));
                dx = nullptr;
            } else {
                OK_OR_RETURN(product<PLANES>(x, s));
            }
        }
        Product v{};
        v.a = Operand{bf(p.qt), p.rowsp * p.piece, p.rowsp, n};
        v.b = Operand{bf(p.xt), xt_plane, p.rowsp, a.dim};
        v.steps = a.rows > 0 ? (int)(p.rowsp / BK) : 0;  // no rows: dW is zero
        v.pairs = p.q_pairs();
        v.cut = p.cut_dw(a, n);
        v.out = f32(p.dw);
        v.ldo = a.dim;
        // in one part, stored by the product: planes stored and read again took 1.4 us more where 500 rows of dW of 512
        // leave (backward of 64 rows 35.9 against 34.5 us) and 74 where 50000 of 1024 do (280 against 207 us)
        if (v.cut.parts == 1) {
            v.result = dw + first * a.dim;
            OK_OR_RETURN((product<RESULT, Pieces<T>::N>(v, s)));
        } else {
            OK_OR_RETURN(product<PLANES>(v, s));
            OK_OR_RETURN(finish<T>(v.out, v.cut.parts, 1, n * a.dim, nullptr, dw + first * a.dim, s));
        }
    }
    if (a.rows == 0 || !dx) return hipSuccess;  // no rows, or stored by the product
    return finish<T>(f32(p.dx), p.cut_dx(a).parts, a.rows, a.dim, info, dx, s);
}

}  // namespace

size_t vocabulary_workspace_bytes(const VocabularyArgs& a, bool backward) { return (size_t)plan_of(a, backward).total; }

hipError_t launch_vocabulary_fwd(const VocabularyArgs& a, hipStream_t s) {
    if (a.rows == 0) return hipSuccess;
    return a.dtype ? forward<bf16_t>(a, s) : forward<float>(a, s);
}
hipError_t launch_vocabulary_bwd(const VocabularyArgs& a, hipStream_t s) {
    return a.dtype ? backward<bf16_t>(a, s) : backward<float>(a, s);
}

}  // namespace mdl
