// Packed sequences and their segments, as kernels over packed tokens find them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mdl {

// Rows of elements, `stride` apart.
struct RowView {
    const void* p;
    int64_t stride;
};

// Sequence i is tokens offsets[i] to offsets[i + 1] - 1, cut to [0, tokens] and
// to `longest` tokens. Sequences longer than `seg` tokens are cut into segments
// (seg 0: none is): segment j of sequence i has slot offsets[i] / seg + i + j, so
// that no table is needed; slots in between stay empty.
struct Packed {
    int n;
    int64_t tokens, longest;
    const int64_t* offsets;
    const int32_t* order;  // sequences in the order they are started, or NULL
    int64_t seg, slots;
};

inline int64_t packed_slots(const Packed& p, int64_t seg) { return seg ? p.n + p.tokens / seg : p.n; }

// A sequence or a segment of one: tokens from .. to - 1 of the `len` tokens at t0.
struct Unit {
    int seq;
    int64_t slot, t0, len, from, to;
    int64_t edge;  // of a segment: (t0 + from - 1) / seg
};

__device__ __forceinline__ void sequence_of(const Packed& p, int seq, Unit& u) {
    const int64_t lo = min(max(p.offsets[seq], (int64_t)0), p.tokens), hi = min(max(p.offsets[seq + 1], lo), p.tokens);
    u.seq = seq;
    u.t0 = lo;
    u.len = min(hi - lo, p.longest);
    u.from = 0;
    u.to = u.len;
}

// False where the slot is empty.
__device__ __forceinline__ bool unit_of(const Packed& p, int64_t slot, Unit& u) {
    u.slot = slot;
    if (!p.seg) {
        const int seq = p.order ? p.order[slot] : (int)slot;
        if (seq < 0 || seq >= p.n) return false;
        sequence_of(p, seq, u);
        u.edge = 0;
        return true;
    }
    // The last sequence whose first slot is not behind `slot`: a wave looks at 64 places at once, as a load
    // depends on the one before (128 sequences: two loads, not seven). Called by whole waves.
    int lo = 0, hi = p.n - 1;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, at = lo + ((int)(threadIdx.x & 63) + 1) * step;
        const bool before = at <= hi && at > lo && min(max(p.offsets[at], (int64_t)0), p.tokens) / p.seg + at <= slot;
        const int steps = __popcll(__ballot(before));
        hi = min(hi, lo + (steps + 1) * step - 1);
        lo += steps * step;
    }
    sequence_of(p, lo, u);
    const int64_t before = u.t0 / p.seg;
    u.from = (slot - lo - before) * p.seg;
    u.edge = slot - lo - (before * p.seg == u.t0);
    u.to = min(u.len, u.from + p.seg);
    return u.from >= 0 && (u.from < u.len || u.from == 0);
}

}  // namespace mdl
