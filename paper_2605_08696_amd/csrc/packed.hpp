// Packed sequences on the device: which one a token belongs to, where its slot lies and what it starts from.  Offsets come from device
// memory and are clamped to the tokens that the host has validated, so that other values than the host's cannot lead outside the operands.
#pragma once
#include "common.hpp"

struct Packed {
    const int32_t *offsets, *pos, *slot;             // pos, slot: NULL = all 0, = the sequence's own number
    int32_t n, lo, hi;                               // sequences; the packed tokens are lo .. hi - 1
    int64_t slots;                                   // 0: nothing is kept
};
struct Sequence {
    int begin, end, pos;
    int64_t slot;                                    // -1: none
};
__device__ __forceinline__ Sequence packed_sequence(const Packed &c, int n)
{
    Sequence s;
    if (c.n == 1) {                                  // (one trip to memory less)
        s.begin = c.lo;
        s.end = c.hi;
    } else {
        s.begin = min(max(c.offsets[n], c.lo), c.hi);
        s.end = min(max(c.offsets[n + 1], s.begin), c.hi);
    }
    s.pos = c.pos ? c.pos[n] : 0;
    const int64_t slot = c.slot ? c.slot[n] : n;
    s.slot = slot >= 0 && slot < c.slots ? slot : -1;
    return s;
}
// The last sequence that begins at or before token t, by all lanes of a wavefront together: 64 offsets a look, so that 4096 sequences
// take two trips to memory (a search by halves takes one for each factor of two).
__device__ __forceinline__ int packed_find(const Packed &c, int t, int lane)
{
    int first = 1, left = c.n - 1;                   // offsets[first .. first + left - 1] may still be at or before t
    while (left > 0) {
        const int step = (left + 63) >> 6, at = min((lane + 1) * step, left);
        const int m = __popcll(__ballot(c.offsets[first + at - 1] <= t));
        // (lanes behind the last offset look at the last one: all of them or none count)
        const int gone = min(m * step, left);
        first += gone;
        left = step == 1 ? 0 : min(step - 1, left - gone);
    }
    return first - 1;
}
