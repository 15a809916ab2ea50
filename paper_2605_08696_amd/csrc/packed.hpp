// Packed sequences on the device: which one a token belongs to, where its slot lies and what it starts from.  Offsets come from device
// memory and are clamped to the tokens that the host has validated, so that other values than the host's cannot lead outside the operands.
#pragma once
#include "common.hpp"
#include "packed_spans.hpp"

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
        const Span span = packed_clamped(c.offsets[n], c.offsets[n + 1], c.lo, c.hi);
        s.begin = span.begin;
        s.end = span.end;
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
    return packed_find_by(c.n, [&](int first, int step, int left) {
        return __popcll(__ballot(c.offsets[first + min((lane + 1) * step, left) - 1] <= t));
    });
}
