// Which tokens of packed sequences a work-group takes, in whole numbers alone: no device code, so that it can be run on the host over any
// offsets.  Offsets come from device memory.  Whatever they hold, every span that comes from here lies inside the tokens lo .. hi - 1 that the
// host has validated and is not empty: a kernel forms the bound of its loads from a span's length, and one below zero would be a bound of 4 GB.
#pragma once

#define PACKED_INLINE __attribute__((always_inline))

struct Span {
    int begin, end;
};
// A sequence's offsets, held inside the validated tokens.
PACKED_INLINE constexpr Span packed_clamped(int begin, int end, int lo, int hi)
{
    const int b = begin < lo ? lo : begin > hi ? hi : begin;
    return {b, end < b ? b : end > hi ? hi : end};
}
// The last of n sequences that begins at or before a token: count(first, step, left) looks at every step-th of the offsets first .. first +
// left - 1, the last one at the latest, 64 times, and returns how many looks met one at or before the token.
template <typename Count>
PACKED_INLINE constexpr int packed_find_by(int n, Count &&count)
{
    int first = 1, left = n - 1;                     // offsets[first .. first + left - 1] may still be at or before the token
    while (left > 0) {
        const int step = (left + 63) >> 6, m = count(first, step, left);
        // (lanes behind the last offset look at the last one: all of them or none count)
        const int gone = m * step < left ? m * step : left;
        first += gone;
        left = step == 1 ? 0 : step - 1 < left - gone ? step - 1 : left - gone;
    }
    return first - 1;
}
// What a sequence brings to the end of the segment [t0, t1) from which it runs on; nothing of one that ends there, or begins behind it (which
// the one that holds the segment's last token does not, with the host's offsets).
PACKED_INLINE constexpr Span packed_carried(Span s, int t0, int t1)
{
    if (s.end <= t1 || s.begin >= t1) return {t1, t1};
    return {s.begin > t0 ? s.begin : t0, t1};
}
// piece(sequence, begin, end) for the parts of [t0, t1) that belong to sequence n and those behind it; get(n): the sequence, with its clamped
// .begin and .end.  (Tokens behind the last sequence, which the host's offsets do not have, are left alone.)
template <typename Get, typename Piece>
PACKED_INLINE constexpr void packed_pieces(int t0, int t1, int n, int sequences, Get &&get, Piece &&piece)
{
    for (int t = t0; t < t1;) {
        auto s = get(n);
        while (t >= s.end && n + 1 < sequences) s = get(++n);
        if (t >= s.end) return;
        const int end = s.end < t1 ? s.end : t1;
        piece(s, t, end);
        t = end;
    }
}
