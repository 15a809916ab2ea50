// Runs csrc/packed_spans.hpp on the host as the kernels run it: over the host's own offsets, and over offsets on the device that are others.
#include <algorithm>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "packed_spans.hpp"

static std::mt19937 rng(1);
static int any(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }
static void fail(const char *what, const std::vector<int> &off, int lo, int hi, int seg, int begin, int end)
{
    printf("%s: tokens %d .. %d, segments of %d, span %d .. %d, offsets", what, lo, hi, seg, begin, end);
    for (int o : off) printf(" %d", o);
    printf("\n");
    exit(1);
}

struct Seq {
    int begin, end, number;
};

// One call's spans; `own`: the offsets are the host's, so that every token is taken once, by its sequence.
static void check(const std::vector<int> &off, int lo, int hi, int seg, bool own)
{
    const int n = (int)off.size() - 1;
    auto get = [&](int i) {
        if (i < 0 || i >= n) fail("sequence number", off, lo, hi, seg, i, n);
        const Span s = n == 1 ? Span{lo, hi} : packed_clamped(off[i], off[i + 1], lo, hi);
        return Seq{s.begin, s.end, i};
    };
    auto find = [&](int t) {
        return packed_find_by(n, [&](int first, int step, int left) {
            int m = 0;
            for (int lane = 0; lane < 64; ++lane) {
                const int at = first + std::min((lane + 1) * step, left) - 1;
                if (at < 1 || at > n - 1) fail("offset's index", off, lo, hi, seg, at, n);
                m += off[at] <= t;
            }
            return m;
        });
    };
    auto inside = [&](const char *what, int a, int b, int from, int to) {
        if (!(from <= a && a < b && b <= to)) fail(what, off, lo, hi, seg, a, b);
    };
    std::vector<int> taken(hi - lo, -1);
    for (int w = 0; w < (hi - lo + seg - 1) / seg; ++w) {
        const int t0 = lo + w * seg, t1 = t0 + seg;
        packed_pieces(t0, std::min(t1, hi), find(t0), n, get, [&](const Seq &s, int a, int b) {
            inside("piece", a, b, t0, std::min(t1, hi));
            for (int t = a; t < b; ++t) {
                if (taken[t - lo] >= 0) fail("taken twice", off, lo, hi, seg, a, b);
                taken[t - lo] = s.number;
            }
        });
        if (t1 >= hi) continue;
        const Seq s = get(find(t1 - 1));
        const Span c = packed_carried({s.begin, s.end}, t0, t1);
        if (c.begin != c.end) inside("carried", c.begin, c.end, t0, t1);
        if (own) {
            // the sequence of the segment's last token, if it holds the next token too
            int of = n - 1;
            while (of > 0 && off[of] > t1 - 1) --of;
            const bool on = off[of + 1] > t1;
            if (on != (c.begin != c.end) || (on && c.begin != std::max(off[of], t0))) fail("what is carried", off, lo, hi, seg, c.begin, c.end);
        }
    }
    if (!own) return;
    for (int t = lo; t < hi; ++t) {
        int of = n - 1;
        while (of > 0 && off[of] > t) --of;
        if (taken[t - lo] != of) fail("sequence of a token", off, lo, hi, seg, t, taken[t - lo]);
    }
}

int main()
{
    for (int round = 0; round < 40000; ++round) {
        const int n = round % 50 == 0 ? any(1, 5000) : any(1, 12);
        const int lo = any(0, 1) ? 0 : any(0, 300), seg = any(1, 200);
        std::vector<int> off{lo};
        for (int i = 0; i < n; ++i) off.push_back(off.back() + (any(0, 2) ? any(0, n > 12 ? 3 : 260) : 0));
        const int hi = off.back();
        if (hi == lo) continue;
        check(off, lo, hi, seg, true);
        std::vector<int> other(off);
        const int how = any(0, 5);
        for (int &o : other) {
            if (how == 0) o = any(lo - 50, hi + 50);
            if (how == 1) o = any(INT_MIN, INT_MAX);
            if (how == 2) o = 0;                     // not copied yet
            if (how == 3) o += any(0, 400);          // another call's
            if (how == 4) o = any(0, 1) ? INT_MAX : INT_MIN;
            if (how == 5 && any(0, 3) == 0) o = any(lo, hi);
        }
        check(other, lo, hi, seg, false);
    }
    printf("ok\n");
}
