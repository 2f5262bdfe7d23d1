// Equal shares of a line of tiles (see dart_attend.cuh).  Plain C++ on host and device, in 32 bits: a share begins inside the line or
// at its end, so that no product here passes the line's length.
#pragma once

#ifdef __CUDACC__
#define DART_BOTH __host__ __device__ __forceinline__
#else
#define DART_BOTH inline
#endif

namespace dart {
namespace attend {

constexpr long long kLongestLine = 0x7ffffffell;

struct Shares {
    int each, more, all; // every worker's `each`, the first `more` of them one more, as far as the line of `all` goes

    // A line of `line` tiles in `items` items (0 <= line <= kLongestLine) for n workers.  least: the most that a share's least size may be.
    // Long items in small shares are slower to join than to read (narrow form, us a call, shares of 1, 2, 4 tiles at least: one sequence of
    // 300 tokens 16, 17, 18; of 6000 19.6, 18.0, 19.9; of 24000 34.5, 34.5, 27.5): a tile for each 64 of an item, up to `least`.
    static DART_BOTH Shares of(int line, long long items, int n, int least)
    {
        Shares s;
        s.all = line, s.each = (int)((unsigned)line / (unsigned)n), s.more = line - s.each * n;
        int most = 1;
        if (least > 1) {
            const int want = (int)((unsigned)line / ((unsigned)(items > 1 ? items : 1) * 64u + 1u));
            most = want < least ? want : least;
        }
        if (most < 1) most = 1;
        if (s.each < most) s.each = most, s.more = 0;
        return s;
    }
    // Where worker w < n begins (beyond `all`: it has nothing), and how much is its.
    DART_BOTH int begin(int w) const { return each * w + (w < more ? w : more); }
    DART_BOTH int size(int w) const
    {
        const int left = all - begin(w), mine = each + (w < more ? 1 : 0);
        return left < 0 ? 0 : left < mine ? left : mine;
    }
};

} // namespace attend
} // namespace dart
