// Index arithmetic of the paged cache: what the kernels derive from numbers that
// only the device holds (starts, lengths, page numbers).  Whatever these say,
// the results stay within the arrays.
#pragma once

#include <math.h>

#ifdef __CUDACC__
#define WDC_INDEX __host__ __device__ __forceinline__
#else
#define WDC_INDEX inline
#endif

namespace wdc {

// A sequence's chunk: rows row0 .. row0 + n - 1 of T, the last n of its len tokens.
struct PagedSeq {
    int row0, n, len;
};
WDC_INDEX int index_clamp(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }
WDC_INDEX PagedSeq paged_seq(int start, int end, int length, int T, int room) {
    PagedSeq s;
    s.row0 = index_clamp(start, 0, T);
    s.n = index_clamp(end, s.row0, T) - s.row0;
    s.len = index_clamp(length, 0, room);
    return s;
}
// Whether the numbers are as a caller should give them, `most` new tokens at most; if
// not, paged_seq takes the nearest that are.
WDC_INDEX bool paged_given(int start, int end, int length, int T, int room, int most) {
    return start >= 0 && end >= start && end <= T && length >= 0 && length <= room && end - start <= length &&
           end - start <= most;
}
// Place of the chunk's token i in its sequence; negative where the sequence is
// shorter than its chunk.
WDC_INDEX int paged_place(const PagedSeq& s, int i) { return s.len - s.n + i; }
// Tokens that the chunk's token i sees: all (frame 0), or those of its frame and
// of the frames before it.  Does not fall with i.
WDC_INDEX int paged_limit(const PagedSeq& s, int frame, int i) {
    if (frame == 0) return s.len;
    const int p = paged_place(s, i);
    if (p < 0) return 0;
    const long long end = ((long long)(p / frame) + 1) * frame;
    return end < s.len ? (int)end : s.len;
}
// A page number that the pool has, or -1.
WDC_INDEX int paged_page(int p, int pages) { return p >= 0 && p < pages ? p : -1; }
// The middle of whole numbers lo <= hi <= 2^24, rounded down.  (Their sum may not be
// a float; with a middle rounded up to hi a bisection would not end.)
WDC_INDEX float plan_middle(float lo, float hi) { return lo + floorf(0.5f * (hi - lo)); }

}  // namespace wdc
