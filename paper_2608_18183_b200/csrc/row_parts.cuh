// How a row is split over CTAs, and how the groups of a staged row are dealt to the warps of one.  No CUDA in here: it also compiles as
// plain C++.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define HBSJD_ANYWHERE __host__ __device__ __forceinline__
#else
#define HBSJD_ANYWHERE inline
#endif

namespace hbsjd {

constexpr int PHASES = 8;  // places behind a 16-byte boundary, at most

// A slice of n elements, the first of them P < PHASES elements behind a 16-byte boundary in shared memory, as groups of G; warp `warp` of WARPS
// has the groups [j0, j1) to itself.  It stages them, sums over them and writes their gradient without waiting for other warps, and
// then stages its part of the next row, which may lie at another P: so where a part begins depends on `dealt` alone, which is
// the same (n, or more) for all slices that take one another's place.
template <int G, int WARPS>
struct Part {
    int P, n, j0, j1;
    HBSJD_ANYWHERE Part(int P, int n, int warp) : Part(P, n, warp, n) {}
    HBSJD_ANYWHERE Part(int P, int n, int warp, int dealt) : P(P), n(n) {
        // (of the groups that `dealt` elements take at P = 0; even: 16 bytes of bf16.  The last warp has what another place adds, too.)
        const int groups = (P + n + G - 1) / G, each = ((dealt + G - 1) / G + 2 * WARPS - 1) / (2 * WARPS) * 2;
        j0 = warp * each < groups ? warp * each : groups;
        j1 = warp < WARPS - 1 && j0 + each < groups ? j0 + each : groups;
    }
    // groups [inner(), outer()) are the row's in whole
    HBSJD_ANYWHERE int inner() const { return j0 * G >= P ? j0 : (P + G - 1) / G < j1 ? (P + G - 1) / G : j1; }
    HBSJD_ANYWHERE int outer() const {
        const int whole = (P + n) / G < j1 ? (P + n) / G : j1;
        return whole > inner() ? whole : inner();
    }
    // staged elements [first(), last()) are the row's, in it from element first() - P on
    HBSJD_ANYWHERE int first() const { return j0 * G > P ? j0 * G : P; }
    HBSJD_ANYWHERE int last() const { return j1 * G < P + n ? j1 * G : P + n; }
};

// The part of tile `tile` of a row of V elements that one CTA takes in tiles of `slice`, one after another in the same place of shared
// memory, and behind the last the first of another row.  The last tile is shorter: it is dealt as the others are, else a warp would fetch into
// groups that its neighbour still reads.
template <int G, int WARPS>
HBSJD_ANYWHERE Part<G, WARPS> tile_part(int P, int V, int slice, int tile, int warp) {
    const int left = V - tile * slice;
    return Part<G, WARPS>(P, left < slice ? left : slice, warp, slice);
}

constexpr int ROW_CTAS = 8;  // CTAs of a row, at most (the portable cluster size)
constexpr int SHARED_SM = 72 * 1024;

// How a row is split: CTAs (a cluster, where more than one) and the elements that each holds.
struct RowSplit {
    int ctas, slice;
};
// 72 KB a CTA, so that three share an SM; parts of 4096 entries and more where there are SMs to spare, if `spread` (a row of 16384
// fp32 on 1, 2, 4, 8 CTAs: divergence with gradient 6.0, 6.0, 4.8, 4.3 us, from a list of 64 8.8, 7.9, 6.9, 6.7; one of 4096 is fastest on one).
inline RowSplit split_row(int64_t rows, int V, int bytes_per_element, int sms, int most_bytes, bool spread) {
    int ctas = 1;
    while (ctas < ROW_CTAS && (int64_t)V * bytes_per_element > (int64_t)most_bytes * ctas) ctas *= 2;
    while (spread && ctas < ROW_CTAS && rows * ctas * 2 <= sms && V > 4096 * ctas) ctas *= 2;
    return {ctas, ((V + ctas - 1) / ctas + 7) / 8 * 8};
}

}  // namespace hbsjd
