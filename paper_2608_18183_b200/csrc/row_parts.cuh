// How the groups of a staged row are dealt to the warps of a CTA.  No CUDA in here: it also compiles as plain C++.
#pragma once

#ifdef __CUDACC__
#define HBSJD_ANYWHERE __host__ __device__ __forceinline__
#else
#define HBSJD_ANYWHERE inline
#endif

namespace hbsjd {

constexpr int PHASES = 8;  // places behind a 16-byte boundary, at most

// A slice of n elements, the first of them P < PHASES elements behind a 16-byte boundary in shared memory, as groups of G; warp `warp` of WARPS
// has the groups [j0, j1) to itself.  It stages them, sums over them and writes their gradient without waiting for other warps, and
// then stages its part of the next row, which may lie at another P: so where a part begins depends on n alone.
template <int G, int WARPS>
struct Part {
    int P, n, j0, j1;
    HBSJD_ANYWHERE Part(int P, int n, int warp) : P(P), n(n) {
        // (of the groups that n elements take at P = 0; even: 16 bytes of bf16.  The last warp has what another place adds, too.)
        const int groups = (P + n + G - 1) / G, each = ((n + G - 1) / G + 2 * WARPS - 1) / (2 * WARPS) * 2;
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

}  // namespace hbsjd
