// Launcher of the kernels that clip many arrays by their common norm.
#pragma once
#include "logit_rows.cuh"

namespace hbsjd {

constexpr int CLIP_PARTS = 1024;              // CTAs of a launch of the norm's kernel, at most: a part each
constexpr int CLIP_FEW = 128, CLIP_MANY = 1024;  // arrays of a launch: 4 KB of parameters, or 30 KB

struct ClipArray {
    const void* in;
    void* out;
    int64_t n;
    int bytes;  // an element's
};
struct ClipArgs {
    double* parts;      // [CLIP_PARTS clip_launches(count)]
    float* norm;
    float limit;
    int max_norm, scale, copy;  // the largest magnitude in place of the root of the squares' sum; to scale at all; out is not in
};
int clip_launches(int count);
int64_t clip_chunks(const ClipArray* arrays, int count);  // no fewer than a launch has
// arrays of at least one element
cudaError_t launch_clip(const ClipArray* arrays, int count, const ClipArgs& a, Stream& s);

}  // namespace hbsjd
