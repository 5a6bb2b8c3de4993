// Losses of pairs of sequences from the log-probabilities of their tokens, and each row's slope.
//
//   S_s = sum over the rows of sequence s of w (l - ref),  h = S_chosen - S_rejected,
//   sigmoid: z = beta h - margin, (1 - e) log(1 + e^-z) + e log(1 + e^z);  hinge: max(0, 1 - z);  square: (h - 1 / (2 beta))^2.
// The sums are in 64 bits: h is a difference of sums over hundreds of rows, small beside them.
#include "../../include/hbsjd.h"
#include "logit_rows.cuh"

namespace hbsjd {

namespace {

constexpr int PAIR_THREADS = 256;

__device__ __forceinline__ double sum_of_block(double v, double* parts) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (lane == 0) parts[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < PAIR_THREADS / 32; ++i) v += parts[i];
    return v;
}

// (loss, its slope in h)
__device__ __forceinline__ double2 pair_loss(const PairArgs& a, double h) {
    if (a.kind == HBSJD_PREFERENCE_SQUARE) {
        const double d = h - 0.5 / a.beta;
        return {d * d, 2.0 * d};
    }
    const double z = (double)a.beta * h - a.margin;
    if (a.kind == HBSJD_PREFERENCE_HINGE) return {z < 1.0 ? 1.0 - z : z == z ? 0.0 : z, z < 1.0 ? -(double)a.beta : z == z ? 0.0 : z};
    const double s = exp(-fabs(z)), near = log1p(s), e = a.smoothing;
    const double up = z > 0 ? 1.0 / (1.0 + s) : s / (1.0 + s), down = z > 0 ? s / (1.0 + s) : 1.0 / (1.0 + s);  // of z and -z
    return {(e < 1.0 ? (1.0 - e) * (near + (z > 0 ? 0.0 : -z)) : 0.0) + (e > 0.0 ? e * (near + (z > 0 ? z : 0.0)) : 0.0),
            a.beta * (e * up - (1.0 - e) * down)};
}

// A CTA a pair.
__global__ void __launch_bounds__(PAIR_THREADS) k_pairs(PairArgs a) {
    __shared__ double parts[PAIR_THREADS / 32];
    pdl_wait();
    pdl_trigger();
    // offsets that decrease, or leave the rows: nothing is known of any sequence
    bool wrong = false;
    for (int i = threadIdx.x; i <= 2 * a.pairs; i += PAIR_THREADS) {
        const int at = __ldg(a.offsets + i), before = i ? __ldg(a.offsets + i - 1) : 0;
        wrong |= at < before || at > a.rows;
    }
    wrong = __syncthreads_or(wrong);
    const int pair = blockIdx.x;
    const int seq[2] = {a.interleaved ? 2 * pair : pair, a.interleaved ? 2 * pair + 1 : a.pairs + pair};
    if (wrong) {
        if (threadIdx.x == 0) {
            if (a.loss) a.loss[pair] = NAN;
            if (a.sums) a.sums[seq[0]] = a.sums[seq[1]] = NAN;
        }
        if (a.slope)
            for (int64_t r = (int64_t)pair * PAIR_THREADS + threadIdx.x; r < a.rows; r += (int64_t)gridDim.x * PAIR_THREADS) a.slope[r] = NAN;
        return;
    }
    double sum[2];
    for (int k = 0; k < 2; ++k) {
        const int end = __ldg(a.offsets + seq[k] + 1);
        double v = 0.0;
        for (int r = __ldg(a.offsets + seq[k]) + threadIdx.x; r < end; r += PAIR_THREADS) {
            const float w = a.weight ? __ldg(a.weight + r) : 1.f;
            if (w != 0.f) v += (double)w * ((double)a.logp[r] - (a.ref ? (double)__ldg(a.ref + r) : 0.0));
        }
        sum[k] = sum_of_block(v, parts);
    }
    const double2 f = pair_loss(a, sum[0] - sum[1]);
    if (threadIdx.x == 0) {
        if (a.loss) a.loss[pair] = (float)f.x;
        if (a.sums) a.sums[seq[0]] = (float)sum[0], a.sums[seq[1]] = (float)sum[1];
    }
    if (a.slope) {
        const double slope = f.y * (a.pair_weight ? (double)__ldg(a.pair_weight + pair) : 1.0);
        for (int k = 0; k < 2; ++k) {
            const int end = __ldg(a.offsets + seq[k] + 1);
            for (int r = __ldg(a.offsets + seq[k]) + threadIdx.x; r < end; r += PAIR_THREADS) {
                const float w = a.weight ? __ldg(a.weight + r) : 1.f;
                a.slope[r] = w == 0.f ? 0.f : (float)(k ? -slope * w : slope * w);
            }
        }
        // rows of no sequence
        const int from = __ldg(a.offsets), to = __ldg(a.offsets + 2 * a.pairs);
        for (int r = pair * PAIR_THREADS + threadIdx.x; r < a.rows; r += gridDim.x * PAIR_THREADS)
            if (r < from || r >= to) a.slope[r] = 0.f;
    }
}

}  // namespace

cudaError_t launch_pairs(const PairArgs& a, Stream& s) {
    return launch_k(k_pairs, dim3((unsigned)a.pairs), dim3(PAIR_THREADS), 0, s, a);
}

}  // namespace hbsjd
