// Losses of pairs of sequences from the log-probabilities of their tokens, and each row's slope.
//
//   S_s = sum over the rows of sequence s of w (l - ref),  h = S_chosen - S_rejected,
//   sigmoid: z = beta h - margin, (1 - e) log(1 + e^-z) + e log(1 + e^z);  hinge: max(0, 1 - z);  square: (h - 1 / (2 beta))^2.
// The sums are in 64 bits, and l comes with what its rounding left: h is a difference of sums over hundreds of rows, small beside them.
//
// A row's gradient needs its whole pair's sums, so the call is three kernels: k_token sums over the rows and keeps 16 bytes of each, k_pairs (here,
// 5 us of latencies) makes the slopes, k_spread writes the gradient from what was kept, reading the logits a second time, the last rows
// first.  That second reading is what bounds it: 16 pairs of 256 positions of 16384 fp32 246 us, where two readings and a writing take 229 at a
// copy's rate (one reading 156).  L2 does not save it: a pair is 33 MB there, and gradients some rows behind the sums, in one kernel, still read 0.92
// of all logits twice (350 us); batches of fewer pairs a launch pay 5 us of ramp each.
#include "../../include/hbsjd.h"
#include "logit_rows.cuh"

namespace hbsjd {

namespace {

constexpr int PAIR_THREADS = 256;

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

// A CTA a pair (or several in turn: each looks at all offsets), half of it a sequence.  The offsets are the caller's and nothing of the kernel in front:
// behind one that triggers late they are read before the wait (see pdl_wait).
__global__ void __launch_bounds__(PAIR_THREADS) k_pairs(PairArgs a) {
    constexpr int HALF = PAIR_THREADS / 2;
    __shared__ double parts[PAIR_THREADS / 32];
    const int tid = threadIdx.x, side = tid / HALF;
    // offsets that decrease, or leave the rows: nothing is known of any sequence
    bool wrong = false;
    if (!a.early) pdl_wait();
    for (int i = tid; i <= 2 * a.pairs; i += PAIR_THREADS) {
        const int at = __ldcg(a.offsets + i), before = i ? __ldcg(a.offsets + i - 1) : 0;
        wrong |= at < before || at > a.rows;
    }
    const int from = __ldcg(a.offsets), to = __ldcg(a.offsets + 2 * a.pairs);
    const auto sequence = [&](int pair, bool rejected) { return a.interleaved ? 2 * pair + rejected : rejected ? a.pairs + pair : pair; };
    // rows of the first pair's sequence (read here, else they are another read from L2 behind the wait)
    int2 rows = {__ldcg(a.offsets + sequence(blockIdx.x, side)), __ldcg(a.offsets + sequence(blockIdx.x, side) + 1)};
    pdl_wait();
    pdl_trigger();
    // a row's weight; 0: it is left out
    const auto weight = [&](int r) {
        const int t = __ldg(a.tokens + r);
        return t < 0 || t >= a.V ? 0.f : a.weight ? __ldg(a.weight + r) : 1.f;
    };
    wrong = __syncthreads_or(wrong);
    for (int pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
        const int chosen = sequence(pair, false), other = sequence(pair, true);
        if (wrong) {
            if (tid == 0 && a.loss) a.loss[pair] = NAN;
            if (tid == 0 && a.sums) a.sums[chosen] = a.sums[other] = NAN;
            continue;
        }
        if (pair != blockIdx.x) rows = {__ldcg(a.offsets + (side ? other : chosen)), __ldcg(a.offsets + (side ? other : chosen) + 1)};
        const int begin = rows.x + tid % HALF, end = rows.y;
        double v = 0.0;
#pragma unroll 4
        for (int r = begin; r < end; r += HALF) {
            const float w = weight(r), l = a.logp[r], low = a.stats[r].w, ref = a.ref ? __ldg(a.ref + r) : 0.f;
            if (w != 0.f) v += (double)w * (((double)l - (double)ref) + (double)low);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (tid % 32 == 0) parts[tid / 32] = v;
        __syncthreads();
        double sum[2] = {0.0, 0.0};
#pragma unroll
        for (int i = 0; i < PAIR_THREADS / 32; ++i) sum[i / (HALF / 32)] += parts[i];
        const double2 f = pair_loss(a, sum[0] - sum[1]);
        if (tid == 0) {
            if (a.loss) a.loss[pair] = (float)f.x;
            if (a.sums) a.sums[chosen] = (float)sum[0], a.sums[other] = (float)sum[1];
        }
        if (a.slope) {
            const double slope = (side ? -f.y : f.y) * (a.pair_weight ? (double)__ldg(a.pair_weight + pair) : 1.0);
#pragma unroll 4
            for (int r = begin; r < end; r += HALF) {
                const float w = weight(r);
                a.slope[r] = w == 0.f ? 0.f : (float)(slope * w);
            }
        }
        __syncthreads();  // the sums have been read
    }
    // rows of no sequence
    if (a.slope && (wrong || from > 0 || to < a.rows))
        for (int64_t r = (int64_t)blockIdx.x * PAIR_THREADS + tid; r < a.rows; r += (int64_t)gridDim.x * PAIR_THREADS)
            if (wrong || r < from || r >= to) a.slope[r] = wrong ? NAN : 0.f;
}

}  // namespace

cudaError_t launch_pairs(const PairArgs& args, Stream& s) {
    PairArgs a = args;
    a.early = s.late;
    return launch_k(k_pairs, dim3((unsigned)std::min(a.pairs, 4 * device_sm_count())), dim3(PAIR_THREADS), 0, s, a);
}

}  // namespace hbsjd
