// Log-probabilities of sampled tokens, the clipped policy loss and what both give back to the logits, in one pass over memory (see
// token_rows.cuh for the formulas).
//
// Two sums over a row (exponentials, and weighted by their exponents where the entropy is wanted) give the loss, and a second look at the row
// the gradient.  In between the row stays in shared memory: it is read from HBM once and the gradient written once, which bounds fp32; in bf16
// the two exponentials an entry and about 18 instructions (a third of them what a warp does once a row) share the time with it.  Rows are
// dealt to resident CTAs; a warp has a part of each to itself, as in the divergences, meets the others for the sums alone, and fetches its part of the
// next row group by group as it reads this one for the last time, wherever that row lies behind 16 bytes.  Long rows, and few, are split over a
// cluster.  Measured, the kernel alone: log-probabilities and entropies of 8192 rows of 16384 fp32 88 us (0.94 of a copy's rate); policy
// loss with gradient of 16384 such rows, an eighth left out, 327 us (0.95); with entropy, 8192 rows in bf16 110 us (0.75); backward of 3001 rows of 24001 bf16 70 us
// (0.63, as at whole turns and with aligned rows: four rows fit an SM, whose latencies leave issue slots and exponentials half idle).  Warps whose
// part of a row begins with a stretch of -inf go entry by entry: a third of the row masked takes two to four times as long.
#include <type_traits>

#include "token_rows.cuh"

namespace hbsjd {

namespace {

template <bool ENT, int WARPS>
__device__ __forceinline__ void post_sums(const TokenSums& x, TokenSums* slots, int ctas, int rank) {
    const int lane = threadIdx.x & 31;
    if (lane < ctas) {
        float* f = reinterpret_cast<float*>(slots + rank * WARPS + (threadIdx.x >> 5));
        post_float(f, ctas, lane, x.m);
        post_float(f + 1, ctas, lane, x.z);
        if (ENT) post_float(f + 2, ctas, lane, x.a);
    }
}
// Sums of two sets of entries.
template <bool ENT>
__device__ __forceinline__ TokenSums merged(const TokenSums& x, const TokenSums& y, float c, bool summed) {
    TokenSums r = {fmaxf(x.m, y.m), 0.f, 0.f};
    const auto add = [&](const TokenSums& s) {
        const float f = summed ? rescale_without_lean(s.m, r.m, c) : rescale(s.m, r.m, c);
        r.z += s.z * f;
        if (ENT && f != 0.f) r.a += f * fmaf(s.z, s.m == r.m ? 0.f : (s.m - r.m) * c, s.a);
    };
    add(x);
    add(y);
    return r;
}
// The row's sums from its warps', the same bits in every warp.
template <bool ENT>
__device__ __forceinline__ TokenSums collect_sums(const TokenSums* slots, int count, float c, bool summed) {
    const int lane = threadIdx.x & 31;
    TokenSums r = TokenSums::none();
    for (int j = lane; j < count; j += 32) r.m = fmaxf(r.m, slots[j].m);
    r.m = max_of_warp(r.m);
    for (int j = lane; j < count; j += 32) {
        const TokenSums s = slots[j];
        const float f = summed ? rescale_without_lean(s.m, r.m, c) : rescale(s.m, r.m, c);
        r.z += s.z * f;
        if (ENT && f != 0.f) r.a += f * fmaf(s.z, s.m == r.m ? 0.f : (s.m - r.m) * c, s.a);
    }
    r.z = sum_of_warp(r.z);
    if (ENT) r.a = sum_of_warp(r.a);
    return r;
}

// (e^d - 1 - d, e^d - 1), the first within 8 half steps of itself: by series where |d| < 1/2, whose next terms are below 5.1e-8 of it at either sign,
// else from expm1f, whose step is at most 4.1e-7 of what is left of it.
__device__ __forceinline__ float2 exp_excess(float d) {
    if (fabsf(d) < 0.5f) {
        const float d2 = d * d, even = fmaf(d2, fmaf(d2, fmaf(d2, 1.f / 40320, 1.f / 720), 1.f / 24), 0.5f);
        const float excess = d2 * fmaf(d, fmaf(d2, fmaf(d2, 1.f / 5040, 1.f / 120), 1.f / 6), even);
        return {excess, excess + d};
    }
    const float slope = expm1f(d);
    return {d > 40.f ? slope : slope - d, slope};
}

// What a row has besides its logits: its weight, advantage, old and reference log-probability; or the slopes in log q and in the entropy.
struct RowTerms {
    float a, b, c, d;
};
__device__ __forceinline__ RowTerms terms_of(const TokenArgs& a, int row) {
    const auto get = [&](const float* p, float other) { return p ? __ldg(p + row) : other; };
    if (a.d_logp) return {__ldg(a.d_logp + row), get(a.d_entropy, 0.f), 0.f, 0.f};
    return {get(a.weight, 1.f), get(a.advantage, 0.f), get(a.old_logp, 0.f), get(a.ref, 0.f)};
}

// The loss of a token whose log-probability is l, but for the entropy's part, and its slope in l.
__device__ __forceinline__ float2 policy(const TokenArgs& a, const RowTerms& row, float l) {
    const float A = row.b, r = !a.old_logp || l == row.c ? (l == l ? 1.f : l) : ex2((l - row.c) * LOG2E);
    // (comparisons that let NaN pass; no advantage times an infinite ratio is none)
    const float low = 1.f - a.low, high = 1.f + a.high, clipped = r < low ? low : r > high ? high : r;
    const float kept = A == 0.f && r == INFINITY ? 0.f : r * A, other = clipped * A;
    float gain = other < kept ? other : kept, slope = other < kept ? 0.f : -kept;
    if (a.dual > 0.f && A < 0.f && gain < a.dual * A) gain = a.dual * A, slope = 0.f;
    float loss = -gain;
    if (a.kl != 0.f && a.ref) {
        const float2 e = exp_excess(l == row.d ? 0.f : row.d - l);
        loss = fmaf(a.kl, e.x, loss);
        slope = fmaf(-a.kl, e.y, slope);
    }
    return {loss, slope};
}

// TILED (no gradient): a CTA takes a.tiles slices of a row in turn.
template <typename T, bool ENT, bool GRAD, bool TILED, int THREADS, int PER_SM>
__global__ void __launch_bounds__(THREADS, PER_SM) k_token(TokenArgs a) {
    constexpr int G = 16 / sizeof(T), WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_wait();
    pdl_trigger();
    const int wid = threadIdx.x >> 5;
    const int rank = blockIdx.x % a.ctas, v0 = rank * a.slice, n = max(0, min(a.slice, a.V - v0));
    const int step = gridDim.x / a.ctas, places = WARPS * a.ctas;
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    T* ss = (T*)smem;
    TokenSums* slots = (TokenSums*)(ss + a.slice + 16);  // [2][places], by turns: a CTA may be a row ahead of others
    if (a.ctas > 1) cluster_barrier();                    // every CTA of the rows runs
    // a row's token, -1: the row is left out
    const auto token_of = [&](int row) {
        if (row >= a.rows) return -1;
        int32_t t;
        if (a.at) {
            const int2 at = __ldg(a.at + row);
            if (at.x < 0 || at.y >= a.T || at.y < __ldg(a.prefix_len + at.x)) return -1;
            t = __ldg(a.tokens + (int64_t)at.x * a.T + at.y);
        } else {
            t = __ldg(a.tokens + row);
            if (a.weight && __ldg(a.weight + row) == 0.f) return -1;
            if (a.d_logp && __ldg(a.d_logp + row) == 0.f && (!a.d_entropy || __ldg(a.d_entropy + row) == 0.f)) return -1;
        }
        return t >= 0 && t < a.V ? (int)t : -1;
    };
    const auto row_at = [&](int row) { return (const T*)a.x + (int64_t)row * a.ld; };
    const auto logit_of = [&](int row, int t) { return t < 0 ? 0.f : to_f<T>(row_at(row)[t]); };
    const auto part_of = [&](const T* x) { return Part<G, WARPS>(phase_of(x), n, wid); };
    const int64_t stride = (int64_t)step * a.ld;
    const bool summed = !ENT && !GRAD && a.summed;  // (the preference loss asks for no entropies)
    int row = blockIdx.x / a.ctas, parity = 0;
    int t = token_of(row), t1 = token_of(row + step);
    float xt = logit_of(row, t);
    const T* x0 = row_at(row) + v0;
    Part<G, WARPS> p = part_of(x0);
    if (t >= 0) stage_part(ss, x0, p);
    for (; row < a.rows; row += step) {
        // (so that no fetch waits for a token, and no row for its logit; no gradient that takes a row's place has been written yet)
        const int t2 = token_of(row + 2 * step);
        const float xt1 = logit_of(row + step, t1);
        const RowTerms terms = terms_of(a, row);
        T* g = GRAD ? (T*)a.grad + (int64_t)row * a.ld_g + v0 : nullptr;
        const T* x1 = x0 + stride;
        const Part<G, WARPS> p1 = part_of(x1);
        Next<T, G, WARPS> next = {ss, x1, p1, t1 >= 0};
        const int lo = p.first() - p.P, hi = p.last() - p.P;  // the warp's entries of the slice
        const bool first = rank == 0 && threadIdx.x == 0;
        if (t < 0) {  // (all CTAs of the row)
            if constexpr (GRAD) put_zeros(g, lo, hi);
            if (first && !a.at) {
                if (a.loss) a.loss[row] = 0.f;
                if (a.logp) a.logp[row] = 0.f;
                if (a.entropy) a.entropy[row] = 0.f;
            }
        } else {
            const int mine = t - v0 >= lo && t - v0 < hi ? t - v0 : -1;  // the token, if it is one of the warp's
            cp_async_wait_all();
            __syncwarp();
            // (one order of the sums, whatever is asked for)
            TokenSums v;
            if constexpr (GRAD) {
                v = part_sums<ENT>(ss, p, x0, mine, c, [&](auto&& f) { each_of(p, f); });
            } else if constexpr (!TILED) {
                v = part_sums<ENT>(ss, p, x0, mine, c, [&](auto&& f) { each_then(p, next, f); });
            } else {  // a long row tile by tile: nobody looks at it again
                v = TokenSums::none();
                for (int tile = 0; tile < a.tiles; ++tile) {
                    const bool last = tile + 1 == a.tiles;
                    const int at = tile * a.slice;
                    const T *x = row_at(row) + at, *behind = last ? x1 : x + a.slice;
                    const auto q = tile_part<G, WARPS>(phase_of(x), a.V, a.slice, tile, wid);
                    const auto q1 = tile_part<G, WARPS>(phase_of(behind), a.V, a.slice, last ? 0 : tile + 1, wid);
                    Next<T, G, WARPS> then = {ss, behind, q1, !last || next.more};
                    if (tile) {
                        cp_async_wait_all();
                        __syncwarp();
                    }
                    const int place = t - at, in = place >= q.first() - q.P && place < q.last() - q.P ? place : -1;
                    v = merged<ENT>(v, part_sums<ENT>(ss, q, x, in, c, [&](auto&& f) { each_then(q, then, f); }), c, summed);
                }
                next.more = false;
            }
            const bool alone = WARPS == 1 && a.ctas == 1;  // the warp has the whole row
            if (!alone) {
                post_sums<ENT, WARPS>(v, slots + parity * places, a.ctas, rank);
                posted(a.ctas);
                parity ^= 1;
            }
            TokenCoefs k;
            if (GRAD || wid == 0) {  // (each warp for itself: one for all, and a barrier, cost 16384 rows of 16384 365 us in place of 351)
                if (!alone) v = collect_sums<ENT>(slots + (parity ^ 1) * places, places, c, summed);
                const TokenRow r(v, xt, inv_tau, summed);
                float H = 0.f;
                if (ENT && !r.empty) H = (v.z == 0.f || r.qo == 0.f ? 0.f : r.qo * (r.Lk - LN2 * __fdividef(v.a, v.z))) - (r.qt == 0.f ? 0.f : r.qt * r.l);
                float2 f = {0.f, 0.f};
                if (a.advantage) f = policy(a, terms, r.l);
                if (first) {
                    int64_t place = row;
                    if (a.at) {
                        const int2 at = __ldg(a.at + row);
                        place = (int64_t)at.x * a.T + at.y;
                    }
                    if (a.loss) a.loss[row] = r.empty ? 0.f : a.bonus != 0.f ? fmaf(-a.bonus, H, f.x) : f.x;
                    if (a.logp) a.logp[place] = r.logp();
                    if (ENT && a.entropy) a.entropy[place] = H;
                    if (!GRAD && a.stats) a.stats[row] = make_float4(v.m, v.z, r.empty ? 0.f : r.qo, r.empty ? 0.f : r.low);
                }
                if constexpr (GRAD)
                    k.set<ENT>(r, v, H, a.d_logp ? terms.a : f.y, a.d_logp ? -terms.b : a.bonus, a.d_logp ? inv_tau : terms.a * inv_tau, c);
            }
            if constexpr (GRAD) part_gradient<ENT>(ss, p, g, n, mine, k, c, next, [&](auto&& f) { each_then(p, next, f); });
        }
        __syncwarp();  // the warp's part is done
        if (next.more) stage_part(ss, x1, p1);
        x0 = x1, p = p1;
        t = t1, t1 = t2, xt = xt1;
    }
}

// Whole rows are staged as in k_token, but nobody waits for anybody here.
template <typename T, int THREADS, int PER_SM>
__global__ void __launch_bounds__(THREADS, PER_SM) k_spread(SpreadArgs a) {
    constexpr int G = 16 / sizeof(T), WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_wait();
    pdl_trigger();
    const int wid = threadIdx.x >> 5, step = gridDim.x;
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    T* ss = (T*)smem;
    struct Row {
        float slope;
        float4 stat;
        int token;  // -1: the row is left out
    };
    const auto row_of = [&](int row) {
        Row r = {0.f, {}, -1};
        if (row < 0) return r;
        r.slope = __ldg(a.slope + row), r.stat = __ldg(a.stats + row), r.token = __ldg(a.tokens + row);
        if (r.slope == 0.f || r.token >= a.V) r.token = -1;
        return r;
    };
    const auto part_of = [&](const T* x) { return Part<G, WARPS>(phase_of(x), a.V, wid); };
    int row = a.rows - 1 - (int)blockIdx.x;
    Row r = row_of(row), r1 = row_of(row - step);
    const T* x0 = (const T*)a.x + (int64_t)row * a.ld;
    Part<G, WARPS> p = part_of(x0);
    if (r.token >= 0) stage_part(ss, x0, p);
    for (; row >= 0; row -= step) {
        const Row r2 = row_of(row - 2 * step);  // (so that no fetch waits for a slope)
        const T* x1 = x0 - (int64_t)step * a.ld;
        const Part<G, WARPS> p1 = part_of(x1);
        T* g = (T*)a.grad + (int64_t)row * a.ld_g;
        Next<T, G, WARPS> next = {ss, x1, p1, r1.token >= 0};
        const int lo = p.first() - p.P, hi = p.last() - p.P;  // the warp's entries
        if (r.token < 0) {
            put_zeros(g, lo, hi);
        } else {
            TokenSums v = TokenSums::none();
            v.m = r.stat.x, v.z = r.stat.y;
            TokenCoefs k;
            k.set<false>(TokenRow(r.stat.y, r.stat.z), v, 0.f, r.slope, 0.f, inv_tau, c);
            cp_async_wait_all();
            __syncwarp();
            // (two loops here: 16 pairs of 256 positions of 16384 fp32 246 us in place of 261)
            part_gradient<false>(ss, p, g, a.V, r.token >= lo && r.token < hi ? r.token : -1, k, c, next, [&](auto&& f) {
                if (next.more)
                    each_then(p, next, f);
                else
                    each_of(p, f);
            });
        }
        __syncwarp();
        if (next.more) stage_part(ss, x1, p1);
        r = r1, r1 = r2, x0 = x1, p = p1;
    }
}

// The same by parts of rows of up to 4 KB, a warp each, from HBM to HBM.
constexpr int SPREAD_THREADS = 256, SPREAD_WARPS = SPREAD_THREADS / 32, SPREAD_BYTES = 4096;
// SHIFTED: the gradient may lie at another place behind 16 bytes than the logits.
template <typename T, bool SHIFTED>
__global__ void __launch_bounds__(SPREAD_THREADS, 4) k_spread_parts(SpreadArgs a) {
    constexpr int G = 16 / sizeof(T), AHEAD = SHIFTED ? 2 : 4;  // groups a lane has on their way
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    const unsigned step = gridDim.x * SPREAD_WARPS, items = (unsigned)a.rows * a.parts;
    unsigned u = blockIdx.x * SPREAD_WARPS + (threadIdx.x >> 5);
    const auto row_of = [&](unsigned u) { return a.rows - 1 - (int)(u / a.parts); };
    float slope = u < items ? __ldg(a.slope + row_of(u)) : 0.f;
    float4 stat = u < items ? __ldg(a.stats + row_of(u)) : make_float4(0.f, 0.f, 0.f, 0.f);
    int token = u < items ? __ldg(a.tokens + row_of(u)) : -1;
    for (; u < items; u += step) {
        const int row = row_of(u), v0 = (int)(u % a.parts) * a.part, n = min(a.part, a.V - v0);
        const T* x = (const T*)a.x + (int64_t)row * a.ld + v0;
        T* g = (T*)a.grad + (int64_t)row * a.ld_g + v0;
        const unsigned u1 = u + step;
        float slope1 = 0.f;
        float4 stat1 = {};
        int token1 = -1;
        if (u1 < items) slope1 = __ldg(a.slope + row_of(u1)), stat1 = __ldg(a.stats + row_of(u1)), token1 = __ldg(a.tokens + row_of(u1));
        if (slope == 0.f || token < 0 || token >= a.V) {
            put_zeros(g, 0, n);
        } else {
            TokenSums v = TokenSums::none();
            v.m = stat.x, v.z = stat.y;
            TokenCoefs k;
            k.set<false>(TokenRow(stat.y, stat.z), v, 0.f, slope, 0.f, inv_tau, c);
            const f32x2 o = both(-k.mc), c2 = both(c), K0 = both(k.k0);
            const auto of = [&](f32x2 e) { return mul2(ex2(fma2(e, c2, o)), K0); };
            const int P = phase_of(x), first = P ? G - P : 0, groups = max(0, n - first) / G;  // whole groups of 16 bytes from x + first
            if (k.way == 2) {
                put_zeros(g, 0, n);
            } else if (k.way == 1) {
                for (int e = lane; e < n; e += 32) {
                    const float q = ex2(held((to_f<T>(x[e]) - k.m) * c)) * k.K;
                    g[e] = from_f<T>(q == 0.f && k.is_number(k.A) ? 0.f : q * -k.A * k.scale);
                }
            } else if (SHIFTED && P != phase_of(g)) {
                Shifted<T, G> to(g, 0, n, P);
                for (int j0 = to.first; j0 <= to.last + 1; j0 += 32 * AHEAD) {
                    uint4 w[AHEAD];
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) {
                        const int e = (j0 + i * 32 + lane) * G - P;
                        if (e >= 0 && e + G <= n)
                            w[i] = __ldcs(reinterpret_cast<const uint4*>(x + e));
                        else
#pragma unroll
                            for (int h = 0; h < G; ++h) reinterpret_cast<T*>(&w[i])[h] = e + h >= 0 && e + h < n ? x[e + h] : from_f<T>(0.f);
                    }
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) {
                        float y[G];
                        uint32_t own[4];
                        read<false>(reinterpret_cast<const T*>(&w[i]), y);
#pragma unroll
                        for (int h = 0; h < G; h += 2) split(of(both(y[h], y[h + 1])), y[h], y[h + 1]);
                        packed(y, own);
                        to.put(j0 + i * 32 + lane, own);
                    }
                }
            } else {
                const T* xs = x + first;
                T* gs = g + first;
                for (int j0 = 0; j0 < groups; j0 += 32 * AHEAD) {
                    uint4 w[AHEAD];
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) {
                        const int j = j0 + i * 32 + lane;
                        if (j < groups) w[i] = __ldcs(reinterpret_cast<const uint4*>(xs) + j);
                    }
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) {
                        const int j = j0 + i * 32 + lane;
                        float y[G];
                        read<false>(reinterpret_cast<const T*>(&w[i]), y);
#pragma unroll
                        for (int e = 0; e < G; e += 2) split(of(both(y[e], y[e + 1])), y[e], y[e + 1]);
                        if (j < groups) put<G>(gs + j * G, y);
                    }
                }
                // what is left in front and behind, less than 16 bytes each
                const int tail = first + groups * G;
                const int e = lane < 16 ? lane : tail + lane - 16;
                if (lane < 16 ? lane < min(first, n) : e < n) {
                    float lo, hi;
                    split(of(both(to_f<T>(x[e]))), lo, hi);
                    g[e] = from_f<T>(lo);
                }
            }
            __syncwarp();  // the token's place was written above
            if (token >= v0 && token - v0 < n && lane == 0) g[token - v0] = from_f<T>(k.token);
        }
        slope = slope1, stat = stat1, token = token1;
    }
}

template <typename T, bool ENT, bool GRAD, bool TILED>
cudaError_t run_token(const TokenArgs& a, Stream& s) {
    const auto bytes = [&](int threads) { return (a.slice + 16) * sizeof(T) + 2 * threads / 32 * a.ctas * sizeof(TokenSums); };
    const auto fit = [&](int threads) { return (int)(227 * 1024 / (bytes(threads) + 1024 + 128)); };  // (1 KB is the system's)
    const auto run = [&](auto threads, auto lanes) {
        constexpr int THREADS = decltype(threads)::value, PER_SM = std::min(32, decltype(lanes)::value / THREADS);
        const size_t smem = bytes(THREADS);
        cudaError_t e = allow_row_smem<k_token<T, ENT, GRAD, TILED, THREADS, PER_SM>>();
        if (e != cudaSuccess) return e;
        int clusters = 0;
        e = resident_clusters<k_token<T, ENT, GRAD, TILED, THREADS, PER_SM>>(a.ctas, THREADS, std::max(1, std::min(PER_SM, fit(THREADS))), smem, a.rows, &clusters);
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_token<T, ENT, GRAD, TILED, THREADS, PER_SM>, dim3((unsigned)clusters * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    };
    // Threads of a CTA: what a warp does once a row is a good part of its work, so that fewer warps are faster as long as an SM has 24 of
    // them, which is what 80 registers leave room for, beside the rows that its shared memory holds (8192 rows of 16384 fp32 on 512, 256 and
    // 128 threads: 121, 90 and 94 us; with gradients in bf16 134, 109 and 126).
    constexpr std::integral_constant<int, 768> full;
    if constexpr (TILED) return fit(128) <= 3 ? run(std::integral_constant<int, 256>(), full) : run(std::integral_constant<int, 128>(), full);
    if ((int64_t)a.rows * a.ctas > device_sm_count()) {
        const int f = fit(128);
        if constexpr (GRAD && sizeof(T) == 4) {
            // Writing fp32 beside, HBM is busy with 128 KB of rows an SM: 16 warps with 128 registers (16384 rows of 16384: 342 us in place of
            // 381, of 8192 164 in place of 181).  Not for clusters, whose barriers want more rows to cover them (8192 rows of 32768 389 in
            // place of 363), nor for short rows (60000 of 1000: 124 in place of 97).
            constexpr std::integral_constant<int, 512> wide;
            if (a.ctas == 1 && f <= 3) return run(std::integral_constant<int, 256>(), wide);
            if (a.ctas == 1 && f <= 6) return run(std::integral_constant<int, 128>(), wide);
            if (a.ctas == 1 && f <= 14) return run(std::integral_constant<int, 64>(), wide);
        }
        if (f <= 3) return run(std::integral_constant<int, 256>(), full);
        if (f <= 6) return run(std::integral_constant<int, 128>(), full);
        if (f <= 14) return run(std::integral_constant<int, 64>(), full);
        return run(std::integral_constant<int, 32>(), full);
    }
    const int per = 4 * 16 / (int)sizeof(T);  // entries a thread
    if (a.slice <= 32 * per) return run(std::integral_constant<int, 32>(), full);
    if (a.slice <= 64 * per) return run(std::integral_constant<int, 64>(), full);
    if (a.slice <= 128 * per) return run(std::integral_constant<int, 128>(), full);
    if (a.slice <= 256 * per) return run(std::integral_constant<int, 256>(), full);
    return run(std::integral_constant<int, 512>(), std::integral_constant<int, 1024>());
}

template <typename T>
cudaError_t run_token(const TokenArgs& a, bool entropy, Stream& s) {
    if (a.grad) return entropy ? run_token<T, true, true, false>(a, s) : run_token<T, false, true, false>(a, s);
    if (a.tiles > 1) return entropy ? run_token<T, true, false, true>(a, s) : run_token<T, false, false, true>(a, s);
    return entropy ? run_token<T, true, false, false>(a, s) : run_token<T, false, false, false>(a, s);
}

template <typename T>
cudaError_t run_spread(const SpreadArgs& args, Stream& s) {
    SpreadArgs a = args;
    const int sms = device_sm_count();
    const bool shifted = ((uintptr_t)a.x - (uintptr_t)a.grad) % 16 || (a.ld - a.ld_g) * (int64_t)sizeof(T) % 16;
    // Rows of 64 KB on 256 threads, two an SM, or smaller ones alike; fp32 is staged whole for the same order of reads and writes in HBM as
    // in k_token (16 pairs of 256 positions of 16384 266 us, of 16385 300; by parts 269 and 333).  In bf16 parts are as fast (64 pairs of 64 of
    // 16384 148 and 153 us, 20 of 256 of 24001 306 and 277), unless the gradient lies otherwise (one of 4096, a stride of 16385: 172
    // us, by parts 228).
    const size_t smem = (a.V + 24) / 8 * 8 * sizeof(T);
    const int fit = (int)(227 * 1024 / (smem + 1024 + 128));  // (1 KB is the system's)
    const auto run = [&](auto threads) {
        constexpr int THREADS = decltype(threads)::value, PER_SM = 512 / THREADS;
        const cudaError_t e = allow_row_smem<k_spread<T, THREADS, PER_SM>>();
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_spread<T, THREADS, PER_SM>, dim3((unsigned)std::min(a.rows, sms * std::min(PER_SM, fit))), dim3(THREADS), smem, s, 1, a);
    };
    if (a.rows > sms && smem <= SHARED_SM && (sizeof(T) == 4 || shifted)) {
        if (fit <= 3) return run(std::integral_constant<int, 256>());
        if (fit <= 6) return run(std::integral_constant<int, 128>());
        if (fit <= 14) return run(std::integral_constant<int, 64>());
    }
    const int most = SPREAD_BYTES / (int)sizeof(T);
    a.parts = (a.V + most - 1) / most;
    a.part = ((a.V + a.parts - 1) / a.parts + 7) / 8 * 8;
    const int64_t items = (int64_t)a.rows * a.parts;
    const dim3 grid((unsigned)std::min<int64_t>((int64_t)sms * 4, (items + SPREAD_WARPS - 1) / SPREAD_WARPS));
    if (shifted) return launch_k(k_spread_parts<T, true>, grid, dim3(SPREAD_THREADS), 0, s, a);
    return launch_k(k_spread_parts<T, false>, grid, dim3(SPREAD_THREADS), 0, s, a);
}

}  // namespace

cudaError_t launch_token(const TokenArgs& args, int rows, int dtype, Stream& s) {
    TokenArgs a = args;
    const RowSplit sp = split_row(rows, a.V, dtype ? 2 : 4, device_sm_count(), SHARED_SM, true);
    a.rows = rows, a.ctas = sp.ctas, a.slice = sp.slice, a.tiles = 1;
    // Where nothing is looked at again, long rows are one CTA's, if there are enough of them: no barriers of clusters (8192 rows of 32768 fp32 175 ->
    // 158 us, 4096 of 65537 217 -> 181).  Not for the
    // policy's loss, which is to have the same bits with and without its gradient.
    if (!a.grad && !a.advantage && rows > device_sm_count()) a.tiles = a.ctas, a.ctas = 1;
    const bool entropy = a.entropy || a.d_entropy || a.bonus != 0.f;
    return dtype ? run_token<bf16>(a, entropy, s) : run_token<float>(a, entropy, s);
}

cudaError_t launch_spread(const SpreadArgs& args, int rows, int dtype, Stream& s) {
    SpreadArgs a = args;
    a.rows = rows;
    return dtype ? run_spread<bf16>(a, s) : run_spread<float>(a, s);
}

}  // namespace hbsjd
