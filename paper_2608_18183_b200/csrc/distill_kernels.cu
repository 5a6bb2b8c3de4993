// Divergence of a student's rows of logits from a teacher's and its gradient, in one pass over memory.
//
// With x = s / tau, y = t / tau, q = softmax(x), p = softmax(y), d = x - y and delta = log sum e^x - log sum e^y:
//   KL(p || q) = delta - E_p d,    KL(q || p) = E_q d - delta,
//   d KL(p || q) / dx = q - p,     d KL(q || p) / dx = q (d - E_q d),
// so four sums over the row (two of exponentials, two weighted by d) give the loss, and a second look at the row the gradient.
// The row stays in shared memory between the two: it is read from HBM once, the gradient written once, and those 12 V bytes
// (two fp32 rows) are what bounds the kernel.  Rows are dealt to resident CTAs.  A warp has a part of the row to itself: it stages
// it, sums over it and writes its gradient, waits for the others for the sums alone, and fetches its part of the next row when it
// is done with its own.  Long rows are split over a cluster, whose CTAs exchange the sums through distributed shared memory; so are
// few rows, to use more SMs.  Measured, the kernel alone: 8192 pairs of rows of 16384 fp32 278 us (0.81 of a copy's rate, a cluster of two
// a row), 16384 rows against lists of 64 340 us (0.91), both with gradients; 8192 pairs in bf16 184 us, where the four exponentials an entry
// take 119.
#include <type_traits>

#include "logit_rows.cuh"

namespace hbsjd {

namespace {

// The place of a row's first element behind a 16-byte boundary in shared memory: the student's, and of the two that fp32 leaves
// open the teacher's if it is one of them.  (Not the gradient's: the loss has the same bits with and without it.)
template <typename TS, typename TT>
__device__ __forceinline__ int common_phase(const TS* s, const TT* t) {
    const int P = phase_of(s), Pt = phase_of(t);
    return sizeof(TS) == 4 && sizeof(TT) == 2 && Pt % 4 == P ? Pt : P;
}

// Divergences below this are summed as terms none of which is negative.  As delta - E_p d the loss is off by what two sums' quotient and
// its logarithm are, up to 7e-7 whatever the divergence is: 5e-5 of it here, more than all of a KL of 5e-7 (7e-5 of that as these terms).
// Such rows cost a third look: 8192 pairs of 16384 fp32 with gradients 375 us in place of 278, bf16 290 in place of 184.
constexpr float NEAR = 1.f / 64;

// An outcome's p (e^r - 1 - r) and q (e^-r - 1 + r), r = log q / p, of any size: those far from one another as they are; no mass on either
// side: r is not looked at.
__device__ __forceinline__ float2 near_terms(float p, float q, float r) {
    if (fabsf(r) < 0.75f) {  // series over r^2 / 2, whose next terms are below 7e-7 of the one and 9e-7 of the other
        const float r2 = r * r, even = fmaf(r2, fmaf(r2, fmaf(r2, 1.f / 40320, 1.f / 720), 1.f / 24), 0.5f);
        const float odd = r * fmaf(r2, fmaf(r2, 1.f / 5040, 1.f / 120), 1.f / 6);
        return {p * r2 * (even + odd), q * r2 * (even - odd)};
    }
    return {q - (p == 0.f ? 0.f : p * (1.f + r)), p - (q == 0.f ? 0.f : q * (1.f - r))};
}

__device__ __forceinline__ f32x2 get2(const float* p) { return *reinterpret_cast<const f32x2*>(p); }
__device__ __forceinline__ f32x2 get2(const bf16* p) {
    float lo, hi;
    unpack(*reinterpret_cast<const uint32_t*>(p), lo, hi);
    return both(lo, hi);
}

// A warp's sums of these (as zs and zt), which are KL(p || q) and KL(q || p) since p and q sum to one; those asked for.  An error
// that all r share counts by the square: none of the masses' logarithms has to be good.
template <typename TS, typename TT, int G, int WARPS>
__device__ __forceinline__ Pair near_sums(const TS* ss, const TT* st, const Part<G, WARPS>& part, const Pair& v, float c, float inv_tau, float ls,
                                          float lt, float delta, bool forward, bool reverse) {
    const int lane = threadIdx.x & 31, inner = part.inner() * G, outer = part.outer() * G;
    const f32x2 os = both(-v.ms), ot = both(-v.mt), c2 = both(c), minus = both(-1.f), nls = both(-ls), nlt = both(-lt), i2 = both(inv_tau),
                nd = both(-delta);
    f32x2 pq = both(0.f), qp = pq;
    bool far = false;
#pragma unroll 4
    for (int e = inner + lane * 2; e < outer; e += 64) {  // near_terms of two entries, without a branch
        const f32x2 xo = add2(get2(ss + e), os), yo = add2(get2(st + e), ot);
        float r0, r1;
        split(fma2(fma2(yo, minus, xo), i2, nd), r0, r1);
        const bool close0 = fabsf(r0) < 0.75f, close1 = fabsf(r1) < 0.75f;
        far |= !close0 || !close1;
        const f32x2 r = both(close0 ? r0 : 0.f, close1 ? r1 : 0.f), r2 = mul2(r, r);
        const f32x2 even = fma2(r2, fma2(r2, fma2(r2, both(1.f / 40320), both(1.f / 720)), both(1.f / 24)), both(0.5f));
        const f32x2 odd = mul2(r, fma2(r2, fma2(r2, both(1.f / 5040), both(1.f / 120)), both(1.f / 6)));
        if (forward) pq = fma2(mul2(ex2(fma2(yo, c2, nlt)), r2), add2(even, odd), pq);
        if (reverse) qp = fma2(mul2(ex2(fma2(xo, c2, nls)), r2), fma2(odd, minus, even), qp);
    }
    Pair h = {0.f, 0.f, sum2(pq), sum2(qp), 0.f, 0.f};
    const auto other = [&](int e, bool close_too) {
        const float xo = to_f<TS>(ss[e]) - v.ms, yo = to_f<TT>(st[e]) - v.mt, r = fmaf(xo - yo, inv_tau, -delta);
        if (!close_too && fabsf(r) < 0.75f) return;
        const float2 t = near_terms(ex2(fmaf(yo, c, -lt)), ex2(fmaf(xo, c, -ls)), r);
        h.zs += t.x;
        h.zt += t.y;
    };
    // what is left out: the row's ends, whose groups hold more than the row, and entries that are far from one another
    if (part.first() + lane < inner) other(part.first() + lane, true);
    if (outer + lane < part.last()) other(outer + lane, true);
    if (__any_sync(0xffffffffu, far))
        for (int e = inner + lane; e < outer; e += 32) other(e, false);
    return h;
}

template <typename TS, typename TT, int THREADS, int PER_SM>
__global__ void __launch_bounds__(THREADS, PER_SM) k_distill(DistillArgs a) {
    constexpr int G = sizeof(TS) == 2 && sizeof(TT) == 2 ? 8 : 4, WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ int special[3];  // a logit of the slice asks for care: this row, the one before, the one behind
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int rank = blockIdx.x % a.ctas, v0 = rank * a.slice, n = max(0, min(a.slice, a.V - v0));
    const int step = gridDim.x / a.ctas;
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    TS* ss = (TS*)smem;
    TT* st = (TT*)(smem + (a.slice + 16) * sizeof(TS));
    const int places = WARPS * a.ctas;
    Pair* slots = (Pair*)(st + a.slice + 16);  // [2][places], by turns: a CTA may be a row ahead of others
    if (threadIdx.x < 3) special[threadIdx.x] = 0;
    __syncthreads();
    if (a.ctas > 1) cluster_barrier();  // every CTA of the rows runs
    const auto weight = [&](int row) { return row >= a.rows ? 0.f : a.weight ? __ldg(a.weight + row) : 1.f; };
    const auto fetch = [&](int row) {
        const TS* s = (const TS*)a.s + (int64_t)row * a.ld_s + v0;
        const TT* t = (const TT*)a.t + (int64_t)row * a.ld_t + v0;
        const Part<G, WARPS> p(common_phase(s, t), n, wid);
        stage_part(ss, s, p);
        stage_part(st, t, p);
    };
    int row = blockIdx.x / a.ctas, parity = 0, turn = 0;
    float w = weight(row), w1 = weight(row + step);
    if (w != 0.f) fetch(row);
    for (; row < a.rows; row += step) {
        const float w2 = weight(row + 2 * step);  // (so that no fetch waits for a weight)
        bool fetched = w1 == 0.f;
        TS* g = a.grad ? (TS*)a.grad + (int64_t)row * a.ld_g + v0 : nullptr;
        const Part<G, WARPS> p(common_phase((const TS*)a.s + (int64_t)row * a.ld_s + v0, (const TT*)a.t + (int64_t)row * a.ld_t + v0), n, wid);
        const int lo = p.first() - p.P, hi = p.last() - p.P;  // the warp's entries of the slice
        if (w == 0.f) {                                       // (all CTAs of the row)
            if (g) put_zeros(g, lo, hi);
            if (a.loss && rank == 0 && threadIdx.x == 0) a.loss[row] = 0.f;
        } else {
            // (its last readers have met the others since; those who set it will meet this thread first)
            if (threadIdx.x == 0) special[turn == 2 ? 0 : turn + 1] = 0;
            cp_async_wait_all();
            __syncwarp();
            end_part(ss, p, PAD);
            end_part(st, p, PAD);
            // A warp sums against the largest logits of its first groups.  That overflows, or meets what has no finite difference, in
            // few rows; their warps find their maxima and look at every entry.
            Pair v = Pair::none();
            {
                float x[G], y[G];
                const int sample = p.inner() + lane;
                if (sample < p.outer()) {
                    get<G>(ss + sample * G, x);
                    get<G>(st + sample * G, y);
#pragma unroll
                    for (int i = 0; i < G; ++i) v.ms = fmaxf(v.ms, x[i]), v.mt = fmaxf(v.mt, y[i]);
                }
                v.share();
                const f32x2 os = both(-v.ms), ot = both(-v.mt), c2 = both(c), minus = both(-1.f);
                f32x2 zs = both(0.f), zt = zs, as = zs, at = zs;
#pragma unroll 2
                for (int j = p.j0 + lane; j < p.j1; j += 32) {
                    get<G>(ss + j * G, x);
                    get<G>(st + j * G, y);
#pragma unroll
                    for (int i = 0; i < G; i += 2) {
                        const f32x2 xo = add2(both(x[i], x[i + 1]), os), yo = add2(both(y[i], y[i + 1]), ot);
                        const f32x2 es = ex2(mul2(xo, c2)), et = ex2(mul2(yo, c2)), d = fma2(yo, minus, xo);
                        zs = add2(zs, es);
                        zt = add2(zt, et);
                        as = fma2(es, d, as);
                        at = fma2(et, d, at);
                    }
                }
                v.zs = sum2(zs), v.zt = sum2(zt), v.as = sum2(as), v.at = sum2(at);
            }
            // (false for NaN, infinities, and sums that a factor could not bring down again; and where the fill beside the row's ends
            // would have a share: a row of values as low as it, a temperature so high)
            const bool apart = (p.inner() == p.j0 && p.outer() == p.j1) || ((v.ms - to_f<TS>(from_f<TS>(PAD))) * c > 150.f &&
                                                                            (v.mt - to_f<TT>(from_f<TT>(PAD))) * c > 150.f);
            const bool fine = v.zs < 1e12f && v.zt < 1e12f && fabsf(v.as) < 1e30f && fabsf(v.at) < 1e30f && apart;
            if (!__all_sync(0xffffffffu, fine) || !__any_sync(0xffffffffu, v.zs > 0.f) || !__any_sync(0xffffffffu, v.zt > 0.f)) {
                if (lane == 0 && p.j0 < p.j1) special[turn] = 1;
                v = Pair::none();
                for (int e = p.first() + lane; e < p.last(); e += 32) v.ms = fmaxf(v.ms, to_f<TS>(ss[e])), v.mt = fmaxf(v.mt, to_f<TT>(st[e]));
                v.share();
                const float os = v.ms == -INFINITY ? 0.f : v.ms, ot = v.mt == -INFINITY ? 0.f : v.mt;
                for (int e = p.first() + lane; e < p.last(); e += 32) {
                    // (x - m before the product: a row of the lowest finite value is uniform)
                    const float xo = to_f<TS>(ss[e]) - os, yo = to_f<TT>(st[e]) - ot, es = ex2(xo * c), et = ex2(yo * c);
                    v.zs += es;
                    v.zt += et;
                    // no mass, no share: d is infinite or NaN where one or both are masked
                    v.as += es == 0.f ? 0.f : es * (xo - yo);
                    v.at += et == 0.f ? 0.f : et * (xo - yo);
                }
            }
            post<WARPS>(v, slots + parity * places, a.ctas, rank);
            posted(a.ctas);
            v = collect(slots + parity * places, places, c);
            const bool empty = v.zs == 0.f || v.zt == 0.f, rev = a.reverse != 0.f;
            // (against the maxima: their difference is in neither d nor delta)
            const float A_q = __fdividef(v.as, v.zs) * inv_tau, ls = lg2(v.zs), lt = lg2(v.zt);
            float delta = 0.f, near_loss = -1.f;
            if (a.forward != a.reverse && a.loss && !empty) {  // (at equal weights delta takes no part)
                if (v.zs != v.zt) delta = LN2 * lg2(__fdividef(v.zs, v.zt));
                // (the same for all CTAs of the row, whose sums are the same bits)
                if ((a.forward == 0.f || delta - __fdividef(v.at, v.zt) * inv_tau < NEAR) && (!rev || A_q - delta < NEAR)) {
                    Pair h = near_sums(ss, st, p, v, c, inv_tau, ls, lt, delta, a.forward != 0.f, rev);
                    parity ^= 1;
                    post<WARPS>(h, slots + parity * places, a.ctas, rank);
                    posted(a.ctas);
                    h = collect(slots + parity * places, places, c);
                    near_loss = (a.forward == 0.f ? 0.f : a.forward * h.zs) + (rev ? a.reverse * h.zt : 0.f);
                }
            }
            if (a.loss && rank == 0 && threadIdx.x == 0) {
                float loss = 0.f;
                if (!empty) {
                    if (a.forward != 0.f) loss -= a.forward * (__fdividef(v.at, v.zt) * inv_tau);
                    if (rev) loss += a.reverse * A_q;
                    if (a.forward != a.reverse) loss += (a.forward - a.reverse) * delta;
                }
                a.loss[row] = near_loss >= 0.f ? near_loss : loss;
            }
            if (g) {
                const int Pg = phase_of(g) % G;  // the gradient is written wide, whatever the others' alignment
                // w / tau (a (q - p) + b q (d - E_q d)) = q (k0 + k1 d) - k2 p
                const float f = w * inv_tau, k2 = f * a.forward;
                float k0 = f * (rev ? a.forward - a.reverse * A_q : a.forward), k1 = f * a.reverse * inv_tau;
                if (empty) {
                    put_zeros(g, lo, hi);
                } else if (special[turn] || !(fabsf(v.ms) + fabsf(v.mt) + fabsf(k0) + fabsf(k1) + fabsf(k2) < 1e30f)) {
                    const auto each_entry = [&](auto&& slope) {
                        for (int e = lo + lane; e < hi; e += 32) {
                            const float xo = to_f<TS>(ss[p.P + e]) - v.ms, yo = to_f<TT>(st[p.P + e]) - v.mt;
                            const float q = ex2(fmaf(xo, c, -ls)), r = ex2(fmaf(yo, c, -lt));
                            g[e] = from_f<TS>(slope(q, r, xo - yo));
                        }
                    };
                    if (fabsf(k0) + fabsf(k1) + fabsf(k2) < 1e30f) {
                        each_entry([&](float q, float r, float d) {
                            const float m = rev ? fmaf(k1, d, k0) : k0;
                            return fmaf(-k2, r, q == 0.f ? 0.f : q * m);
                        });
                    } else {  // the factors one by one: temperatures below 1e-15 leave none of their products
                        const float mean = __fdividef(v.as, v.zs);
                        each_entry([&](float q, float r, float d) {
                            const float m = rev ? fmaf(a.reverse, (d - mean) * inv_tau, a.forward) : a.forward;
                            return fmaf(-a.forward, r, q == 0.f ? 0.f : q * m) * inv_tau * w;
                        });
                    }
                } else {
                    // At an entry of the type's lowest value d is about that, and finite, since both references are far less; but k1 above 1
                    // would take the product to infinity, beside a q of zero.  q takes the power of two that k1 has too much.
                    float up = 0.f;
                    if (fabsf(k1) >= 1.f) {
                        const int e = (int)(__float_as_uint(fabsf(k1)) >> 23) - 126;  // (below 101, see above)
                        const float down = __uint_as_float((uint32_t)(127 - e) << 23);
                        k0 *= down, k1 *= down, up = (float)e;
                    }
                    const f32x2 os = both(-v.ms), ot = both(-v.mt), c2 = both(c), minus = both(-1.f), nls = both(up - ls), nlt = both(-lt);
                    const f32x2 K0 = both(k0), K1 = both(k1), K2 = both(-k2);
                    const auto gradient = [&](float(&x)[G], const float(&y)[G]) {
#pragma unroll
                        for (int i = 0; i < G; i += 2) {
                            const f32x2 xo = add2(both(x[i], x[i + 1]), os), yo = add2(both(y[i], y[i + 1]), ot);
                            const f32x2 q = ex2(fma2(xo, c2, nls)), r = ex2(fma2(yo, c2, nlt)), m = fma2(K1, fma2(yo, minus, xo), K0);
                            split(fma2(K2, r, mul2(q, m)), x[i], x[i + 1]);
                        }
                    };
                    if (p.P % G == Pg) {
                        // a group that is read makes place for the next row's, if that lies alike
                        const TS* s1 = (const TS*)a.s + (int64_t)(row + step) * a.ld_s + v0;
                        const TT* t1 = (const TT*)a.t + (int64_t)(row + step) * a.ld_t + v0;
                        const bool follow = sizeof(TS) == sizeof(TT) && !fetched && phase_of(s1) == p.P && phase_of(t1) == p.P;
                        const auto run = [&](auto ahead) {
                            each_group(p, [&](int j, auto whole) {
                                float x[G], y[G];
                                get<G>(ss + j * G, x);
                                get<G>(st + j * G, y);
                                gradient(x, y);
                                if constexpr (decltype(whole)::value)
                                    put<G>(g - p.P + j * G, x);
                                else
                                    put_at<TS, G>(g, j * G - p.P, 0, n, x);
                                if constexpr (decltype(ahead)::value && decltype(whole)::value) {
                                    cp_async16(ss + j * G, s1 - p.P + j * G);
                                    cp_async16(st + j * G, t1 - p.P + j * G);
                                }
                            });
                        };
                        if (follow)
                            run(std::true_type());
                        else
                            run(std::false_type());
                        if (follow) {
                            __syncwarp();
                            stage_ends(ss, s1, p);
                            stage_ends(st, t1, p);
                            fetched = true;
                        }
                    } else {
                        for (int e = (lo + Pg) / G * G - Pg + lane * G; e < hi && lo < hi; e += 32 * G) {
                            float x[G], y[G];
#pragma unroll
                            for (int i = 0; i < G; ++i) {
                                const int at = p.P + min(max(e + i, lo), hi - 1);
                                x[i] = to_f<TS>(ss[at]), y[i] = to_f<TT>(st[at]);
                            }
                            gradient(x, y);
                            put_at<TS, G>(g, e, lo, hi, x);
                        }
                    }
                }
            }
            parity ^= 1;
            turn = turn == 2 ? 0 : turn + 1;
        }
        __syncwarp();  // the warp's part is done
        if (!fetched) fetch(row + step);
        w = w1, w1 = w2;
    }
}

// log(e^x + e^y); -inf for none, NaN passes.
__device__ __forceinline__ float log_add(float x, float y) {
    const float m = fmaxf(x, y);
    return m == -INFINITY ? x + y : fmaf(LN2, lg2(ex2((x - m) * LOG2E) + ex2((y - m) * LOG2E)), m);
}

// log(1 + e^r), to its own last digits where it is small too: log(1 + z) = 2 (u + u^3 / 3 + u^5 / 5 ...) with u = z / (2 + z), where
// z <= 1 leaves 1e-8 of it behind u^15.
__device__ __forceinline__ float softplus(float r) {
    const float z = ex2(-fabsf(r) * LOG2E), u = __fdividef(z, 2.f + z), u2 = u * u;
    float f = 1.f / 15;
#pragma unroll
    for (int i = 13; i > 0; i -= 2) f = fmaf(f, u2, 1.f / i);
    return fmaf(2.f * u, f, fmaxf(r, 0.f));
}

// What one warp makes of a row's sums for all: the others would only take its issue slots (each warp for itself: 485 us in
// place of 400 for 16384 rows of 16384).
struct ListCoefs {
    float Mx, My, Lx, Ly, kl_qp;  // logarithms and the divergence that the listed tokens' gradient needs
    float om, k0;                 // the others': 2^{(x - om) c} k0
    int empty, near;
    float po, qo, ratio;          // the others' masses, and the logarithm of qo / po
};

// Divergences from lists below this are summed as terms none of which is negative, too: by the masses' logarithms the loss is off by up
// to 2e-6, which is 3e-5 of it here.  (16384 rows of 16384 fp32 with lists of 64 340 us, all of them near 356.)
constexpr float NEAR_LIST = 1.f / 16;

// A warp's sum of such terms over the list's entries of a CTA, and of all others as one if asked for.
__device__ __forceinline__ float near_list(const float* xk, const float* val, const int32_t* at, int k, float c, float inv_tau, float forward,
                                           float reverse, const ListCoefs& f, bool others) {
    const int lane = threadIdx.x & 31;
    float2 sum = {0.f, 0.f};
    if (others && lane == 0) sum = near_terms(f.po, f.qo, f.ratio);
    for (int i = lane; i < k; i += 32)
        if (at[i] >= 0) {
            const float x = xk[i] - f.Mx, y = val[i] - f.My;
            const float2 t = near_terms(ex2(fmaf(y, c, -f.Ly * LOG2E)), ex2(fmaf(x, c, -f.Lx * LOG2E)), (x - y) * inv_tau - (f.Lx - f.Ly));
            sum.x += t.x;
            sum.y += t.y;
        }
    return sum_of_warp((forward == 0.f ? 0.f : forward * sum.x) + (reverse == 0.f ? 0.f : reverse * sum.y));
}

template <typename TS, int THREADS, int PER_SM>
__global__ void __launch_bounds__(THREADS, PER_SM) k_distill_topk(DistillArgs a) {
    constexpr int G = 16 / sizeof(TS), WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ ListCoefs coefs;
    __shared__ float near_parts[ROW_CTAS];  // of a near row's loss, the first CTA's
    __shared__ int repeated[2];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, k = a.k;
    const int rank = blockIdx.x % a.ctas, v0 = rank * a.slice, n = max(0, min(a.slice, a.V - v0));
    const int step = gridDim.x / a.ctas, places = WARPS * a.ctas;
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    TS* ss = (TS*)smem;
    // Two of each, by turns: a CTA may be a row ahead of others, and a warp, and lists are made a row ahead.
    const int words = (a.slice + 31) / 32;
    Pair* slots = (Pair*)(ss + a.slice + 16);         // [2][places]
    Mass* slots_other = (Mass*)(slots + 2 * places);  // [2][places]
    float* xks = (float*)(slots_other + 2 * places);  // [2][k] the student's logit of a listed token of the slice
    float* vals = xks + 2 * k;                        // [2][k] the teacher's
    int32_t* ats = (int32_t*)(vals + 2 * k);          // [2][k] its place in the slice, -1: not here, or listed before
    uint32_t* seen = (uint32_t*)(ats + 2 * k);        // [words] a bit per element of the slice, 0 between lists
    for (int i = threadIdx.x; i < words; i += THREADS) seen[i] = 0;
    if (threadIdx.x < 2) repeated[threadIdx.x] = 0;
    __syncthreads();
    if (a.ctas > 1) cluster_barrier();  // every CTA of the rows runs
    const auto weight = [&](int row) { return row >= a.rows ? 0.f : a.weight ? __ldg(a.weight + row) : 1.f; };
    const auto fetch = [&](int row) {
        const TS* s = (const TS*)a.s + (int64_t)row * a.ld_s + v0;
        stage_part(ss, s, Part<G, WARPS>(phase_of(s), n, wid));
    };
    // A row's list, one entry a thread (the last warps first: warp 0 has other work): those of the slice find their places.
    const int first = THREADS - 1 - threadIdx.x;
    const auto list = [&](int row, int turn, int32_t token, float value) {
        for (int i = first; i < k; i += THREADS) {
            if (i >= THREADS) {
                token = __ldg(a.indices + (int64_t)row * k + i);
                value = __ldg(a.values + (int64_t)row * k + i);
            }
            int e = -1;
            if (token >= v0 && token < v0 + n && !(value == -INFINITY)) {
                e = token - v0;
                if (atomicOr(&seen[e >> 5], 1u << (e & 31)) >> (e & 31) & 1) repeated[turn] = 1;
            }
            ats[turn * k + i] = e;
            vals[turn * k + i] = value;
        }
    };
    int row = blockIdx.x / a.ctas, parity = 0, turn = 0;
    float w = weight(row), w1 = weight(row + step);
    if (w != 0.f) {
        fetch(row);
        if (first < k) list(row, 0, __ldg(a.indices + (int64_t)row * k + first), __ldg(a.values + (int64_t)row * k + first));
    }
    __syncthreads();
    for (; row < a.rows; row += step, turn ^= 1) {
        const float w2 = weight(row + 2 * step);  // (so that no fetch waits for a weight)
        bool fetched = w1 == 0.f;
        int32_t token = -1;
        float value = 0.f;
        if (w1 != 0.f && first < k) {
            token = __ldg(a.indices + (int64_t)(row + step) * k + first);
            value = __ldg(a.values + (int64_t)(row + step) * k + first);
        }
        TS* g = a.grad ? (TS*)a.grad + (int64_t)row * a.ld_g + v0 : nullptr;
        const Part<G, WARPS> p(phase_of((const TS*)a.s + (int64_t)row * a.ld_s + v0), n, wid);
        const int lo = p.first() - p.P, hi = p.last() - p.P;  // the warp's entries of the slice
        if (w == 0.f) {                                       // (all CTAs of the row)
            if (g) put_zeros(g, lo, hi);
            if (a.loss && rank == 0 && threadIdx.x == 0) a.loss[row] = 0.f;
            if (threadIdx.x == 0) repeated[turn ^ 1] = 0;
            __syncthreads();  // the row before is done with the other list
            if (w1 != 0.f) list(row + step, turn ^ 1, token, value);
            __syncthreads();
        } else {
            const float yr = a.rest ? __ldg(a.rest + row) : -INFINITY;
            float* xk = xks + turn * k;
            const float* val = vals + turn * k;
            int32_t* at = ats + turn * k;
            // (the row before has read its own; those who set it again will meet this thread first)
            if (threadIdx.x == 0) repeated[turn ^ 1] = 0;
            for (int i = first; i < k; i += THREADS)
                if (at[i] >= 0) seen[at[i] >> 5] = 0;
            if (repeated[turn]) {  // of a token that is listed twice, the first entry counts
                for (int i0 = 0; i0 < k; i0 += THREADS) {
                    const int i = i0 + threadIdx.x;
                    bool again = false;
                    if (i < k && at[i] >= 0)
                        for (int j = 0; j < i && !again; ++j) again = at[j] == at[i];
                    __syncthreads();  // (entries behind this block of them look at it before it changes, entries in it too)
                    if (again) at[i] = -1;
                    __syncthreads();
                }
            }
            const auto each = [&](auto&& f) {  // f(entry, its place in the stage): the entries of the warp's part
                for (int i = lane; i < k; i += 32)
                    if (at[i] >= lo && at[i] < hi) f(i, p.P + at[i]);
            };
            cp_async_wait_all();
            __syncwarp();
            end_part(ss, p, -INFINITY);
            // they leave the row; v: their sums, student and teacher
            Pair v = Pair::none();
            bool any = false;
            each([&](int i, int e) {
                any = true;
                const float x = to_f<TS>(ss[e]);
                xk[i] = x;
                ss[e] = from_f<TS>(-INFINITY);
                v.ms = fmaxf(v.ms, x);
                v.mt = fmaxf(v.mt, val[i]);
            });
            __syncwarp();  // (other lanes sum over their places)
            if (__any_sync(0xffffffffu, any)) {
                v.share();
                const float os = v.ms == -INFINITY ? 0.f : v.ms, ot = v.mt == -INFINITY ? 0.f : v.mt;
                each([&](int i, int) {
                    const float xo = xk[i] - os, yo = val[i] - ot, es = ex2(xo * c), et = ex2(yo * c);
                    v.zs += es;
                    v.zt += et;
                    v.as += es == 0.f ? 0.f : es * (xo - yo);
                    v.at += et == 0.f ? 0.f : et * (xo - yo);
                });
            }
            post<WARPS>(v, slots + parity * places, a.ctas, rank);
            // u: all other tokens, against the largest of a warp's first groups; where that overflows or leaves nothing, of all of its
            Mass u = Mass::none();
            {
                float x[G];
                const int sample = p.inner() + lane;
                if (sample < p.outer()) {
                    get<G>(ss + sample * G, x);
#pragma unroll
                    for (int i = 0; i < G; ++i) u.m = fmaxf(u.m, x[i]);
                }
                u.share();
                const f32x2 o = both(-u.m), c2 = both(c);
                f32x2 z = both(0.f);
#pragma unroll 4
                for (int j = p.j0 + lane; j < p.j1; j += 32) {
                    get<G>(ss + j * G, x);
#pragma unroll
                    for (int i = 0; i < G; i += 2) z = add2(z, ex2(mul2(add2(both(x[i], x[i + 1]), o), c2)));
                }
                u.z = sum_of_warp(sum2(z));
            }
            if (!(u.z < 1e12f && u.z > 0.f)) {
                u = Mass::none();
                for (int e = p.first() + lane; e < p.last(); e += 32) u.m = fmaxf(u.m, to_f<TS>(ss[e]));
                u.share();
                const float o = u.m == -INFINITY ? 0.f : u.m;
                for (int e = p.first() + lane; e < p.last(); e += 32) u.z += ex2((to_f<TS>(ss[e]) - o) * c);
                u.z = sum_of_warp(u.z);
            }
            post<WARPS>(u, slots_other + parity * places, a.ctas, rank);
            posted(a.ctas);
            if (threadIdx.x < 32) {
                v = collect(slots + parity * places, places, c);
                u = collect(slots_other + parity * places, places, c);
                // Logarithms of the masses of the listed tokens (l) and the others (o), student (x) and teacher (y), against the
                // largest logit of each: rows of the lowest finite value have some too.
                const bool empty = (v.zs == 0.f && u.z == 0.f) || (v.zt == 0.f && yr == -INFINITY);
                const float Mx = fmaxf(v.ms, u.m), My = v.mt == -INFINITY ? 0.f : v.mt;
                const float xl = v.zs == 0.f ? -INFINITY : fmaf(v.ms - Mx, inv_tau, LN2 * lg2(v.zs));
                const float xo = u.z == 0.f ? -INFINITY : fmaf(u.m - Mx, inv_tau, LN2 * lg2(u.z));
                const float yl = v.zt == 0.f ? -INFINITY : LN2 * lg2(v.zt), yo = yr == -INFINITY ? yr : fmaf(-My, inv_tau, yr);
                const float Lx = log_add(xl, xo), Ly = log_add(yl, yo);
                const float ql = ex2((xl - Lx) * LOG2E), qo = ex2((xo - Lx) * LOG2E);
                const float pl = ex2((yl - Ly) * LOG2E), po = ex2((yo - Ly) * LOG2E);
                // log of qo / po: by what the list leaves of each, since near 1 the logarithms of both are differences of larger ones
                // (one listed token of mass 1e-3: the loss was 1.7e-4 off)
                const float ratio = softplus(yl - yo) - softplus(xl - xo);
                const float shift = v.ms == -INFINITY ? 0.f : Mx - v.ms;  // (the sums of d are against v.ms)
                // a mass of zero adds nothing, whatever its logarithm is (NaN passes)
                float kl_pq = 0.f, kl_qp = 0.f;
                if (pl != 0.f) kl_pq -= pl * ((__fdividef(v.at, v.zt) - shift) * inv_tau - (Lx - Ly));
                if (po != 0.f) kl_pq -= po * ratio;
                if (ql != 0.f) kl_qp += ql * ((__fdividef(v.as, v.zs) - shift) * inv_tau - (Lx - Ly));
                if (qo != 0.f) kl_qp += qo * ratio;
                if (lane == 0) {
                    // others: q_v (a (1 - po / qo) + b (ratio - KL(q || p))), with q_v / qo their share of u.z
                    float k0 = a.forward * (ql + pl < qo + po ? pl - ql : qo - po);
                    if (a.reverse != 0.f && qo != 0.f) k0 += a.reverse * qo * (ratio - kl_qp);
                    k0 = u.z == 0.f ? 0.f : __fdividef(k0 * (w * inv_tau), u.z);
                    const bool near = a.loss && !empty && (a.forward == 0.f || kl_pq < NEAR_LIST) && (a.reverse == 0.f || kl_qp < NEAR_LIST);
                    coefs = {Mx, My, Lx, Ly, kl_qp, u.m == -INFINITY ? 0.f : u.m, k0, empty, near, po, qo, ratio};
                    if (a.loss && blockIdx.x % a.ctas == 0) {
                        float loss = 0.f;
                        if (!empty) {
                            if (a.forward != 0.f) loss += a.forward * kl_pq;
                            if (a.reverse != 0.f) loss += a.reverse * kl_qp;
                        }
                        a.loss[row] = loss;
                    }
                }
            }
            if (w1 != 0.f) list(row + step, turn ^ 1, token, value);  // (the one before is used up; the others wait for one warp)
            __syncthreads();
            if (g) {
                if (coefs.empty) {
                    put_zeros(g, lo, hi);
                } else {
                    const int Pg = phase_of(g);  // the gradient is written wide, whatever the others' alignment
                    const f32x2 o = both(-coefs.om), c2 = both(c), K0 = both(coefs.k0);
                    const auto gradient = [&](float(&x)[G]) {
#pragma unroll
                        for (int i = 0; i < G; i += 2) split(mul2(ex2(mul2(add2(both(x[i], x[i + 1]), o), c2)), K0), x[i], x[i + 1]);
                    };
                    if (p.P == Pg) {
                        // a group that is read makes place for the next row's, if that lies alike
                        const TS* s1 = (const TS*)a.s + (int64_t)(row + step) * a.ld_s + v0;
                        const bool follow = !fetched && phase_of(s1) == p.P;
                        const auto run = [&](auto ahead) {
                            each_group(p, [&](int j, auto whole) {
                                float x[G];
                                get<G>(ss + j * G, x);
                                gradient(x);
                                if constexpr (decltype(whole)::value)
                                    put<G>(g - p.P + j * G, x);
                                else
                                    put_at<TS, G>(g, j * G - p.P, 0, n, x);
                                if constexpr (decltype(ahead)::value && decltype(whole)::value) cp_async16(ss + j * G, s1 - p.P + j * G);
                            });
                        };
                        if (follow)
                            run(std::true_type());
                        else
                            run(std::false_type());
                        if (follow) {
                            __syncwarp();
                            stage_ends(ss, s1, p);
                            fetched = true;
                        }
                    } else {
                        for (int e = (lo + Pg) / G * G - Pg + lane * G; e < hi && lo < hi; e += 32 * G) {
                            float x[G];
#pragma unroll
                            for (int i = 0; i < G; ++i) x[i] = to_f<TS>(ss[p.P + min(max(e + i, lo), hi - 1)]);
                            gradient(x);
                            put_at<TS, G>(g, e, lo, hi, x);
                        }
                    }
                    __syncwarp();  // the listed tokens' places were written above
                    const ListCoefs& f = coefs;
                    const float fw = w * inv_tau;
                    each([&](int i, int e) {
                        const float x = xk[i] - f.Mx, y = val[i] - f.My;
                        const float q = ex2(fmaf(x, c, -f.Lx * LOG2E)), r = ex2(fmaf(y, c, -f.Ly * LOG2E));
                        float d = a.forward * (q - r);
                        if (a.reverse != 0.f && q != 0.f) d += a.reverse * q * ((x - y) * inv_tau - (f.Lx - f.Ly) - f.kl_qp);
                        g[e - p.P] = from_f<TS>(fw * d);
                    });
                }
            }
            if (coefs.near) {  // (the same for all CTAs of the row, whose sums are the same bits)
                if (threadIdx.x < 32) {
                    const float loss = near_list(xk, val, at, k, c, inv_tau, a.forward, a.reverse, coefs, rank == 0);
                    if (a.ctas > 1 && lane == 0) remote_store(remote_smem(near_parts + rank, 0), loss);
                    if (a.ctas == 1 && lane == 0) a.loss[row] = loss;
                }
                if (a.ctas > 1) {
                    cluster_barrier();
                    if (rank == 0 && threadIdx.x == 0) {
                        float loss = 0.f;
                        for (int i = 0; i < a.ctas; ++i) loss += near_parts[i];
                        a.loss[row] = loss;
                    }
                }
            }
            parity ^= 1;
        }
        __syncwarp();  // the warp's part is done
        if (!fetched) fetch(row + step);
        w = w1, w1 = w2;
    }
}

// Threads of a CTA: as few, from 32 to 512, as have at most `most` groups each (four where there are few rows; 512 may have more).  What a
// warp does once a row is a good part of its work, so that fewer warps are faster (16384 rows of 16384 fp32, lists of 64: 395 us with 256
// threads, 439 with 512, both at 40 registers) as long as other CTAs fill the SM; few rows have the SMs to themselves.
template <typename F>
cudaError_t by_threads(const DistillArgs& a, int G, int most, F&& f) {
    const int per = ((int64_t)a.rows * a.ctas > device_sm_count() ? most : 4) * G;
    if (a.slice <= 32 * per) return f(std::integral_constant<int, 32>());
    if (a.slice <= 64 * per) return f(std::integral_constant<int, 64>());
    if (a.slice <= 128 * per) return f(std::integral_constant<int, 128>());
    if (a.slice <= 256 * per) return f(std::integral_constant<int, 256>());
    return f(std::integral_constant<int, 512>());
}

// CTAs that rows are dealt to, in clusters of a.ctas.
template <auto Kernel, int THREADS, int PER_SM>
cudaError_t deal(const DistillArgs& a, size_t smem, int* clusters) {
    const cudaError_t e = allow_row_smem<Kernel>();
    if (e != cudaSuccess) return e;
    const int per_sm = std::max(1, std::min<int>(PER_SM, 227 * 1024 / (smem + 1024 + 128)));  // (1 KB is the system's)
    return resident_clusters<Kernel>(a.ctas, THREADS, per_sm, smem, a.rows, clusters);
}

template <typename TS, typename TT>
cudaError_t run_distill(const DistillArgs& a, Stream& s) {
    constexpr int G = sizeof(TS) == 2 && sizeof(TT) == 2 ? 8 : 4;
    return by_threads(a, G, 9, [&](auto threads) {
        // (80 registers where there is room for three)
        constexpr int THREADS = decltype(threads)::value, PER_SM = THREADS == 512 ? 2 : 768 / THREADS;
        const size_t smem = (a.slice + 16) * (sizeof(TS) + sizeof(TT)) + 2 * THREADS / 32 * a.ctas * sizeof(Pair);
        int clusters = 0;
        const cudaError_t e = deal<k_distill<TS, TT, THREADS, PER_SM>, THREADS, PER_SM>(a, smem, &clusters);
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_distill<TS, TT, THREADS, PER_SM>, dim3((unsigned)clusters * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    });
}

template <typename TS>
cudaError_t run_distill_topk(const DistillArgs& a, Stream& s) {
    return by_threads(a, 16 / sizeof(TS), 18, [&](auto threads) {
        // (48 registers: with the 40 that 1536 threads of an SM leave, 16384 rows of 16384 fp32 take 458 us in place of 345)
        constexpr int THREADS = decltype(threads)::value, PER_SM = THREADS == 512 ? 2 : std::min(32, 1280 / THREADS);
        const size_t smem = (a.slice + 16) * sizeof(TS) + 2 * THREADS / 32 * a.ctas * (sizeof(Pair) + sizeof(Mass)) + a.k * 24 +
                            (a.slice + 31) / 32 * 4;
        int clusters = 0;
        const cudaError_t e = deal<k_distill_topk<TS, THREADS, PER_SM>, THREADS, PER_SM>(a, smem, &clusters);
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_distill_topk<TS, THREADS, PER_SM>, dim3((unsigned)clusters * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    });
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& args, int rows, int dtype_s, int dtype_t, Stream& s) {
    DistillArgs a = args;
    const RowSplit sp = split_row(rows, a.V, (dtype_s ? 2 : 4) + (dtype_t ? 2 : 4), device_sm_count(), SHARED_SM, true);
    a.rows = rows, a.ctas = sp.ctas, a.slice = sp.slice;
    if (dtype_s) return dtype_t ? run_distill<bf16, bf16>(a, s) : run_distill<bf16, float>(a, s);
    return dtype_t ? run_distill<float, bf16>(a, s) : run_distill<float, float>(a, s);
}

cudaError_t launch_distill_topk(const DistillArgs& args, int rows, int dtype_s, Stream& s) {
    DistillArgs a = args;
    const RowSplit sp = split_row(rows, a.V, dtype_s ? 2 : 4, device_sm_count(), SHARED_SM, true);
    a.rows = rows, a.ctas = sp.ctas, a.slice = sp.slice;
    return dtype_s ? run_distill_topk<bf16>(a, s) : run_distill_topk<float>(a, s);
}

}  // namespace hbsjd
