// Log-probabilities of sampled tokens, the clipped policy loss and what both give back to the logits, in one pass over memory.
//
// With x = logits / tau, q = softmax(x), t the row's token and o all others:
//   D = log sum_o e^x - x_t,   l = log q_t = -log(1 + e^D),   sum_o q = 1 / (1 + e^-D),
//   H = -sum q log q,          d (a l + b H) / dx_v = a (1[v = t] - q_v) - b q_v (log q_v + H).
// The token leaves the row before the row is summed, so that neither l nor 1 - q_t is a difference of near numbers: a token of almost
// all the mass has digits in both.  Two sums over the others (exponentials, and weighted by their exponents where the entropy is
// wanted) give the loss, and a second look at the row the gradient.
#include <type_traits>

#include "logit_rows.cuh"

namespace hbsjd {

namespace {

// Sums of e = 2^t, t = (x - m) c, over entries of a row, and of e t.
struct TokenSums {
    float m, z, a;
    __device__ __forceinline__ static TokenSums none() { return {-INFINITY, 0.f, 0.f}; }
};

// No less than this is an exponent taken to be: 2^t is zero below 2^-126, and zero times it is zero.  NaN passes.
__device__ __forceinline__ float held(float t) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(t), "f"(-200.f));
    return r;
}

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
// The row's sums from its warps', the same bits in every warp.
template <bool ENT>
__device__ __forceinline__ TokenSums collect_sums(const TokenSums* slots, int count, float c) {
    const int lane = threadIdx.x & 31;
    TokenSums r = TokenSums::none();
    for (int j = lane; j < count; j += 32) r.m = fmaxf(r.m, slots[j].m);
    r.m = max_of_warp(r.m);
    for (int j = lane; j < count; j += 32) {
        const TokenSums s = slots[j];
        const float f = rescale(s.m, r.m, c);
        r.z += s.z * f;
        if (ENT && f != 0.f) r.a += f * fmaf(s.z, s.m == r.m ? 0.f : (s.m - r.m) * c, s.a);
    }
    r.z = sum_of_warp(r.z);
    if (ENT) r.a = sum_of_warp(r.a);
    return r;
}

// e^d - 1 - d: by series where |d| < 3/4, whose next terms are below 7e-7 of it.
__device__ __forceinline__ float exp_excess(float d) {
    if (fabsf(d) < 0.75f) {
        const float d2 = d * d, even = fmaf(d2, fmaf(d2, fmaf(d2, 1.f / 40320, 1.f / 720), 1.f / 24), 0.5f);
        return d2 * fmaf(d, fmaf(d2, fmaf(d2, 1.f / 5040, 1.f / 120), 1.f / 6), even);
    }
    return d > 40.f ? expf(d) : expf(d) - 1.f - d;
}

// What a row has besides its logits.
struct RowTerms {
    float weight, A, old, ref, d_logp, d_entropy;
};
__device__ __forceinline__ RowTerms terms_of(const TokenArgs& a, int row) {
    const auto get = [&](const float* p, float other) { return p ? __ldg(p + row) : other; };
    return {get(a.weight, 1.f), get(a.advantage, 0.f), get(a.old_logp, 0.f), get(a.ref, 0.f), get(a.d_logp, 0.f), get(a.d_entropy, 0.f)};
}

// The loss of a token whose log-probability is l, but for the entropy's part, and its slope in l.
__device__ __forceinline__ float2 policy(const TokenArgs& a, const RowTerms& row, float l) {
    const float A = row.A, r = !a.old_logp || l == row.old ? (l == l ? 1.f : l) : expf(l - row.old);
    // (comparisons that let NaN pass; no advantage times an infinite ratio is none)
    const float low = 1.f - a.low, high = 1.f + a.high, clipped = r < low ? low : r > high ? high : r;
    const float kept = A == 0.f && r == INFINITY ? 0.f : r * A, other = clipped * A;
    float gain = other < kept ? other : kept, slope = other < kept ? 0.f : -kept;
    if (a.dual > 0.f && A < 0.f && gain < a.dual * A) gain = a.dual * A, slope = 0.f;
    float loss = -gain;
    if (a.kl != 0.f && a.ref) {
        const float d = l == row.ref ? 0.f : row.ref - l, excess = exp_excess(d);
        loss = fmaf(a.kl, excess, loss);
        slope = fmaf(-a.kl, d < -20.f ? -1.f : excess + d, slope);  // (e^d - 1)
    }
    return {loss, slope};
}

template <typename T, bool ENT, int THREADS, int PER_SM>
__global__ void __launch_bounds__(THREADS, PER_SM) k_token(TokenArgs a) {
    constexpr int G = 16 / sizeof(T), WARPS = THREADS / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
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
    const auto fetch = [&](int row) {
        const T* x = row_at(row) + v0;
        stage_part(ss, x, Part<G, WARPS>(phase_of(x), n, wid));
    };
    int row = blockIdx.x / a.ctas, parity = 0;
    int t = token_of(row), t1 = token_of(row + step);
    float xt = logit_of(row, t);
    if (t >= 0) fetch(row);
    for (; row < a.rows; row += step) {
        // (so that no fetch waits for a token, and no row for its logit; no gradient that takes a row's place has been written yet)
        const int t2 = token_of(row + 2 * step);
        const float xt1 = logit_of(row + step, t1);
        const RowTerms terms = terms_of(a, row);
        bool fetched = t1 < 0;
        T* g = a.grad ? (T*)a.grad + (int64_t)row * a.ld_g + v0 : nullptr;
        const T* x0 = row_at(row) + v0;
        const T* x1 = row_at(row + step) + v0;
        const Part<G, WARPS> p(phase_of(x0), n, wid);
        const int lo = p.first() - p.P, hi = p.last() - p.P;  // the warp's entries of the slice
        const int64_t place = a.at ? (int64_t)__ldg(a.at + row).x * a.T + __ldg(a.at + row).y : row;
        const bool first = rank == 0 && threadIdx.x == 0;
        if (t < 0) {  // (all CTAs of the row)
            if (g) put_zeros(g, lo, hi);
            if (first && !a.at) {
                if (a.loss) a.loss[row] = 0.f;
                if (a.logp) a.logp[row] = 0.f;
                if (a.entropy) a.entropy[row] = 0.f;
            }
        } else {
            const int mine = t - v0 >= lo && t - v0 < hi ? t - v0 : -1;  // the token, if it is one of the warp's
            // a group that is read for the last time makes place for the next row's, if that lies alike
            const bool alike = !fetched && phase_of(x1) == p.P;
            cp_async_wait_all();
            __syncwarp();
            if (mine >= 0 && lane == 0) ss[p.P + mine] = from_f<T>(-INFINITY);
            end_part(ss, p, -INFINITY);
            // A warp sums against the largest logit of its first groups.  That overflows, or leaves nothing, in few rows; their warps
            // find their maxima and look at every entry.
            TokenSums v = TokenSums::none();
            {
                float x[G];
                const int sample = p.inner() + lane;
                if (sample < p.outer()) {
                    get<G>(ss + sample * G, x);
#pragma unroll
                    for (int i = 0; i < G; ++i) v.m = fmaxf(v.m, x[i]);
                }
                v.m = max_of_warp(v.m);
                __syncwarp();  // (the groups of the sample are other lanes' below, and may make place there)
                const f32x2 o = both(-v.m), c2 = both(c);
                f32x2 z = both(0.f), w = z;
                const auto add = [&](int j) {
                    get<G>(ss + j * G, x);
#pragma unroll
                    for (int i = 0; i < G; i += 2) {
                        f32x2 e = mul2(add2(both(x[i], x[i + 1]), o), c2);
                        if constexpr (ENT) {
                            float e0, e1;
                            split(e, e0, e1);
                            e = both(held(e0), held(e1));
                        }
                        const f32x2 q = ex2(e);
                        z = add2(z, q);
                        if constexpr (ENT) w = fma2(q, e, w);
                    }
                };
                if (!g && alike) {
                    each_group(p, [&](int j, auto whole) {
                        add(j);
                        if constexpr (decltype(whole)::value) cp_async16(ss + j * G, x1 - p.P + j * G);
                    });
                    __syncwarp();
                    stage_ends(ss, x1, p);
                    fetched = true;
                } else {
#pragma unroll 4
                    for (int j = p.j0 + lane; j < p.j1; j += 32) add(j);
                }
                v.z = sum_of_warp(sum2(z));
                if (ENT) v.a = sum_of_warp(sum2(w));
            }
            if (!(v.z < 1e12f && v.z > 0.f)) {
                v = TokenSums::none();
                for (int e = lo + lane; e < hi; e += 32)
                    if (e != mine) v.m = fmaxf(v.m, to_f<T>(x0[e]));
                v.m = max_of_warp(v.m);
                const float o = v.m == -INFINITY ? 0.f : v.m;
                for (int e = lo + lane; e < hi; e += 32)
                    if (e != mine) {
                        const float s = held((to_f<T>(x0[e]) - o) * c), q = ex2(s);
                        v.z += q;
                        v.a = fmaf(q, s, v.a);
                    }
                v.z = sum_of_warp(v.z);
                v.a = sum_of_warp(v.a);
            }
            post_sums<ENT, WARPS>(v, slots + parity * places, a.ctas, rank);
            if (!g && !fetched) {
                __syncwarp();
                fetch(row + step);
                fetched = true;
            }
            posted(a.ctas);
            v = collect_sums<ENT>(slots + parity * places, places, c);
            parity ^= 1;
            const bool empty = v.z == 0.f && xt == -INFINITY;
            // (logf: log q is as good as its rounding; with lg2 alone it is 2e-6 off.  An infinite logit: NaN)
            const float D = xt < INFINITY ? fmaf(v.m - xt, inv_tau, logf(v.z)) : NAN, s = expf(-fabsf(D)), share = __fdividef(1.f, 1.f + s);
            const float qo = D > 0.f ? share : s * share, qt = D > 0.f ? s * share : share;  // masses of the others and of the token
            const float near = log1pf(s);                                                    // log q of the larger of both, negative
            const float l = -(near + fmaxf(D, 0.f));
            const float Lk = logf(v.z) + (near + fmaxf(-D, 0.f));  // log q_v = ln2 t_v - Lk
            float H = 0.f;
            if (ENT) H = (v.z == 0.f || qo == 0.f ? 0.f : qo * (Lk - LN2 * __fdividef(v.a, v.z))) - (qt == 0.f ? 0.f : qt * l);
            float2 f = {0.f, 0.f};
            if (a.advantage) f = policy(a, terms, l);
            if (first) {
                if (a.loss) a.loss[row] = empty ? 0.f : a.bonus != 0.f ? fmaf(-a.bonus, H, f.x) : f.x;
                if (a.logp) a.logp[place] = empty ? -INFINITY : l == 0.f ? 0.f : l;
                if (ENT && a.entropy) a.entropy[place] = empty ? 0.f : H;
            }
            if (g) {
                const int Pg = phase_of(g);  // the gradient is written wide, whatever the others' alignment
                const float scale = terms.weight * inv_tau, A = a.d_logp ? terms.d_logp : f.y, B = a.d_entropy ? -terms.d_entropy : a.bonus;
                // others: e_v (k0 + k1 t_v)
                const float K = __fdividef(qo, v.z), k0 = scale * K * (ENT ? fmaf(B, H - Lk, -A) : -A), k1 = ENT ? scale * K * B * LN2 : 0.f;
                if (empty || (v.z == 0.f && xt < INFINITY)) {
                    put_zeros(g, lo, hi);
                } else if (!(fabsf(k0) + fabsf(k1) < 1e30f)) {  // the factors one by one; NaN passes
                    for (int e = lo + lane; e < hi; e += 32) {
                        const float u = held((to_f<T>(ss[p.P + e]) - v.m) * c), q = ex2(u) * K;
                        const float m = ENT ? fmaf(B, fmaf(LN2, u, H - Lk), -A) : -A;
                        g[e] = from_f<T>(q == 0.f ? 0.f : q * m * scale);
                    }
                } else {
                    const f32x2 o = both(-v.m), c2 = both(c), K0 = both(k0), K1 = both(k1);
                    const auto gradient = [&](float(&x)[G]) {
#pragma unroll
                        for (int i = 0; i < G; i += 2) {
                            f32x2 u = mul2(add2(both(x[i], x[i + 1]), o), c2);
                            if constexpr (ENT) {
                                float u0, u1;
                                split(u, u0, u1);
                                u = both(held(u0), held(u1));
                                split(mul2(ex2(u), fma2(K1, u, K0)), x[i], x[i + 1]);
                            } else {
                                split(mul2(ex2(u), K0), x[i], x[i + 1]);
                            }
                        }
                    };
                    if (p.P == Pg) {
                        const auto run = [&](auto ahead) {
                            each_group(p, [&](int j, auto whole) {
                                float x[G];
                                get<G>(ss + j * G, x);
                                gradient(x);
                                if constexpr (decltype(whole)::value)
                                    put<G>(g - p.P + j * G, x);
                                else
                                    put_at<T, G>(g, j * G - p.P, 0, n, x);
                                if constexpr (decltype(ahead)::value && decltype(whole)::value) cp_async16(ss + j * G, x1 - p.P + j * G);
                            });
                        };
                        if (alike)
                            run(std::true_type());
                        else
                            run(std::false_type());
                        if (alike) {
                            __syncwarp();
                            stage_ends(ss, x1, p);
                            fetched = true;
                        }
                    } else {
                        for (int e = (lo + Pg) / G * G - Pg + lane * G; e < hi && lo < hi; e += 32 * G) {
                            float x[G];
#pragma unroll
                            for (int i = 0; i < G; ++i) x[i] = to_f<T>(ss[p.P + min(max(e + i, lo), hi - 1)]);
                            gradient(x);
                            put_at<T, G>(g, e, lo, hi, x);
                        }
                    }
                }
                __syncwarp();  // the token's place was written above
                if (mine >= 0 && lane == 0 && !empty) {
                    float d = A * qo;
                    if (ENT) d += B * (qt == 0.f ? 0.f : qt * (l + H));
                    g[mine] = from_f<T>(scale * d);
                }
            }
        }
        __syncwarp();  // the warp's part is done
        if (!fetched) fetch(row + step);
        t = t1, t1 = t2, xt = xt1;
    }
}

template <typename T, bool ENT>
cudaError_t run_token(const TokenArgs& a, Stream& s) {
    // Threads of a CTA: see by_threads in distill_kernels.cu
    const auto run = [&](auto threads) {
        constexpr int THREADS = decltype(threads)::value, PER_SM = THREADS == 512 ? 2 : std::min(32, 1280 / THREADS);
        const size_t smem = (a.slice + 16) * sizeof(T) + 2 * THREADS / 32 * a.ctas * sizeof(TokenSums);
        cudaError_t e = allow_row_smem<k_token<T, ENT, THREADS, PER_SM>>();
        if (e != cudaSuccess) return e;
        const int per_sm = std::max(1, std::min<int>(PER_SM, 227 * 1024 / (smem + 1024 + 128)));  // (1 KB is the system's)
        int clusters = 0;
        e = resident_clusters<k_token<T, ENT, THREADS, PER_SM>>(a.ctas, THREADS, per_sm, smem, a.rows, &clusters);
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_token<T, ENT, THREADS, PER_SM>, dim3((unsigned)clusters * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    };
    const int per = ((int64_t)a.rows * a.ctas > device_sm_count() ? 18 : 4) * 16 / (int)sizeof(T);
    if (a.slice <= 32 * per) return run(std::integral_constant<int, 32>());
    if (a.slice <= 64 * per) return run(std::integral_constant<int, 64>());
    if (a.slice <= 128 * per) return run(std::integral_constant<int, 128>());
    if (a.slice <= 256 * per) return run(std::integral_constant<int, 256>());
    return run(std::integral_constant<int, 512>());
}

}  // namespace

cudaError_t launch_token(const TokenArgs& args, int rows, int dtype, Stream& s) {
    TokenArgs a = args;
    const RowSplit sp = split_row(rows, a.V, dtype ? 2 : 4, device_sm_count(), SHARED_SM, true);
    a.rows = rows, a.ctas = sp.ctas, a.slice = sp.slice;
    const bool entropy = a.entropy || a.d_entropy || a.bonus != 0.f;
    if (dtype) return entropy ? run_token<bf16, true>(a, s) : run_token<bf16, false>(a, s);
    return entropy ? run_token<float, true>(a, s) : run_token<float, false>(a, s);
}

}  // namespace hbsjd
