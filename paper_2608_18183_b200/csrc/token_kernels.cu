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

// G elements of a staged row; with FLOOR none below -1e30, so that exponents stay finite.  NaN passes.
constexpr float FLOOR_VALUE = -1e30f;
__device__ __forceinline__ float above(float x) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(x) : "f"(FLOOR_VALUE));
    return x;
}
template <bool FLOOR>
__device__ __forceinline__ void read(const float* p, float (&x)[4]) {
    get<4>(p, x);
    if constexpr (FLOOR) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = above(x[i]);
    }
}
template <bool FLOOR>
__device__ __forceinline__ void read(const bf16* p, float (&x)[8]) {
    uint4 v = *reinterpret_cast<const uint4*>(p);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FLOOR) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(w[i]) : "r"(0xf149f149u));  // (-9.95e29)
        unpack(w[i], x[2 * i], x[2 * i + 1]);
    }
}

__device__ __forceinline__ void put2(float* p, float lo, float hi) { __stcs(reinterpret_cast<float2*>(p), make_float2(lo, hi)); }
__device__ __forceinline__ void put2(bf16* p, float lo, float hi) { __stcs(reinterpret_cast<uint32_t*>(p), pack(lo, hi)); }

// Where x c - m c may be taken as one multiply-add of x: t is as good as its own rounding, and m c is off by `rest`, less than 2^-4.
__device__ __forceinline__ bool is_plain(float m, float c) { return fabsf(m) < 1e28f && fabsf(m * c) < 1048576.f && c > 1e-20f && c < 1e8f; }
// 2^-rest
__device__ __forceinline__ float less(float rest) {
    const float y = rest * -LN2;
    return fmaf(y, fmaf(y, fmaf(y, 1.f / 6, 0.5f), 1.f), 1.f);
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

// ln z of a normal z, within 2^-22 and its own rounding: the power of two apart, so that lg2 has its absolute error.
__device__ __forceinline__ float ln(float z) {
    const uint32_t b = __float_as_uint(z);
    // (zero, infinities and NaN as lg2 has them)
    const int k = b - 0x00800000u < 0x7f000000u ? (int)(b >> 23) - 127 : 0;
    return LN2 * ((float)k + lg2(__uint_as_float(b - ((uint32_t)k << 23))));
}

// log(1 + s), s in 0..1, to its own last digits: 2 (u + u^3 / 3 + u^5 / 5 ...) with u = s / (2 + s), which leaves 1e-8 of it behind u^15.
__device__ __forceinline__ float log1p_of(float s) {
    const float u = __fdividef(s, 2.f + s), u2 = u * u;
    float f = 1.f / 15;
#pragma unroll
    for (int i = 13; i > 0; i -= 2) f = fmaf(f, u2, 1.f / i);
    return 2.f * u * f;
}

// e^d - 1 - d: by series where |d| < 3/4, whose next terms are below 7e-7 of it.
__device__ __forceinline__ float exp_excess(float d) {
    if (fabsf(d) < 0.75f) {
        const float d2 = d * d, even = fmaf(d2, fmaf(d2, fmaf(d2, 1.f / 40320, 1.f / 720), 1.f / 24), 0.5f);
        return d2 * fmaf(d, fmaf(d2, fmaf(d2, 1.f / 5040, 1.f / 120), 1.f / 6), even);
    }
    const float e = ex2(d * LOG2E);
    return d > 40.f ? e : e - 1.f - d;
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
    const float A = row.A, r = !a.old_logp || l == row.old ? (l == l ? 1.f : l) : ex2((l - row.old) * LOG2E);
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

// each_group with a count of turns that all lanes share: where lanes differ in it, an unrolled loop runs its rest beside its last turn
// (rows of 24001 bf16 took 15 turns' instructions for 12).
template <int G, int WARPS, typename F>
__device__ __forceinline__ void each_of(const Part<G, WARPS>& p, F&& f) {
    const int lane = threadIdx.x & 31, inner = p.inner(), outer = p.outer();
    int j = inner + lane;
#pragma unroll 4
    for (int left = (outer - inner) >> 5; left > 0; --left, j += 32) f(j, std::true_type());
    if (j < outer) f(j, std::true_type());
    // of the others, at most two hold some of the row: one in front, one behind
    if (inner > p.j0 && lane == 0) f(inner - 1, std::false_type());
    if (outer < p.j1 && lane == 1) f(outer, std::false_type());
}

// What a warp makes of a row's sums for its gradient.
struct TokenCoefs {
    int way;               // 0: k0, k1 as below; 1: the factors one by one; 2: no gradient
    float mc, k0, k1;      // others: 2^t (k0 + k1 t), t = x c - mc
    float token;           // the token's gradient
    float m, K, A, B, base, scale;  // one by one: q = K 2^((x - m) c), scale q (B (ln2 t + base) - A)
};

template <typename T, bool ENT, bool GRAD, int THREADS, int PER_SM>
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
    const auto part_of = [&](const T* x) { return Part<G, WARPS>(phase_of(x), n, wid); };
    const int64_t stride = (int64_t)step * a.ld;
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
        bool fetched = t1 < 0;
        const int lo = p.first() - p.P, hi = p.last() - p.P;  // the warp's entries of the slice
        const bool first = rank == 0 && threadIdx.x == 0;
        // Groups that are read for the last time make place for those of the next row: f(j, whole) of the warp's groups, and the copies.
        const auto each_then_next = [&](auto&& f) {
            const int inner = p1.inner(), count = fetched ? 0 : p1.outer() - inner;
            const T* base = x1 - p1.P;
            each_of(p, [&](int j, auto whole) {
                f(j, whole);
                if ((unsigned)(j - inner) < (unsigned)count) cp_async16(ss + j * G, base + j * G);
            });
            if (!fetched) {
                __syncwarp();
                // (at another place behind 16 bytes a part may have groups that this one had not)
                const int from = p.inner() - (p.inner() > p.j0), to = p.outer() + (p.outer() < p.j1);
                for (int j = inner + lane; j < min(inner + count, from); j += 32) cp_async16(ss + j * G, base + j * G);
                for (int j = max(inner, to) + lane; j < inner + count; j += 32) cp_async16(ss + j * G, base + j * G);
                stage_ends(ss, x1, p1);
                fetched = true;
            }
        };
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
                const float mc = v.m * c;
                const f32x2 o = both(-mc), c2 = both(c);
                f32x2 z = both(0.f), w = z;
                const auto add = [&](int j) {
                    read<ENT>(ss + j * G, x);
#pragma unroll
                    for (int i = 0; i < G; i += 2) {
                        const f32x2 e = fma2(both(x[i], x[i + 1]), c2, o), q = ex2(e);
                        z = add2(z, q);
                        if constexpr (ENT) w = fma2(q, e, w);
                    }
                };
                // (one order of the sums, whatever is asked for)
                if constexpr (!GRAD)
                    each_then_next([&](int j, auto) { add(j); });
                else
                    each_of(p, [&](int j, auto) { add(j); });
                const float rest = fmaf(v.m, c, -mc), f = less(rest);
                v.z = sum_of_warp(sum2(z)) * f;
                if (ENT) v.a = fmaf(-rest, v.z, sum_of_warp(sum2(w)) * f);
            }
            if (!(v.z < 1e12f && v.z > 0.f && is_plain(v.m, c))) {
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
            posted(a.ctas);
            parity ^= 1;
            TokenCoefs k;
            if (GRAD || wid == 0) {  // (each warp for itself: one for all, and a barrier, cost 16384 rows of 16384 365 us in place of 351)
                v = collect_sums<ENT>(slots + (parity ^ 1) * places, places, c);
                const bool empty = v.z == 0.f && xt == -INFINITY;
                // (an infinite logit: NaN)
                const float lz = ln(v.z), D = xt < INFINITY ? fmaf(v.m - xt, inv_tau, lz) : NAN, s = ex2(-fabsf(D) * LOG2E);
                // masses of the others and of the token
                const float share = __fdividef(1.f, 1.f + s), qo = D > 0.f ? share : s * share, qt = D > 0.f ? s * share : share;
                const float near = log1p_of(s), l = -(near + fmaxf(D, 0.f));
                const float Lk = lz + (near + fmaxf(-D, 0.f));  // log q_v = ln2 t_v - Lk
                float H = 0.f;
                if (ENT) H = (v.z == 0.f || qo == 0.f ? 0.f : qo * (Lk - LN2 * __fdividef(v.a, v.z))) - (qt == 0.f ? 0.f : qt * l);
                float2 f = {0.f, 0.f};
                if (a.advantage) f = policy(a, terms, l);
                if (first) {
                    int64_t place = row;
                    if (a.at) {
                        const int2 at = __ldg(a.at + row);
                        place = (int64_t)at.x * a.T + at.y;
                    }
                    if (a.loss) a.loss[row] = empty ? 0.f : a.bonus != 0.f ? fmaf(-a.bonus, H, f.x) : f.x;
                    if (a.logp) a.logp[place] = empty ? -INFINITY : l == 0.f ? 0.f : l;
                    if (ENT && a.entropy) a.entropy[place] = empty ? 0.f : H;
                }
                if constexpr (GRAD) {
                    k.scale = terms.weight * inv_tau, k.A = a.d_logp ? terms.d_logp : f.y, k.B = a.d_entropy ? -terms.d_entropy : a.bonus;
                    k.m = v.m, k.mc = v.m * c, k.K = __fdividef(qo, v.z), k.base = H - Lk;
                    const float rest = fmaf(v.m, c, -k.mc), f1 = less(rest);
                    const float k0 = k.scale * k.K * (ENT ? fmaf(k.B, k.base, -k.A) : -k.A), k1 = ENT ? k.scale * k.K * k.B * LN2 : 0.f;
                    k.k0 = fmaf(-k1, rest, k0) * f1, k.k1 = k1 * f1;
                    float d = k.A * qo;
                    if (ENT) d += k.B * (qt == 0.f ? 0.f : qt * (l + H));
                    k.token = empty ? 0.f : k.scale * d;
                    // (NaN passes)
                    k.way = empty || (v.z == 0.f && xt < INFINITY) ? 2 : fabsf(k0) + fabsf(k1) < 1e30f && is_plain(v.m, c) ? 0 : 1;
                }
            }
            if constexpr (GRAD) {
                const int Pg = phase_of(g);  // the gradient is written wide, whatever the others' alignment
                if (k.way == 2) {
                    put_zeros(g, lo, hi);
                } else if (k.way == 1) {
                    for (int e = lo + lane; e < hi; e += 32) {
                        const float u = held((to_f<T>(ss[p.P + e]) - k.m) * c), q = ex2(u) * k.K;
                        const float m = ENT ? fmaf(k.B, fmaf(LN2, u, k.base), -k.A) : -k.A;
                        g[e] = from_f<T>(q == 0.f ? 0.f : q * m * k.scale);
                    }
                } else {
                    const f32x2 o = both(-k.mc), c2 = both(c), K0 = both(k.k0), K1 = both(k.k1);
                    const auto of = [&](f32x2 x) {
                        const f32x2 u = fma2(x, c2, o);
                        return mul2(ex2(u), ENT ? fma2(K1, u, K0) : K0);
                    };
                    if (p.P == Pg) {
                        T* out = g - p.P;
                        each_then_next([&](int j, auto whole) {
                            float x[G];
                            read<ENT>(ss + j * G, x);
#pragma unroll
                            for (int i = 0; i < G; i += 2) split(of(both(x[i], x[i + 1])), x[i], x[i + 1]);
                            if constexpr (decltype(whole)::value)
                                put<G>(out + j * G, x);
                            else
                                put_at<T, G>(g, j * G - p.P, 0, n, x);
                        });
                    } else {  // two entries a lane: neighbours in the gradient, in order in shared memory
                        for (int e = (lo + Pg) / 2 * 2 - Pg + lane * 2; e < hi; e += 64) {
                            float x0 = to_f<T>(ss[p.P + max(e, lo)]), x1 = to_f<T>(ss[p.P + min(e + 1, hi - 1)]);
                            if (ENT) x0 = above(x0), x1 = above(x1);
                            split(of(both(x0, x1)), x0, x1);
                            if (e >= lo && e + 1 < hi) {
                                put2(g + e, x0, x1);
                            } else {
                                if (e >= lo) g[e] = from_f<T>(x0);
                                if (e + 1 < hi) g[e + 1] = from_f<T>(x1);
                            }
                        }
                    }
                }
                __syncwarp();  // the token's place was written above
                if (mine >= 0 && lane == 0) g[mine] = from_f<T>(k.token);
            }
        }
        __syncwarp();  // the warp's part is done
        if (!fetched) stage_part(ss, x1, p1);
        t = t1, t1 = t2, xt = xt1, x0 = x1, p = p1;
    }
}

template <typename T, bool ENT, bool GRAD>
cudaError_t run_token(const TokenArgs& a, Stream& s) {
    const auto bytes = [&](int threads) { return (a.slice + 16) * sizeof(T) + 2 * threads / 32 * a.ctas * sizeof(TokenSums); };
    const auto fit = [&](int threads) { return (int)(227 * 1024 / (bytes(threads) + 1024 + 128)); };  // (1 KB is the system's)
    const auto run = [&](auto threads, auto lanes) {
        constexpr int THREADS = decltype(threads)::value, PER_SM = std::min(32, decltype(lanes)::value / THREADS);
        const size_t smem = bytes(THREADS);
        cudaError_t e = allow_row_smem<k_token<T, ENT, GRAD, THREADS, PER_SM>>();
        if (e != cudaSuccess) return e;
        int clusters = 0;
        e = resident_clusters<k_token<T, ENT, GRAD, THREADS, PER_SM>>(a.ctas, THREADS, std::max(1, std::min(PER_SM, fit(THREADS))), smem, a.rows, &clusters);
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_token<T, ENT, GRAD, THREADS, PER_SM>, dim3((unsigned)clusters * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    };
    // Threads of a CTA: what a warp does once a row is a good part of its work, so that fewer warps are faster as long as an SM has 24 of
    // them, which is what 80 registers leave room for, beside the rows that its shared memory holds (8192 rows of 16384 fp32 on 512, 256 and
    // 128 threads: 121, 90 and 94 us; with gradients in bf16 134, 109 and 126).
    constexpr std::integral_constant<int, 768> full;
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
    if (a.grad) return entropy ? run_token<T, true, true>(a, s) : run_token<T, false, true>(a, s);
    return entropy ? run_token<T, true, false>(a, s) : run_token<T, false, false>(a, s);
}

}  // namespace

cudaError_t launch_token(const TokenArgs& args, int rows, int dtype, Stream& s) {
    TokenArgs a = args;
    const RowSplit sp = split_row(rows, a.V, dtype ? 2 : 4, device_sm_count(), SHARED_SM, true);
    a.rows = rows, a.ctas = sp.ctas, a.slice = sp.slice;
    const bool entropy = a.entropy || a.d_entropy || a.bonus != 0.f;
    return dtype ? run_token<bf16>(a, entropy, s) : run_token<float>(a, entropy, s);
}

}  // namespace hbsjd
