// What the operators on rows and their tokens have in common: a warp's sums over its part of a staged row without the row's token, what
// the sums say of the token, and the part's gradient.
//
// With x = logits / tau, q = softmax(x), t the row's token and o all others:
//   D = log sum_o e^x - x_t,   l = log q_t = -log(1 + e^D),   sum_o q = 1 / (1 + e^-D),
//   H = -sum q log q,          d (a l + b H) / dx_v = a (1[v = t] - q_v) - b q_v (log q_v + H).
// The token leaves the row before the row is summed, so that neither l nor 1 - q_t is a difference of near numbers: a token of almost
// all the mass has digits in both.
#pragma once
#include "logit_rows.cuh"

namespace hbsjd {

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

// Where x c - m c may be taken as one multiply-add of x: t is as good as its own rounding, and m c is off by `rest`, less than 2^-4.
__device__ __forceinline__ bool is_plain(float m, float c) { return fabsf(m) < 1e28f && fabsf(m * c) < 1048576.f && c > 1e-20f && c < 1e8f; }
// 2^-rest
__device__ __forceinline__ float less(float rest) {
    const float y = rest * -LN2;
    return fmaf(y, fmaf(y, fmaf(y, 1.f / 6, 0.5f), 1.f), 1.f);
}

// ln z of a normal z as a sum of two: the power of two apart, so that lg2 has its absolute error of 2^-22.
__device__ __forceinline__ float2 ln(float z) {
    const uint32_t b = __float_as_uint(z);
    // (zero, infinities and NaN as lg2 has them)
    const int k = b - 0x00800000u < 0x7f000000u ? (int)(b >> 23) - 127 : 0;
    const float f = LN2 * lg2(__uint_as_float(b - ((uint32_t)k << 23))), hi = (float)k * LN2;
    return {hi, f + fmaf((float)k, LN2, -hi) - (float)k * 1.90465e-9f};  // (LN2 is that much above ln 2)
}
// The same for sums over many rows, where what all rows are off alike adds up (lg2 leaves up to 2e-8 a row, by its argument): z = 2^k f with
// f in [sqrt 1/2, sqrt 2), and ln f = 2 (u + u^3 / 3 + u^5 / 5 ...) with u = (f - 1) / (f + 1), which leaves 1e-9 behind u^9.
__device__ __forceinline__ float2 ln_without_lean(float z) {
    const int b = __float_as_int(z);
    if ((uint32_t)(b - 0x00800000) >= 0x7f000000u) return ln(z);  // zero, infinities and NaN
    const int k = (b - 0x3f3504f3) >> 23;  // (sqrt 1/2)
    const float f = __int_as_float(b - (k << 23)), u = __fdividef(f - 1.f, f + 1.f), u2 = u * u;
    const float g = 2.f * u * fmaf(u2, fmaf(u2, fmaf(u2, fmaf(u2, 1.f / 9, 1.f / 7), 0.2f), 1.f / 3), 1.f), hi = (float)k * LN2;
    return {hi, g + (fmaf((float)k, LN2, -hi) - (float)k * 1.90465e-9f)};
}
// rescale for such sums.  ex2 is exact at whole numbers and 5e-8 below 2^x on average elsewhere: sums that are brought from a warp's reference to
// the row's, or from a tile's, would lean by as much each time.  2^p = 2^i e^y with |y| <= ln2 / 2; the series leaves 5e-9 behind y^7.
// (What is left of it is in the entries: l is up to 5e-8 times the others' mass too high on average, and the rounding of c, at a temperature of 1 1.3e-8
// of their mean distance from the largest, takes from that.  Of 2 to 131072 normal logits with a deviation of 0.1 to 10: a mean of -3e-8 to 3e-8
// a row; where all others are alike, none.)
__device__ __forceinline__ float rescale_without_lean(float from, float to, float c) {
    if (from == -INFINITY) return 0.f;
    if (from == to) return 1.f;
    const float p = (from - to) * c, i = rintf(p), y = (p - i) * LN2;
    if (!(i >= -126.f)) return 0.f;
    const float e = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 5040, 1.f / 720), 1.f / 120), 1.f / 24), 1.f / 6), 0.5f), 1.f), 1.f);
    return e * __int_as_float(((int)i + 127) << 23);
}

// log(1 + s), s in 0..1, to its own last digits: 2 (u + u^3 / 3 + u^5 / 5 ...) with u = s / (2 + s), which leaves 1e-8 of it behind u^15.
__device__ __forceinline__ float log1p_of(float s) {
    const float u = __fdividef(s, 2.f + s), u2 = u * u;
    float f = 1.f / 15;
#pragma unroll
    for (int i = 13; i > 0; i -= 2) f = fmaf(f, u2, 1.f / i);
    return 2.f * u * f;
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

// A warp's sums over its part of a slice at x0, staged at ss; `mine`: the token's place in the slice, if it is one of the part's, else -1.
// walk(f) has f read every group of the part in one order.  A warp sums against the largest logit of its first groups.  That
// overflows, or leaves nothing, in few rows; their warps find their maxima and look at every entry.
template <bool ENT, typename T, int G, int WARPS, typename W>
__device__ __forceinline__ TokenSums part_sums(T* ss, const Part<G, WARPS>& p, const T* x0, int mine, float c, W&& walk) {
    const int lane = threadIdx.x & 31, lo = p.first() - p.P, hi = p.last() - p.P;
    if (mine >= 0 && lane == 0) ss[p.P + mine] = from_f<T>(-INFINITY);
    end_part(ss, p, -INFINITY);
    TokenSums v = TokenSums::none();
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
    walk([&](int j, auto) {
        read<ENT>(ss + j * G, x);
#pragma unroll
        for (int i = 0; i < G; i += 2) {
            const f32x2 e = fma2(both(x[i], x[i + 1]), c2, o), q = ex2(e);
            z = add2(z, q);
            if constexpr (ENT) w = fma2(q, e, w);
        }
    });
    const float rest = fmaf(v.m, c, -mc), f = less(rest);
    v.z = sum_of_warp(sum2(z)) * f;
    if (ENT) v.a = fmaf(-rest, v.z, sum_of_warp(sum2(w)) * f);
    if (!(v.z < 1e12f && v.z > 0.f && is_plain(v.m, c))) {
        v = TokenSums::none();
        for (int e = lo + lane; e < hi; e += 32)
            if (e != mine) v.m = fmaxf(v.m, to_f<T>(x0[e]));
        v.m = max_of_warp(v.m);
        const float base = v.m == -INFINITY ? 0.f : v.m;
        for (int e = lo + lane; e < hi; e += 32)
            if (e != mine) {
                const float s = held((to_f<T>(x0[e]) - base) * c), q = ex2(s);
                v.z += q;
                v.a = fmaf(q, s, v.a);
            }
        v.z = sum_of_warp(v.z);
        v.a = sum_of_warp(v.a);
    }
    return v;
}

// What a row's sums over the others and its token's logit say.
struct TokenRow {
    bool empty;      // nothing has mass
    bool alone;      // the token alone has
    float l, qo, qt; // log q of the token, masses of the others and of the token
    float Lk;        // log q_v = ln2 t_v - Lk
    float low;       // what l's own rounding left, if asked for
    // of what was kept of one
    __device__ __forceinline__ TokenRow(float z, float others) : empty(false), alone(z == 0.f && others == 0.f), l(0.f), qo(others), qt(0.f), Lk(0.f), low(0.f) {}
    // summed: l and low are for sums over many rows
    __device__ __forceinline__ TokenRow(const TokenSums& v, float xt, float inv_tau, bool summed) {
        empty = v.z == 0.f && xt == -INFINITY;
        alone = v.z == 0.f && xt < INFINITY;
        // (an infinite logit: NaN)
        // (D's parts are as large as l: what the rounding of their sum leaves is added before the next, so that l is about as good as its own)
        const float2 lz = summed ? ln_without_lean(v.z) : ln(v.z);
        const float gap = v.m - xt, big = fmaf(gap, inv_tau, lz.x);
        float rest = fmaf(gap, inv_tau, lz.x - big) + lz.y, D = big + lz.y;
        if (!(xt < INFINITY)) D = NAN;
        const float s = ex2(-fabsf(D) * LOG2E);
        const float share = __fdividef(1.f, 1.f + s);
        qo = D > 0.f ? share : s * share, qt = D > 0.f ? s * share : share;
        const float near = log1p_of(s);
        if (summed) {  // all that the roundings left
            const float back = gap - v.m, off = (v.m - (gap - back)) - (xt + back), p = gap * inv_tau, t = big - p;
            rest = (p - (big - t)) + (lz.x - t) + (fmaf(gap, inv_tau, -p) + off * inv_tau) + lz.y;
        }
        l = D > 0.f && D < INFINITY ? -(big + (rest + near)) : -(near + fmaxf(D, 0.f));
        low = summed && D > 0.f ? -((big + l) + (rest + near)) : 0.f;
        if (!(fabsf(low) < 1.f)) low = 0.f;
        Lk = lz.x + (lz.y + (near + fmaxf(-D, 0.f)));
    }
    __device__ __forceinline__ float logp() const { return empty ? -INFINITY : l == 0.f ? 0.f : l; }
};

// What a warp makes of a row's sums for its gradient.
struct TokenCoefs {
    int way;               // 0: k0, k1 as below; 1: the factors one by one; 2: no gradient
    float mc, k0, k1;      // others: 2^t (k0 + k1 t), t = x c - mc
    float token;           // the token's gradient
    float m, K, A, B, base, scale;  // one by one: q = K 2^((x - m) c), scale q (B (ln2 t + base) - A)
    // whether no mass times this factor is none
    __device__ __forceinline__ bool is_number(float m) const { return m == m && scale == scale; }
    // a (1[v = t] - q_v) + b q_v (log q_v + H), times scale
    template <bool ENT>
    __device__ __forceinline__ void set(const TokenRow& r, const TokenSums& v, float H, float a, float b, float s, float c) {
        A = a, B = b, scale = s, m = v.m, mc = v.m * c, K = __fdividef(r.qo, v.z), base = ENT ? H - r.Lk : 0.f;
        const float rest = fmaf(v.m, c, -mc), f = less(rest);
        const float y0 = scale * K * (ENT ? fmaf(B, base, -A) : -A), y1 = ENT ? scale * K * B * LN2 : 0.f;
        k0 = fmaf(-y1, rest, y0) * f, k1 = y1 * f;
        float d = A * r.qo;
        if (ENT) d += B * (r.qt == 0.f ? 0.f : r.qt * (r.l + H));
        token = r.empty ? 0.f : scale * d;
        // (NaN passes; masked entries have exponents of down to -1e30 c, which y1 times is to be finite beside their share of zero)
        way = r.empty || (r.alone && A == A && B == B) ? 2 : fabsf(y0) + fabsf(y1) < 1e30f && fabsf(y1) * c < 1e7f && is_plain(v.m, c) ? 0 : 1;
    }
};

// The part p1 of a slice at x1 that comes next, if there is one: groups of the part at hand that were read for the last time make place for
// it in the stage.
template <typename T, int G, int WARPS>
struct Next {
    T* ss;
    const T* x1;
    const Part<G, WARPS>& p1;
    bool more;  // one comes, and nothing of it has been fetched
    // group j was read for the last time, by this lane
    __device__ __forceinline__ void take(int j, int inner, int count) const {
        if ((unsigned)(j - inner) < (unsigned)count) cp_async16(ss + j * G, x1 - p1.P + j * G);
    }
    __device__ __forceinline__ int count() const { return more ? p1.outer() - p1.inner() : 0; }
    // all groups of p were
    __device__ __forceinline__ void taken(const Part<G, WARPS>& p) {
        if (!more) return;
        more = false;
        const int lane = threadIdx.x & 31, inner = p1.inner(), outer = p1.outer();
        const T* base = x1 - p1.P;
        __syncwarp();
        // (at another place behind 16 bytes a part may have groups that this one had not)
        const int from = p.inner() - (p.inner() > p.j0), to = p.outer() + (p.outer() < p.j1);
        for (int j = inner + lane; j < min(outer, from); j += 32) cp_async16(ss + j * G, base + j * G);
        for (int j = max(inner, to) + lane; j < outer; j += 32) cp_async16(ss + j * G, base + j * G);
        stage_ends(ss, x1, p1);
    }
};
// f(j, whole) for all groups of p, the last that reads them.  (One loop whether or not one comes next: two of them in k_token cost 8192 bf16
// rows of 16384 with entropy and gradient 115 us in place of 109.)
template <typename T, int G, int WARPS, typename F>
__device__ __forceinline__ void each_then(const Part<G, WARPS>& p, Next<T, G, WARPS>& next, F&& f) {
    const int inner = next.p1.inner(), count = next.count();
    each_of(p, [&](int j, auto whole) {
        f(j, whole);
        next.take(j, inner, count);
    });
    next.taken(p);
}

// G values as they are stored.
__device__ __forceinline__ void packed(const float (&x)[4], uint32_t (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
}
__device__ __forceinline__ void packed(const float (&x)[8], uint32_t (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack(x[2 * i], x[2 * i + 1]);
}

// Entries [lo, hi) of out by a warp, where they lie at another place behind 16 bytes than in the groups that they come in: of group j, entry
// j G - P is the first.  A lane's 16 bytes are the end of the group before its own, which the lane before it has, and the beginning of
// its own.  (Two entries a lane, one by one from shared memory: 8192 bf16 rows of 16384 with a stride of 16385, policy loss with gradient,
// 139 us; so: 123.)
template <typename T, int G>
struct Shifted {
    T* out;
    int lo, hi, first, last;  // groups [first, last] hold some of them; turns go on to group last + 1
    int Pg, back, words, half;
    uint32_t before[4];  // the lane's group of the turn before
    __device__ __forceinline__ Shifted(T* out, int lo, int hi, int P) : out(out), lo(lo), hi(hi), Pg(phase_of(out)), before{0, 0, 0, 0} {
        const int d = (P - Pg + G) % G;
        back = P < Pg, words = d * (int)sizeof(T) / 4, half = sizeof(T) == 2 && d % 2;
        first = (P + lo) / G, last = lo < hi ? (P + hi - 1) / G : first - 2;
    }
    // all lanes, each with its own group: j = first + lane, and 32 more from turn to turn
    __device__ __forceinline__ void put(int j, const uint32_t (&own)[4]) {
        const int lane = threadIdx.x & 31;
        uint32_t c[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = __shfl_sync(0xffffffffu, lane == 31 ? before[i] : own[i], (lane + 31) & 31);
            c[4 + i] = before[i] = own[i];
        }
        if (words & 2)
#pragma unroll
            for (int i = 0; i < 6; ++i) c[i] = c[i + 2];
        if (words & 1)
#pragma unroll
            for (int i = 0; i < 5; ++i) c[i] = c[i + 1];
        if (half)
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = __funnelshift_r(c[i], c[i + 1], 16);
        const int e = (j - 1 + back) * G - Pg;
        if (e >= lo && e + G <= hi) {
            __stcs(reinterpret_cast<uint4*>(out + e), make_uint4(c[0], c[1], c[2], c[3]));
        } else {
            const T* x = reinterpret_cast<const T*>(c);
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (e + i >= lo && e + i < hi) out[e + i] = x[i];
        }
    }
};

// A warp's part of the gradient at g, n entries of which are the slice's, and the place for what comes next (where no careful way was
// taken).  walk(f) has f read every group, as each_then does.
template <bool ENT, typename T, int G, int WARPS, typename W>
__device__ __forceinline__ void part_gradient(const T* ss, const Part<G, WARPS>& p, T* g, int n, int mine, const TokenCoefs& k, float c,
                                              Next<T, G, WARPS>& next, W&& walk) {
    const int lane = threadIdx.x & 31, lo = p.first() - p.P, hi = p.last() - p.P, Pg = phase_of(g);
    if (k.way == 2) {
        put_zeros(g, lo, hi);
    } else if (k.way == 1) {
        for (int e = lo + lane; e < hi; e += 32) {
            const float u = held((to_f<T>(ss[p.P + e]) - k.m) * c), q = ex2(u) * k.K;
            const float m = ENT ? fmaf(k.B, fmaf(LN2, u, k.base), -k.A) : -k.A;
            g[e] = from_f<T>(q == 0.f && k.is_number(m) ? 0.f : q * m * k.scale);
        }
    } else {
        const f32x2 o = both(-k.mc), c2 = both(c), K0 = both(k.k0), K1 = both(k.k1);
        const auto of = [&](f32x2 x) {
            const f32x2 u = fma2(x, c2, o);
            return mul2(ex2(u), ENT ? fma2(K1, u, K0) : K0);
        };
        if (p.P == Pg) {
            T* out = g - p.P;
            walk([&](int j, auto whole) {
                float x[G];
                read<ENT>(ss + j * G, x);
#pragma unroll
                for (int i = 0; i < G; i += 2) split(of(both(x[i], x[i + 1])), x[i], x[i + 1]);
                if constexpr (decltype(whole)::value)
                    put<G>(out + j * G, x);
                else
                    put_at<T, G>(g, j * G - p.P, 0, n, x);
            });
        } else {
            Shifted<T, G> to(g, lo, hi, p.P);
            const int inner = next.p1.inner(), count = next.count();
#pragma unroll 2
            for (int j0 = to.first; j0 <= to.last + 1; j0 += 32) {
                const int j = j0 + lane;
                uint32_t w[4] = {0, 0, 0, 0};
                if (j <= to.last) {
                    float x[G];
                    read<ENT>(ss + j * G, x);
#pragma unroll
                    for (int i = 0; i < G; i += 2) split(of(both(x[i], x[i + 1])), x[i], x[i + 1]);
                    packed(x, w);
                    next.take(j, inner, count);
                }
                to.put(j, w);
            }
            next.taken(p);
        }
    }
    __syncwarp();  // the token's place was written above
    if (mine >= 0 && lane == 0) g[mine] = from_f<T>(k.token);
}

}  // namespace hbsjd
