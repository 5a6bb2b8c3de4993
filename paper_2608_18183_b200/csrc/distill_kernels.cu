// Divergence of a student's rows of logits from a teacher's and its gradient, in one pass over memory.
//
// With x = s / tau, y = t / tau, q = softmax(x), p = softmax(y), d = x - y and delta = log sum e^x - log sum e^y:
//   KL(p || q) = delta - E_p d,    KL(q || p) = E_q d - delta,
//   d KL(p || q) / dx = q - p,     d KL(q || p) / dx = q (d - E_q d),
// so four sums over the row (two of exponentials, two weighted by d) give the loss, and a second look at the row the gradient.  The row stays in shared memory between the two: it is read from HBM once, the gradient written once, and
// those 12 V bytes (two fp32 rows) are what bounds the kernel.  Rows that a CTA cannot hold beside others are split over a
// cluster, whose CTAs exchange the sums through distributed shared memory; so are few rows, to use more SMs.
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

template <typename TS, typename TT, int THREADS>
__global__ void __launch_bounds__(THREADS) k_distill(DistillArgs a) {
    constexpr int G = sizeof(TS) == 2 && sizeof(TT) == 2 ? 8 : 4;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Slots<Pair, THREADS> slots;
    __shared__ int special;  // a logit of the slice asks for care
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / a.ctas;
    const int rank = blockIdx.x % a.ctas, v0 = rank * a.slice, n = max(0, min(a.slice, a.V - v0));
    const float w = a.weight ? a.weight[row] : 1.f;
    TS* g = a.grad ? (TS*)a.grad + row * a.ld_g + v0 : nullptr;
    if (w == 0.f) {  // the whole cluster leaves the row out
        if (g) put_zeros<TS, THREADS>(g, n);
        if (a.loss && rank == 0 && tid == 0) a.loss[row] = 0.f;
        return;
    }
    if (a.ctas > 1) cluster_arrive();
    const TS* s = (const TS*)a.s + row * a.ld_s + v0;
    const TT* t = (const TT*)a.t + row * a.ld_t + v0;
    const int P = common_phase(s, t), groups = (P + n + G - 1) / G;
    TS* ss = (TS*)smem;
    TT* st = (TT*)(smem + (a.slice + 16) * sizeof(TS));
    stage_row<TS, G, THREADS>(ss, s, n, P, PAD);
    stage_row<TT, G, THREADS>(st, t, n, P, PAD);
    if (tid == 0) special = 0;
    cp_async_wait_all();
    __syncthreads();

    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    // A warp sums against the largest logits of its first groups.  That overflows, or meets what has no finite difference, in few
    // rows; their warps find their maxima and look at every entry.
    Pair v = Pair::none();
    {
        float x[G], y[G];
        if (tid < groups) {
            get<G>(ss + tid * G, x);
            get<G>(st + tid * G, y);
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (tid * G + i >= P && tid * G + i < P + n) v.ms = fmaxf(v.ms, x[i]), v.mt = fmaxf(v.mt, y[i]);
        }
        v.share();
        const f32x2 os = both(-v.ms), ot = both(-v.mt), c2 = both(c), minus = both(-1.f);
        f32x2 zs = both(0.f), zt = zs, as = zs, at = zs;
        for (int j = tid; j < groups; j += THREADS) {
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
        v.zs = sum_of_warp(sum2(zs));
        v.zt = sum_of_warp(sum2(zt));
        v.as = sum_of_warp(sum2(as));
        v.at = sum_of_warp(sum2(at));
    }
    // (false for NaN, infinities, and sums that a factor could not bring down again)
    if (!(v.zs < 1e12f && v.zs > 0.f && v.zt < 1e12f && v.zt > 0.f && fabsf(v.as) < 1e30f && fabsf(v.at) < 1e30f)) {
        const bool any = (tid & ~31) < groups;
        if (any) special = 1;
        v = Pair::none();
        for (int j = tid; j < groups; j += THREADS)
            for (int e = max(j * G, P); e < min(j * G + G, P + n); ++e)
                v.ms = fmaxf(v.ms, to_f<TS>(ss[e])), v.mt = fmaxf(v.mt, to_f<TT>(st[e]));
        v.share();
        const float os = v.ms == -INFINITY ? 0.f : v.ms, ot = v.mt == -INFINITY ? 0.f : v.mt;
        for (int j = tid; j < groups; j += THREADS)
            for (int e = max(j * G, P); e < min(j * G + G, P + n); ++e) {
                // (x - m before the product: a row of the lowest finite value is uniform)
                const float xo = to_f<TS>(ss[e]) - os, yo = to_f<TT>(st[e]) - ot, es = ex2(xo * c), et = ex2(yo * c);
                v.zs += es;
                v.zt += et;
                // no mass, no share: d is infinite or NaN where one or both are masked
                v.as += es == 0.f ? 0.f : es * (xo - yo);
                v.at += et == 0.f ? 0.f : et * (xo - yo);
            }
        v.zs = sum_of_warp(v.zs);
        v.zt = sum_of_warp(v.zt);
        v.as = sum_of_warp(v.as);
        v.at = sum_of_warp(v.at);
    }
    if (a.ctas > 1) cluster_wait();  // every CTA of the row runs
    post(v, slots, a.ctas);
    posted(a.ctas);
    v = collect(slots, a.ctas, c);
    const bool empty = v.zs == 0.f || v.zt == 0.f;
    // (against the maxima: their difference is in neither d nor delta)
    const float A_q = v.as / v.zs * inv_tau, A_p = v.at / v.zt * inv_tau, ls = log2f(v.zs), lt = log2f(v.zt);
    if (a.loss && rank == 0 && tid == 0) {
        float loss = 0.f;
        if (!empty) {
            if (a.forward != 0.f) loss -= a.forward * A_p;
            if (a.reverse != 0.f) loss += a.reverse * A_q;
            if (a.forward != a.reverse) loss += (a.forward - a.reverse) * (LN2 * (ls - lt));
        }
        a.loss[row] = loss;
    }
    if (!g) return;
    if (empty) {
        put_zeros<TS, THREADS>(g, n);
        return;
    }
    // w / tau (a (q - p) + b q (d - E_q d)) = q (k0 + k1 d) - k2 p
    const float f = w * inv_tau;
    const bool rev = a.reverse != 0.f;
    const float k0 = f * (rev ? a.forward - a.reverse * A_q : a.forward), k1 = f * a.reverse * inv_tau, k2 = f * a.forward;
    const int Pg = phase_of(g) % G;  // the gradient is written wide, whatever the others' alignment
    const bool wide = P % G == Pg;
    if (special) {
        for (int e = tid; e < n; e += THREADS) {
            const float xo = to_f<TS>(ss[P + e]) - v.ms, yo = to_f<TT>(st[P + e]) - v.mt;
            const float q = ex2(fmaf(xo, c, -ls)), p = ex2(fmaf(yo, c, -lt)), k = rev ? fmaf(k1, xo - yo, k0) : k0;
            g[e] = from_f<TS>(fmaf(-k2, p, q == 0.f ? 0.f : q * k));
        }
        return;
    }
    const f32x2 os = both(-v.ms), ot = both(-v.mt), c2 = both(c), minus = both(-1.f), nls = both(-ls), nlt = both(-lt);
    const f32x2 K0 = both(k0), K1 = both(k1), K2 = both(-k2);
    for (int e = tid * G - Pg; e < n; e += THREADS * G) {
        float x[G], y[G];
        get_at<TS, G>(ss, P, e, n, wide, x);
        get_at<TT, G>(st, P, e, n, wide, y);
#pragma unroll
        for (int i = 0; i < G; i += 2) {
            const f32x2 xo = add2(both(x[i], x[i + 1]), os), yo = add2(both(y[i], y[i + 1]), ot);
            const f32x2 q = ex2(fma2(xo, c2, nls)), p = ex2(fma2(yo, c2, nlt)), k = fma2(K1, fma2(yo, minus, xo), K0);
            split(fma2(K2, p, mul2(q, k)), x[i], x[i + 1]);
        }
        put_at<TS, G>(g, e, n, x);
    }
}

// log(e^x + e^y); -inf for none, NaN passes.
__device__ __forceinline__ float log_add(float x, float y) {
    const float m = fmaxf(x, y);
    return m == -INFINITY ? x + y : fmaf(LN2, log2f(ex2((x - m) * LOG2E) + ex2((y - m) * LOG2E)), m);
}

template <typename TS, int THREADS>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) k_distill_topk(DistillArgs a) {
    constexpr int G = 16 / sizeof(TS);
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Slots<Pair, THREADS> slots;
    __shared__ Slots<Mass, THREADS> slots_other;
    __shared__ int repeated;
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, k = a.k;
    const int64_t row = blockIdx.x / a.ctas;
    const int rank = blockIdx.x % a.ctas, v0 = rank * a.slice, n = max(0, min(a.slice, a.V - v0));
    const float w = a.weight ? a.weight[row] : 1.f;
    TS* g = a.grad ? (TS*)a.grad + row * a.ld_g + v0 : nullptr;
    if (w == 0.f) {  // the whole cluster leaves the row out
        if (g) put_zeros<TS, THREADS>(g, n);
        if (a.loss && rank == 0 && tid == 0) a.loss[row] = 0.f;
        return;
    }
    if (a.ctas > 1) cluster_arrive();
    const TS* s = (const TS*)a.s + row * a.ld_s + v0;
    const int P = phase_of(s), groups = (P + n + G - 1) / G;
    TS* ss = (TS*)smem;
    float* xk = (float*)(smem + (a.slice + 16) * sizeof(TS));  // [k] the student's logit of a listed token of the slice
    int32_t* at = (int32_t*)(xk + k);                          // [k] its place in the slice, -1: not here
    uint32_t* seen = (uint32_t*)(at + k);                      // a bit per element of the slice
    stage_row<TS, G, THREADS>(ss, s, n, P, PAD);

    // while the row is on its way: which entries lie in the slice, and is a token listed twice (the first entry counts)
    const float* val = a.values + row * k;
    if (tid == 0) repeated = 0;
    for (int i = tid; i < (a.slice + 31) / 32; i += THREADS) seen[i] = 0;
    __syncthreads();
    for (int i = tid; i < k; i += THREADS) {
        const int32_t idx = a.indices[row * k + i];
        int e = -1;
        if (idx >= v0 && idx < v0 + n && !(val[i] == -INFINITY)) {
            e = idx - v0;
            if (atomicOr(&seen[e >> 5], 1u << (e & 31)) >> (e & 31) & 1) repeated = 1;
        }
        at[i] = e;
    }
    cp_async_wait_all();
    __syncthreads();
    if (repeated) {
        for (int i0 = 0; i0 < k; i0 += THREADS) {
            const int i = i0 + tid;
            bool again = false;
            if (i < k && at[i] >= 0)
                for (int j = 0; j < i && !again; ++j) again = at[j] == at[i];
            __syncthreads();  // (entries behind this block of them look at it before it changes, entries in it too)
            if (again) at[i] = -2 - at[i];
            __syncthreads();
        }
    }
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    // listed tokens leave the slice; v: their sums, student and teacher (warps without any have none)
    Pair v = Pair::none();
    const bool lists = (tid & ~31) < k;
    if (lists) {
        for (int i = tid; i < k; i += THREADS)
            if (at[i] >= 0) {
                const float x = to_f<TS>(ss[P + at[i]]);
                xk[i] = x;
                ss[P + at[i]] = from_f<TS>(-INFINITY);
                v.ms = fmaxf(v.ms, x);
                v.mt = fmaxf(v.mt, val[i]);
            }
        v.share();
        const float os = v.ms == -INFINITY ? 0.f : v.ms, ot = v.mt == -INFINITY ? 0.f : v.mt;
        for (int i = tid; i < k; i += THREADS)
            if (at[i] >= 0) {
                const float xo = xk[i] - os, yo = val[i] - ot, es = ex2(xo * c), et = ex2(yo * c);
                v.zs += es;
                v.zt += et;
                v.as += es == 0.f ? 0.f : es * (xo - yo);
                v.at += et == 0.f ? 0.f : et * (xo - yo);
            }
        v.zs = sum_of_warp(v.zs);
        v.zt = sum_of_warp(v.zt);
        v.as = sum_of_warp(v.as);
        v.at = sum_of_warp(v.at);
    }
    __syncthreads();
    // u: all other tokens, against the largest of a warp's first groups; where that overflows or leaves nothing, of all of its
    Mass u = Mass::none();
    {
        float x[G];
        if (tid < groups) {
            get<G>(ss + tid * G, x);
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (tid * G + i >= P && tid * G + i < P + n) u.m = fmaxf(u.m, x[i]);
        }
        u.share();
        const f32x2 o = both(-u.m), c2 = both(c);
        f32x2 z = both(0.f);
        for (int j = tid; j < groups; j += THREADS) {
            get<G>(ss + j * G, x);
#pragma unroll
            for (int i = 0; i < G; i += 2) z = add2(z, ex2(mul2(add2(both(x[i], x[i + 1]), o), c2)));
        }
        u.z = sum_of_warp(sum2(z));
    }
    if (!(u.z < 1e12f && u.z > 0.f)) {
        u = Mass::none();
        for (int j = tid; j < groups; j += THREADS)
            for (int e = max(j * G, P); e < min(j * G + G, P + n); ++e) u.m = fmaxf(u.m, to_f<TS>(ss[e]));
        u.share();
        const float o = u.m == -INFINITY ? 0.f : u.m;
        for (int j = tid; j < groups; j += THREADS)
            for (int e = max(j * G, P); e < min(j * G + G, P + n); ++e) u.z += ex2((to_f<TS>(ss[e]) - o) * c);
        u.z = sum_of_warp(u.z);
    }
    if (a.ctas > 1) cluster_wait();  // every CTA of the row runs
    post(v, slots, a.ctas);
    post(u, slots_other, a.ctas);
    posted(a.ctas);
    v = collect(slots, a.ctas, c);
    u = collect(slots_other, a.ctas, c);

    // Logarithms of the masses of the listed tokens (l) and the others (o), student (x) and teacher (y), against the largest
    // logit of each: rows of the lowest finite value have some too.
    const float yr = a.rest ? a.rest[row] : -INFINITY;
    const bool empty = (v.zs == 0.f && u.z == 0.f) || (v.zt == 0.f && yr == -INFINITY);
    const float Mx = fmaxf(v.ms, u.m), My = v.mt == -INFINITY ? 0.f : v.mt;
    const float xl = v.zs == 0.f ? -INFINITY : fmaf(v.ms - Mx, inv_tau, LN2 * log2f(v.zs));
    const float xo = u.z == 0.f ? -INFINITY : fmaf(u.m - Mx, inv_tau, LN2 * log2f(u.z));
    const float yl = v.zt == 0.f ? -INFINITY : LN2 * log2f(v.zt), yo = yr == -INFINITY ? yr : fmaf(-My, inv_tau, yr);
    const float Lx = log_add(xl, xo), Ly = log_add(yl, yo);
    const float ql = ex2((xl - Lx) * LOG2E), qo = ex2((xo - Lx) * LOG2E);
    const float pl = ex2((yl - Ly) * LOG2E), po = ex2((yo - Ly) * LOG2E);
    const float lo = (xo - Lx) - (yo - Ly);                     // log of qo / po
    // a mass of zero adds nothing, whatever its logarithm is (NaN passes)
    float kl_pq = 0.f, kl_qp = 0.f;
    const float shift = v.ms == -INFINITY ? 0.f : Mx - v.ms;  // (the sums of d are against v.ms)
    if (pl != 0.f) kl_pq -= pl * ((v.at / v.zt - shift) * inv_tau - (Lx - Ly));
    if (po != 0.f) kl_pq -= po * lo;
    if (ql != 0.f) kl_qp += ql * ((v.as / v.zs - shift) * inv_tau - (Lx - Ly));
    if (qo != 0.f) kl_qp += qo * lo;
    if (a.loss && rank == 0 && tid == 0) {
        float loss = 0.f;
        if (!empty) {
            if (a.forward != 0.f) loss += a.forward * kl_pq;
            if (a.reverse != 0.f) loss += a.reverse * kl_qp;
        }
        a.loss[row] = loss;
    }
    if (!g) return;
    if (empty) {
        put_zeros<TS, THREADS>(g, n);
        return;
    }
    const float f = w * inv_tau;
    // others: q_v (a (1 - po / qo) + b (lo - KL(q || p))), with q_v / qo their share of u.z
    float k0 = a.forward * (qo - po);
    if (a.reverse != 0.f && qo != 0.f) k0 += a.reverse * qo * (lo - kl_qp);
    k0 = u.z == 0.f ? 0.f : k0 * f / u.z;
    const float om = u.m == -INFINITY ? 0.f : u.m;
    const int Pg = phase_of(g);  // the gradient is written wide, whatever the others' alignment
    const f32x2 o = both(-om), c2 = both(c), K0 = both(k0);
    for (int e = tid * G - Pg; e < n; e += THREADS * G) {
        float x[G];
        get_at<TS, G>(ss, P, e, n, P == Pg, x);
#pragma unroll
        for (int i = 0; i < G; i += 2) split(mul2(ex2(mul2(add2(both(x[i], x[i + 1]), o), c2)), K0), x[i], x[i + 1]);
        put_at<TS, G>(g, e, n, x);
    }
    __syncthreads();  // the listed tokens' places were written above
    for (int i = tid; i < k; i += THREADS)
        if (at[i] >= 0) {
            const float x = xk[i], y = val[i];
            const float q = ex2(fmaf(x - Mx, c, -Lx * LOG2E)), p = ex2(fmaf(y - My, c, -Ly * LOG2E));
            float d = a.forward * (q - p);
            if (a.reverse != 0.f && q != 0.f) d += a.reverse * q * (((x - Mx) - (y - My)) * inv_tau - (Lx - Ly) - kl_qp);
            g[at[i]] = from_f<TS>(f * d);
        }
}

// Threads of a CTA: at least eight groups each, 128 to 512.
template <typename F>
cudaError_t by_threads(int slice, int G, F&& f) {
    if (slice <= 8 * 128 * G) return f(std::integral_constant<int, 128>());
    if (slice <= 8 * 256 * G) return f(std::integral_constant<int, 256>());
    return f(std::integral_constant<int, 512>());
}

template <typename TS, typename TT>
cudaError_t run_distill(const DistillArgs& a, int rows, Stream& s) {
    constexpr int G = sizeof(TS) == 2 && sizeof(TT) == 2 ? 8 : 4;
    return by_threads(a.slice, G, [&](auto threads) {
        constexpr int THREADS = decltype(threads)::value;
        const size_t smem = (a.slice + 16) * (sizeof(TS) + sizeof(TT));
        const cudaError_t e = allow_row_smem<k_distill<TS, TT, THREADS>>();
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_distill<TS, TT, THREADS>, dim3((unsigned)rows * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    });
}

template <typename TS>
cudaError_t run_distill_topk(const DistillArgs& a, int rows, Stream& s) {
    return by_threads(a.slice, 16 / sizeof(TS), [&](auto threads) {
        constexpr int THREADS = decltype(threads)::value;
        const size_t smem = (a.slice + 16) * sizeof(TS) + a.k * 8 + (a.slice + 31) / 32 * 4;
        const cudaError_t e = allow_row_smem<k_distill_topk<TS, THREADS>>();
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_distill_topk<TS, THREADS>, dim3((unsigned)rows * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    });
}

}  // namespace

cudaError_t launch_distill(const DistillArgs& args, int rows, int dtype_s, int dtype_t, Stream& s) {
    DistillArgs a = args;
    const RowSplit sp = split_row(rows, a.V, (dtype_s ? 2 : 4) + (dtype_t ? 2 : 4), device_sm_count());
    a.ctas = sp.ctas, a.slice = sp.slice;
    if (dtype_s) return dtype_t ? run_distill<bf16, bf16>(a, rows, s) : run_distill<bf16, float>(a, rows, s);
    return dtype_t ? run_distill<float, bf16>(a, rows, s) : run_distill<float, float>(a, rows, s);
}

cudaError_t launch_distill_topk(const DistillArgs& args, int rows, int dtype_s, Stream& s) {
    DistillArgs a = args;
    const RowSplit sp = split_row(rows, a.V, dtype_s ? 2 : 4, device_sm_count());
    a.ctas = sp.ctas, a.slice = sp.slice;
    return dtype_s ? run_distill_topk<bf16>(a, rows, s) : run_distill_topk<float>(a, rows, s);
}

}  // namespace hbsjd
