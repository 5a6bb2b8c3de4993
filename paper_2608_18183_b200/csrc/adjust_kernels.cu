// Rules on rows of logits in front of a sampler: guidance, penalties for tokens that the row's history holds, a bias and masks of
// allowed tokens, one read and one write of each logit.
//
//   x = l (or l_u + s (l_c - l_u));  n = times that v occurs in the history
//   n > 0:  x = x > 0 ? x / rho : x rho,  x -= n f + pr
//   x += bias[v];  x = -inf where the mask's bit v is 0, and where x is NaN (guidance of two masked branches)
//
// A CTA takes a chunk of a row.  The history's tokens of the chunk are counted in shared memory, so that a token that comes
// often costs no more than one that comes once and no order of atomics shows.  HBM-bound: 2 (guided: 3) V elements a row.
#include "logit_rows.cuh"

namespace hbsjd {

namespace {

constexpr int AD_THREADS = 256;

struct Rules {
    const AdjustArgs& a;
    const uint32_t* bits;   // the row's mask, or null
    const int32_t* counts;  // shared: occurrences of the chunk's tokens, or null
    template <int N>
    __device__ __forceinline__ void apply(float (&x)[N], const float (&u)[N], int v, int e, int limit) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (v + i < 0 || v + i >= limit) continue;
            if (a.u) x[i] = fmaf(a.cfg_scale, x[i] - u[i], u[i]);
            if (counts) {
                const int n = counts[e + i];
                if (n) {
                    x[i] = x[i] > 0.f ? x[i] / a.repetition : x[i] * a.repetition;
                    x[i] -= fmaf((float)n, a.frequency, a.presence);
                }
            }
            if (a.bias) x[i] += __ldg(a.bias + v + i);
            if (bits && !(__ldg(bits + ((v + i) >> 5)) >> ((v + i) & 31) & 1)) x[i] = -INFINITY;
            if (x[i] != x[i]) x[i] = -INFINITY;
        }
    }
};

template <typename T>
__global__ void __launch_bounds__(AD_THREADS) k_adjust(AdjustArgs a, int chunk, int chunks) {
    constexpr int G = 16 / sizeof(T);
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / chunks;
    const int v0 = blockIdx.x % chunks * chunk, n = min(chunk, a.V - v0);
    const T* x = (const T*)a.x + row * a.ld + v0;
    const T* u = a.u ? (const T*)a.u + row * a.ld_u + v0 : nullptr;
    T* out = (T*)a.out + row * a.ld_out + v0;
    const int P = phase_of(out);
    const bool wide = phase_of(x) == P && (!u || phase_of(u) == P);
    Rules r = {a, nullptr, nullptr};
    if (a.mask) {
        const int m = a.mask_row ? a.mask_row[row] : 0;
        if (m >= 0 && m < a.masks) r.bits = a.mask + m * a.ld_mask;
    }
    if (a.history) {
        const int64_t h = a.history_row ? a.history_row[row] : row;
        const int len = min(a.history_len ? a.history_len[row] : a.history_cap, a.history_cap);
        if (h >= 0 && h < a.histories && len > 0) {
            int32_t* counts = (int32_t*)smem;  // element P is the chunk's first
            for (int i = tid; i < P + n; i += AD_THREADS) counts[i] = 0;
            __syncthreads();
            const int32_t* tok = a.history + h * a.ld_history;
            for (int i = tid; i < len; i += AD_THREADS) {
                const int64_t e = (int64_t)tok[i] - v0;
                if (e >= 0 && e < n) atomicAdd(&counts[P + e], 1);
            }
            __syncthreads();
            r.counts = counts;
        }
    }
    if (wide) {
        for (int e = tid * G; e < P + n; e += AD_THREADS * G) {
            float f[G], g[G] = {};
            if (e >= P && e + G <= P + n) {
                get<G>(x + e - P, f);
                if (u) get<G>(u + e - P, g);
            } else {
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const bool in = e + i >= P && e + i < P + n;
                    f[i] = in ? to_f<T>(x[e + i - P]) : 0.f;
                    g[i] = in && u ? to_f<T>(u[e + i - P]) : 0.f;
                }
            }
            r.apply<G>(f, g, v0 + e - P, e, v0 + n);
            put_at<T, G>(out, e - P, n, f);
        }
    } else {
        for (int i = tid; i < n; i += AD_THREADS) {
            float f[1] = {to_f<T>(x[i])}, g[1] = {u ? to_f<T>(u[i]) : 0.f};
            r.apply<1>(f, g, v0 + i, P + i, v0 + n);
            out[i] = from_f<T>(f[0]);
        }
    }
}

template <typename T>
cudaError_t run_adjust(const AdjustArgs& a, int rows, Stream& s) {
    int chunk = 8192;
    while (chunk > 1024 && (int64_t)rows * ((a.V + chunk - 1) / chunk) < 2 * device_sm_count()) chunk /= 2;
    const int chunks = (a.V + chunk - 1) / chunk;
    const size_t smem = a.history ? (min(chunk, a.V) + 8) * sizeof(int32_t) : 0;
    return launch_k(k_adjust<T>, dim3((unsigned)rows * chunks), dim3(AD_THREADS), smem, s, a, chunk, chunks);
}

}  // namespace

cudaError_t launch_adjust(const AdjustArgs& a, int rows, int dtype, Stream& s) {
    return dtype ? run_adjust<bf16>(a, rows, s) : run_adjust<float>(a, rows, s);
}

}  // namespace hbsjd
