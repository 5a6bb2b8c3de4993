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
#ifndef ADG
#define ADG 2
#endif
constexpr int AD_GROUPS = ADG;  // 16-byte groups of a thread: all of a CTA's logits are on their way while it counts the history

// (volatile: the loads of all groups are to be under way before the first is used)
__device__ __forceinline__ uint4 load16(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
template <typename T>
__device__ __forceinline__ float element(const uint4& v, int i) {
    if (sizeof(T) == 4) return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w);
    const uint32_t w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
}

// x[i] is entry v + i of the row; those outside [0, V) are not looked at (v may be negative).
template <int G>
__device__ __forceinline__ void apply_rules(const AdjustArgs& a, const uint32_t* bits, const int32_t* counts, float (&x)[G], int v,
                                            int e) {
    if (counts) {
        int n[G];
        bool any = false;
#pragma unroll
        for (int i = 0; i < G; i += 4) {
            const int4 q = *reinterpret_cast<const int4*>(counts + e + i);
            n[i] = q.x, n[i + 1] = q.y, n[i + 2] = q.z, n[i + 3] = q.w;
            any |= (q.x | q.y | q.z | q.w) != 0;
        }
        if (any) {
            // (without a branch: some lane of a warp has such a token nearly always)
            const float inv = 1.f / a.repetition;
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const float y = x[i] * (x[i] > 0.f ? inv : a.repetition) - fmaf((float)n[i], a.frequency, a.presence);
                x[i] = n[i] ? y : x[i];
            }
        }
    }
    if (a.bias) {
        const float* b = a.bias + v;
        if (v >= 0 && v + G <= a.V && ((uintptr_t)b & 15) == 0) {
#pragma unroll
            for (int i = 0; i < G; i += 4) {
                const float4 q = __ldg(reinterpret_cast<const float4*>(b + i));
                x[i] += q.x, x[i + 1] += q.y, x[i + 2] += q.z, x[i + 3] += q.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (v + i >= 0 && v + i < a.V) x[i] += __ldg(b + i);
        }
    }
    if (bits) {
        // the G bits from v on, which may lie in two words
        const int last = (a.V - 1) >> 5, w = v >> 5;
        const uint32_t lo = w >= 0 ? __ldg(bits + w) : 0, hi = (v & 31) + G > 32 && w < last ? __ldg(bits + w + 1) : 0;
        const uint32_t m = __funnelshift_r(lo, hi, v & 31);
#pragma unroll
        for (int i = 0; i < G; ++i)
            if (!(m >> i & 1)) x[i] = -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < G; ++i) x[i] = fmaxf(x[i], -INFINITY);  // (of NaN and a number, the number)
}

template <typename T, bool GUIDED>
__global__ void __launch_bounds__(AD_THREADS) k_adjust(AdjustArgs a, int chunk, int chunks) {
    constexpr int G = 16 / sizeof(T);
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / chunks;
    const int v0 = blockIdx.x % chunks * chunk, n = min(chunk, a.V - v0);
    const T* x = (const T*)a.x + row * a.ld + v0;
    const T* u = (const T*)a.u + (GUIDED ? row * a.ld_u + v0 : 0);
    T* out = (T*)a.out + row * a.ld_out + v0;
    // groups of 16 bytes of the output; P + n <= chunk + G - 1 elements, so a chunk of whole rounds has one group more at most
    const int P = phase_of(out), rounds = (P + n + AD_THREADS * G - 1) / (AD_THREADS * G);
    const bool wide = phase_of(x) == P && (!GUIDED || phase_of(u) == P);
    uint4 f[AD_GROUPS], g[GUIDED ? AD_GROUPS : 1];
#pragma unroll
    for (int r = 0; r < AD_GROUPS; ++r) {
        const int e = (r * AD_THREADS + tid) * G - P;
        if (wide && e >= 0 && e + G <= n) {
            f[r] = load16(x + e);
            if (GUIDED) g[r] = load16(u + e);
        }
    }
    const uint32_t* bits = nullptr;
    if (a.mask) {
        const int m = a.mask_row ? a.mask_row[row] : 0;
        if (m >= 0 && m < a.masks) bits = a.mask + m * a.ld_mask;
    }
    const int32_t* counts = nullptr;
    if (a.history) {
        const int64_t h = a.history_row ? a.history_row[row] : row;
        const int len = min(a.history_len ? a.history_len[row] : a.history_cap, a.history_cap);
        if (h >= 0 && h < a.histories && len > 0) {
            int32_t* count = (int32_t*)smem;  // element P is the chunk's first
            for (int i = tid * 4; i < P + n; i += AD_THREADS * 4) *reinterpret_cast<int4*>(count + i) = make_int4(0, 0, 0, 0);
            __syncthreads();
            const int32_t* tok = a.history + h * a.ld_history;
            for (int i0 = tid; i0 < len; i0 += AD_THREADS * 8) {
                int32_t t[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] = i0 + i * AD_THREADS < len ? tok[i0 + i * AD_THREADS] : -1;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (t[i] >= v0 && t[i] < v0 + n) atomicAdd(&count[P + t[i] - v0], 1);
            }
            __syncthreads();
            counts = count;
        }
    }
#pragma unroll
    for (int r = 0; r < AD_GROUPS + 1; ++r) {
        if (r >= rounds) break;
        const int e = (r * AD_THREADS + tid) * G - P;
        if (e >= n) break;
        float y[G];
        if (r < AD_GROUPS && wide && e >= 0 && e + G <= n) {
#pragma unroll
            for (int i = 0; i < G; ++i) y[i] = element<T>(f[r < AD_GROUPS ? r : 0], i);
            if (GUIDED) {
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const float z = element<T>(g[r < AD_GROUPS ? r : 0], i);
                    y[i] = fmaf(a.cfg_scale, y[i] - z, z);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const bool in = e + i >= 0 && e + i < n;
                y[i] = in ? to_f<T>(x[e + i]) : 0.f;
                if (GUIDED && in) y[i] = fmaf(a.cfg_scale, y[i] - to_f<T>(u[e + i]), to_f<T>(u[e + i]));
            }
        }
        apply_rules<G>(a, bits, counts, y, v0 + e, P + e);
        put_at<T, G>(out, e, 0, n, y);
    }
}

template <typename T, bool GUIDED>
cudaError_t run_adjust(const AdjustArgs& a, int rows, Stream& s) {
    constexpr int G = 16 / sizeof(T);
    int chunk = AD_THREADS * G * AD_GROUPS;
    while (chunk > AD_THREADS * G && (int64_t)rows * ((a.V + chunk - 1) / chunk) < 2 * device_sm_count()) chunk /= 2;
    const int chunks = (a.V + chunk - 1) / chunk;
    const size_t smem = a.history ? (min(chunk, a.V) + 16) * sizeof(int32_t) : 0;
    return launch_k(k_adjust<T, GUIDED>, dim3((unsigned)rows * chunks), dim3(AD_THREADS), smem, s, a, chunk, chunks);
}

}  // namespace

cudaError_t launch_adjust(const AdjustArgs& a, int rows, int dtype, Stream& s) {
    if (a.u) return dtype ? run_adjust<bf16, true>(a, rows, s) : run_adjust<float, true>(a, rows, s);
    return dtype ? run_adjust<bf16, false>(a, rows, s) : run_adjust<float, false>(a, rows, s);
}

}  // namespace hbsjd
