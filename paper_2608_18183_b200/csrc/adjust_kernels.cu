// Rules on rows of logits in front of a sampler: guidance, penalties for tokens that the row's history holds, a bias and masks of
// allowed tokens, one read and one write of each logit.
//
//   x = l (or l_u + s (l_c - l_u));  n = times that v occurs in the history
//   n > 0:  x = x > 0 ? x / rho : x rho,  x -= n f + pr
//   x += bias[v];  x = -inf where the mask's bit v is 0, and where x is NaN (guidance of two masked branches)
//
// A CTA takes a chunk of a row.  The history's tokens of the chunk are counted in shared memory, so that a token that comes
// often costs no more than one that comes once and no order of atomics shows.  2 (guided: 3) V elements a row:
// HBM bounds fp32 (4096 guided rows of 16384, every rule: 131 us, 0.94 of a copy's rate), the rules' instructions bf16 with histories
// (771 rows of 50021, histories of up to 4096: 58 us, 0.42).
#include <type_traits>

#include "logit_rows.cuh"

namespace hbsjd {

namespace {

constexpr int AD_AHEAD = 2;  // groups of 16 bytes that a thread has on their way

// How often the tokens of a chunk occur, in shared memory: 16 bits each where no history is longer than they count to.
template <typename C>
struct Counts {
    static constexpr int PER = 4 / sizeof(C);  // in a word
    __device__ __forceinline__ static void add(uint32_t* table, int e) { atomicAdd(table + e / PER, 1u << (e % PER * 16)); }
    // of G entries from e on, a multiple of G; false if there are none
    template <int G>
    __device__ __forceinline__ static bool get(const uint32_t* table, int e, float (&n)[G]) {
        uint32_t w[G / PER], any = 0;
        const uint32_t* p = table + e / PER;
        if constexpr (G / PER == 2) {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            w[0] = q.x, w[1] = q.y;
        } else {
#pragma unroll
            for (int i = 0; i < G / PER; i += 4) {
                const uint4 q = *reinterpret_cast<const uint4*>(p + i);
                w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
            }
        }
#pragma unroll
        for (int i = 0; i < G / PER; ++i) any |= w[i];
        if (!any) return false;
#pragma unroll
        for (int i = 0; i < G; ++i)  // (16 bits become fp32 as the low ones of 2^23 + n: one step that is no conversion)
            n[i] = PER == 1 ? (float)w[i] : __uint_as_float(__byte_perm(w[i / 2], 0x4b00u, i % 2 ? 0x5432 : 0x5410)) - 8388608.f;
        return true;
    }
};

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
template <int G, typename C>
__device__ __forceinline__ void apply_rules(const AdjustArgs& a, const uint32_t* bits, const uint32_t* counts, float inv, float (&x)[G],
                                            int v, int e) {
    float n[G];
    if (counts && Counts<C>::template get<G>(counts, e, n)) {
        // (without a branch: some lane of a warp has such a token nearly always)
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const float y = x[i] * (x[i] > 0.f ? inv : a.repetition) - fmaf(n[i], a.frequency, a.presence);
            x[i] = n[i] > 0.f ? y : x[i];
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
        } else if (v >= 3 && v + G + 3 <= a.V && ((uintptr_t)b & 3) == 0) {
            // one vector more, from the 16 bytes that b lies in: all lanes lie alike, and single loads took half the kernel's time
            const int shift = (int)((uintptr_t)b >> 2 & 3);
            float w[G + 4];
#pragma unroll
            for (int i = 0; i < G + 4; i += 4) {
                const float4 q = __ldg(reinterpret_cast<const float4*>(b - shift + i));
                w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
            }
            const auto add = [&](auto by) {
#pragma unroll
                for (int i = 0; i < G; ++i) x[i] += w[i + decltype(by)::value];
            };
            if (shift == 1)
                add(std::integral_constant<int, 1>());
            else if (shift == 2)
                add(std::integral_constant<int, 2>());
            else
                add(std::integral_constant<int, 3>());
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

template <typename T, bool GUIDED, typename C, int THREADS>
__global__ void __launch_bounds__(THREADS) k_adjust(AdjustArgs a, int chunk, int chunks) {
    constexpr int G = 16 / sizeof(T);
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x;
    const int64_t row = blockIdx.x / chunks;
    const int v0 = blockIdx.x % chunks * chunk, n = min(chunk, a.V - v0);
    // what the row has of its own, asked for first: the history's tokens wait for it
    const int which = a.mask && a.mask_row ? a.mask_row[row] : 0;
    const int64_t h = a.history && a.history_row ? a.history_row[row] : row;
    int len = !a.history ? 0 : min(a.history_len ? a.history_len[row] : a.history_cap, a.history_cap);
    const T* x = (const T*)a.x + row * a.ld + v0;
    const T* u = (const T*)a.u + (GUIDED ? row * a.ld_u + v0 : 0);
    T* out = (T*)a.out + row * a.ld_out + v0;
    // groups of 16 bytes of the output: the entry of a thread's first, and the entries from one to its next
    const int P = phase_of(out), e0 = tid * G - P;
    constexpr int STEP = THREADS * G;
    const bool wide = phase_of(x) == P && (!GUIDED || phase_of(u) == P);
    uint4 f[AD_AHEAD], g[AD_AHEAD];
    const auto load = [&](int slot, int e) {
        if (wide && e >= 0 && e + G <= n) {
            f[slot] = load16(x + e);
            if (GUIDED) g[slot] = load16(u + e);
        }
    };
#pragma unroll
    for (int i = 0; i < AD_AHEAD; ++i) load(i, e0 + i * STEP);
    const uint32_t* bits = a.mask && which >= 0 && which < a.masks ? a.mask + which * a.ld_mask : nullptr;
    const uint32_t* counts = nullptr;
    if (h < 0 || h >= a.histories) len = 0;
    if (len > 0) {
        uint32_t* table = (uint32_t*)smem;  // element P is the chunk's first
        for (int i = tid * 16; i < (P + n + G) * (int)sizeof(C); i += THREADS * 16) *reinterpret_cast<uint4*>(smem + i) = make_uint4(0, 0, 0, 0);
        __syncthreads();
        const int32_t* tok = a.history + h * a.ld_history;
        for (int i0 = tid; i0 < len; i0 += THREADS * 8) {
            int32_t t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = i0 + i * THREADS < len ? tok[i0 + i * THREADS] : -1;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((uint32_t)t[i] - (uint32_t)v0 < (uint32_t)n) Counts<C>::add(table, P + t[i] - v0);
        }
        __syncthreads();
        counts = table;
    }
    const float inv = 1.f / a.repetition;  // (a product with it has one rounding more than a division an entry, whose instructions bf16 rows have no room for)
    for (int e = e0; e < n;) {
#pragma unroll
        for (int slot = 0; slot < AD_AHEAD; ++slot, e += STEP) {
            if (e >= n) break;
            float y[G];
            if (wide && e >= 0 && e + G <= n) {
#pragma unroll
                for (int i = 0; i < G; ++i) y[i] = element<T>(f[slot], i);
                if (GUIDED) {
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const float z = element<T>(g[slot], i);
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
            load(slot, e + AD_AHEAD * STEP);
            apply_rules<G, C>(a, bits, counts, inv, y, v0 + e, P + e);
            put_at<T, G>(out, e, 0, n, y);
        }
    }
}

template <typename T, bool GUIDED, typename C, int THREADS>
cudaError_t run_adjust(const AdjustArgs& a, int rows, Stream& s) {
    constexpr int G = 16 / sizeof(T);
    const cudaError_t e = allow_row_smem<k_adjust<T, GUIDED, C, THREADS>>();
    if (e != cudaSuccess) return e;
    // Every chunk reads the row's whole history, and its table takes shared memory: 4096 guided rows of 16384 fp32 with histories of 256
    // take 138, 131 and 162 us with chunks of 4096, 8192 and 16384 entries, 771 rows of 50021 bf16 with histories of up to 4096
    // 77, 63 and 68.  Smaller chunks where rows are few.
    int chunk = 32 * THREADS;
    while (chunk > THREADS * G && (int64_t)rows * ((a.V + chunk - 1) / chunk) < 2 * device_sm_count()) chunk /= 2;
    const int chunks = (a.V + chunk - 1) / chunk;
    const size_t smem = a.history ? ((size_t)std::min(chunk, a.V) + 32) * sizeof(C) : 0;
    return launch_k(k_adjust<T, GUIDED, C, THREADS>, dim3((unsigned)rows * chunks), dim3(THREADS), smem, s, a, chunk, chunks);
}

template <typename T, bool GUIDED, typename C>
cudaError_t run_adjust(const AdjustArgs& a, int rows, Stream& s) {
    // Rows of one chunk: threads that have several groups each (16384 rows of 1000 fp32: 31 us with 64 threads, 52 with 256; of 3001:
    // 85 us with 128, 95 with 256).
    if (a.V <= 2048) return run_adjust<T, GUIDED, C, 64>(a, rows, s);
    if (a.V <= 4096) return run_adjust<T, GUIDED, C, 128>(a, rows, s);
    return run_adjust<T, GUIDED, C, 256>(a, rows, s);
}

template <typename T>
cudaError_t run_adjust(const AdjustArgs& a, int rows, Stream& s) {
    if (a.history_cap > 0xffff) return a.u ? run_adjust<T, true, uint32_t>(a, rows, s) : run_adjust<T, false, uint32_t>(a, rows, s);
    return a.u ? run_adjust<T, true, uint16_t>(a, rows, s) : run_adjust<T, false, uint16_t>(a, rows, s);
}

}  // namespace

cudaError_t launch_adjust(const AdjustArgs& a, int rows, int dtype, Stream& s) {
    return dtype ? run_adjust<bf16>(a, rows, s) : run_adjust<float>(a, rows, s);
}

}  // namespace hbsjd
