// Rows of logits held in shared memory by one CTA or by a cluster of CTAs: staging of rows of any alignment, wide reads,
// sums over the CTAs of a row, and the launch rules that the operators on rows share.
#pragma once
#include <math.h>

#include <algorithm>
#include <atomic>

#include "internal.h"

namespace hbsjd {

constexpr int MAX_LOGIT_V = 131072;    // entries of a row: what eight CTAs hold of two fp32 rows
constexpr int MAX_LISTED = 1024;       // entries of a top-K list
constexpr int ROW_CTAS = 8;            // CTAs of a row, at most (the portable cluster size)
constexpr int ROW_SMEM = 200 * 1024;   // dynamic shared memory that a CTA may ask for
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// 2^x.  Below 2^-126: zero.
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 values in one register pair: sums and products of both by one instruction.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 both(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f32x2 both(float v) { return both(v, v); }
__device__ __forceinline__ void split(f32x2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 ex2(f32x2 v) {
    float lo, hi;
    split(v, lo, hi);
    return both(ex2(lo), ex2(hi));
}
__device__ __forceinline__ float sum2(f32x2 v) {
    float lo, hi;
    split(v, lo, hi);
    return lo + hi;
}
// Largest of the warp's values that are numbers.
__device__ __forceinline__ float max_of_warp(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// ------------------------------------------------------------------ clusters
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// address in CTA `rank`'s shared memory of what lies at `p` in this CTA's
__device__ __forceinline__ uint32_t remote_smem(const void* p, uint32_t rank) {
    uint32_t a = (uint32_t)__cvta_generic_to_shared(p), r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ void remote_store(uint32_t a, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}
__device__ __forceinline__ void remote_store(uint32_t a, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}

// ------------------------------------------------------------------ staging
__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(void* dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Place of a row's first element behind a 16-byte boundary, in elements.
template <typename T>
__device__ __forceinline__ int phase_of(const T* p) {
    return (int)((reinterpret_cast<uintptr_t>(p) / sizeof(T)) % (16 / sizeof(T)));
}

// Fills a staged row up to whole groups: no mass beside any logit above it, and no infinities in differences.
constexpr float PAD = -1e30f;

// All threads: src[0, n) to dst[P, P + n), and `pad` in front of it and behind it up to a multiple of G elements (dst starts on
// 16 bytes, 0 <= P < 8).  16 bytes at a time where src lies P elements behind a 16-byte boundary too; then the first and
// last elements go one by one, so that nothing outside src is read.  To be followed by cp_async_wait_all and a barrier.
template <typename T, int G, int THREADS>
__device__ __forceinline__ void stage_row(T* dst, const T* src, int n, int P, float pad) {
    constexpr int VEC = 16 / sizeof(T);
    const int tid = threadIdx.x, end = P + n;
    const int padded = (end + G - 1) / G * G;
    if (phase_of(src) == P % VEC) {
        const int first = (P + VEC - 1) / VEC, last = end / VEC;  // whole vectors
        const T* base = src - P;
#pragma unroll 4
        for (int j = first + tid; j < last; j += THREADS) cp_async16(dst + j * VEC, base + j * VEC);
        // fewer than VEC elements in front, fewer than VEC behind
        const int head_end = min(first * VEC, end), tail = max(last * VEC, head_end);
        if (tid < head_end - P) dst[P + tid] = src[tid];
        if (tid < end - tail) dst[tail + tid] = src[tail - P + tid];
    } else if (sizeof(T) == 4) {
#pragma unroll 8
        for (int i = tid; i < n; i += THREADS) cp_async4(dst + P + i, src + i);
    } else {
#pragma unroll 8
        for (int i = tid; i < n; i += THREADS) dst[P + i] = src[i];
    }
    if (tid < P) dst[tid] = from_f<T>(pad);
    if (tid < padded - end) dst[end + tid] = from_f<T>(pad);
}

// G consecutive elements, aligned to their size.
template <int G>
__device__ __forceinline__ void get(const float* p, float (&x)[G]) {
#pragma unroll
    for (int i = 0; i < G; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(p + i);
        x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
}
__device__ __forceinline__ void unpack(uint32_t w, float& lo, float& hi) {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
}
template <int G>
__device__ __forceinline__ void get(const bf16* p, float (&x)[G]) {
    if constexpr (G == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        unpack(v.x, x[0], x[1]);
        unpack(v.y, x[2], x[3]);
    } else {
        static_assert(G == 8, "a group is 4 or 8 elements");
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        unpack(v.x, x[0], x[1]);
        unpack(v.y, x[2], x[3]);
        unpack(v.z, x[4], x[5]);
        unpack(v.w, x[6], x[7]);
    }
}
template <int G>
__device__ __forceinline__ void put(float* p, const float (&x)[G]) {
#pragma unroll
    for (int i = 0; i < G; i += 4) __stcs(reinterpret_cast<float4*>(p + i), make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <int G>
__device__ __forceinline__ void put(bf16* p, const float (&x)[G]) {
    if constexpr (G == 4)
        __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack(x[0], x[1]), pack(x[2], x[3])));
    else
        __stcs(reinterpret_cast<uint4*>(p),
               make_uint4(pack(x[0], x[1]), pack(x[2], x[3]), pack(x[4], x[5]), pack(x[6], x[7])));
}
// G elements of a staged row from its element i on (element 0 lies at p[P]), those outside [0, n) -inf or anything.  wide: i + P
// is a multiple of G.
template <typename T, int G>
__device__ __forceinline__ void get_at(const T* p, int P, int i, int n, bool wide, float (&x)[G]) {
    if (wide) {
        get<G>(p + P + i, x);
    } else {
#pragma unroll
        for (int e = 0; e < G; ++e) x[e] = i + e >= 0 && i + e < n ? to_f<T>(p[P + i + e]) : -INFINITY;
    }
}
// The elements of [i, i + G) that lie in [0, n) to out (out + i lies on a multiple of G elements).
template <typename T, int G>
__device__ __forceinline__ void put_at(T* out, int i, int n, const float (&x)[G]) {
    if (i >= 0 && i + G <= n) {
        put<G>(out + i, x);
    } else {
#pragma unroll
        for (int e = 0; e < G; ++e)
            if (i + e >= 0 && i + e < n) out[i + e] = from_f<T>(x[e]);
    }
}
// out[0, n) = 0, wide where out's alignment allows it.
template <typename T, int THREADS>
__device__ __forceinline__ void put_zeros(T* out, int n) {
    constexpr int G = 16 / sizeof(T);
    const float zero[G] = {};
    const int P = phase_of(out);
    for (int i = (int)threadIdx.x * G - P; i < n; i += THREADS * G) put_at<T, G>(out, i, n, zero);
}

// ------------------------------------------------------------------ sums of exponentials
// 2^{(from - to) c}; zero where nothing was summed, 1 where both are infinite.  (to >= from)
__device__ __forceinline__ float rescale(float from, float to, float c) {
    return from == -INFINITY ? 0.f : from == to ? 1.f : ex2((from - to) * c);
}

// A sum z of 2^{(x - m) c}, where m is within reach of its largest x (z neither overflows nor vanishes).
struct Mass {
    static constexpr int N = 2, SUMS = 1;
    float m, z;
    __device__ __forceinline__ static Mass none() { return {-INFINITY, 0.f}; }
    __device__ __forceinline__ float* sums() { return &z; }
    __device__ __forceinline__ void raise(Mass& to) const { to.m = fmaxf(to.m, m); }
    __device__ __forceinline__ void share() { m = max_of_warp(m); }
    // against `to`'s reference, which is no less than its own
    __device__ __forceinline__ Mass against(const Mass& to, float c) const { return {to.m, z * rescale(m, to.m, c)}; }
};

__device__ __forceinline__ Mass merge(const Mass& x, const Mass& y, float c) {
    const Mass to = {fmaxf(x.m, y.m), 0.f};
    return {to.m, x.against(to, c).z + y.against(to, c).z};
}

// The masses of two rows s and t over the same entries, and their sums of d = (s - ms) - (t - mt) weighted by each.
// Against references near the largest of both, d does not grow with what is common to a row.
struct Pair {
    static constexpr int N = 6, SUMS = 4;
    float ms, mt, zs, zt, as, at;
    __device__ __forceinline__ static Pair none() { return {-INFINITY, -INFINITY, 0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ float* sums() { return &zs; }
    __device__ __forceinline__ void raise(Pair& to) const { to.ms = fmaxf(to.ms, ms), to.mt = fmaxf(to.mt, mt); }
    __device__ __forceinline__ void share() { ms = max_of_warp(ms), mt = max_of_warp(mt); }
    __device__ __forceinline__ Pair against(const Pair& to, float c) const {
        const float fs = rescale(ms, to.ms, c), ft = rescale(mt, to.mt, c);
        // (a sum whose row has no mass here is infinite or zero: no shift changes it)
        const float shift = (ms == -INFINITY ? 0.f : ms - to.ms) - (mt == -INFINITY ? 0.f : mt - to.mt);
        // no factor of zero times an infinite sum
        return {to.ms, to.mt, zs * fs, zt * ft, fs == 0.f ? 0.f : fs * fmaf(zs, shift, as), ft == 0.f ? 0.f : ft * fmaf(zt, shift, at)};
    }
};

// Lane 0's sum in every lane: one order for all.
__device__ __forceinline__ float sum_of_warp(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Places for the sums of a row's warps.
template <typename S, int THREADS>
struct Slots {
    S s[ROW_CTAS * THREADS / 32];
};
// A warp's sums (the same in all lanes) to all CTAs of the row (of which there are several: they have waited for one
// another's start), or to its own.
template <typename S, int THREADS>
__device__ __forceinline__ void post(const S& x, Slots<S, THREADS>& slots, int ctas) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    if (ctas == 1) {
        if (lane == 0) slots.s[wid] = x;
    } else if (lane < ctas) {
        const uint32_t a = remote_smem(&slots.s[cluster_rank() * WARPS + wid], lane);
        const float* g = reinterpret_cast<const float*>(&x);
#pragma unroll
        for (int e = 0; e < S::N; ++e) remote_store(a + 4 * e, g[e]);
    }
}
// All threads of the row: what was posted before is there after it.  In a cluster, none touches the others' shared memory later.
__device__ __forceinline__ void posted(int ctas) {
    if (ctas == 1) {
        __syncthreads();
    } else {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
}
// The row's sums from its warps', the same bits in every thread.
template <typename S, int THREADS>
__device__ __forceinline__ S collect(const Slots<S, THREADS>& slots, int ctas, float c) {
    const int lane = threadIdx.x & 31, count = THREADS / 32 * ctas;
    S top = S::none();
    for (int j = lane; j < count; j += 32) slots.s[j].raise(top);
    top.share();
    S r = top;
#pragma unroll
    for (int e = 0; e < S::SUMS; ++e) r.sums()[e] = 0.f;
    for (int j = lane; j < count; j += 32) {
        S x = slots.s[j].against(top, c);
#pragma unroll
        for (int e = 0; e < S::SUMS; ++e) r.sums()[e] += x.sums()[e];
    }
#pragma unroll
    for (int e = 0; e < S::SUMS; ++e) r.sums()[e] = sum_of_warp(r.sums()[e]);
    return r;
}

// ------------------------------------------------------------------ launches
// Raises a kernel's limit of dynamic shared memory to ROW_SMEM, once per device; any threads may call it at once.
template <auto Kernel>
inline cudaError_t allow_row_smem() {
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ROW_SMEM);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// How a row is split: CTAs (a cluster, where more than one) and the elements that each holds.
struct RowSplit {
    int ctas, slice;
};
inline RowSplit split_row(int64_t rows, int V, int bytes_per_element, int sms) {
    int ctas = 1;
    while (ctas < ROW_CTAS && (int64_t)V * bytes_per_element > 72 * 1024 * (int64_t)ctas) ctas *= 2;
    while (ctas < ROW_CTAS && rows * ctas * 2 <= sms && V >= 2048 * ctas) ctas *= 2;
    return {ctas, ((V + ctas - 1) / ctas + 7) / 8 * 8};
}

struct DistillArgs {
    const void *s, *t;       // student's and teacher's rows
    int64_t ld_s, ld_t, ld_g;
    const float* weight;     // [rows] or null
    float* loss;             // [rows] or null
    void* grad;              // rows, or null
    int V, ctas, slice;
    float temperature, forward, reverse;
    // the teacher as a list (hbsjd_distill_topk)
    const float* values;     // [rows][k]
    const int32_t* indices;  // [rows][k]
    const float* rest;       // [rows] or null
    int k;
};
// dtypes: HBSJD_DTYPE_*
cudaError_t launch_distill(const DistillArgs& a, int rows, int dtype_s, int dtype_t, Stream& s);
cudaError_t launch_distill_topk(const DistillArgs& a, int rows, int dtype_s, Stream& s);

struct TopkArgs {
    const void* x;
    int64_t ld;
    float* values;     // [rows][k]
    int32_t* indices;  // [rows][k]
    float* rest;       // [rows] or null
    int V, k, ctas, slice;
    float temperature;
    // rows of a scoring forward (null: row r of x is row r of the outputs): row r holds the distribution of position
    // at[r].y + 1 of image at[r].x, and goes to row at[r].x * T + at[r].y if that position lies behind the image's prefix
    const int2* at;
    const int32_t* prefix_len;
    int T;
};
cudaError_t launch_topk(const TopkArgs& a, int rows, int dtype, Stream& s);

struct AdjustArgs {
    const void *x, *u;
    void* out;
    int64_t ld, ld_u, ld_out;
    const float* bias;
    const uint32_t* mask;
    const int32_t *mask_row, *history, *history_row, *history_len;
    int64_t ld_mask, ld_history;
    int V, masks, histories, history_cap;
    float cfg_scale, repetition, frequency, presence;
};
cudaError_t launch_adjust(const AdjustArgs& a, int rows, int dtype, Stream& s);

}  // namespace hbsjd
