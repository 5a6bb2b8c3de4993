// Rows of logits held in shared memory by one CTA or by a cluster of CTAs: staging of rows of any alignment, wide reads,
// sums over the CTAs of a row, and the launch rules that the operators on rows share.
#pragma once
#include <cmath>

#include <algorithm>
#include <atomic>

#include "internal.h"
#include "row_parts.cuh"

namespace hbsjd {

constexpr int MAX_LOGIT_V = 131072;    // entries of a row: what eight CTAs hold of two fp32 rows
constexpr int MAX_LISTED = 1024;       // entries of a top-K list
constexpr int ROW_SMEM = 216 * 1024;   // dynamic shared memory that a CTA may ask for
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// Exponents are taken in powers of two: x log2(e) / temperature.
inline bool is_temperature(float t) { return t > 0.f && std::isfinite(t) && std::isfinite(LOG2E * (1.f / t)); }

// 2^x.  Below 2^-126: zero.
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// log2(x) within 2^-22 (absolute for x in (0.5, 2), else relative): no worse than the sums it is taken of.
__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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
// All threads of a cluster.  (A warp meets first: the aligned form is undefined where its lanes come apart, and rows end in branches by
// lane.  The form that is not aligned costs 8192 pairs of rows of 16384 fp32 283 us in place of 280.)
__device__ __forceinline__ void cluster_barrier() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
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
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All of this thread's groups but the last `pending` (0 or 1) have arrived.
__device__ __forceinline__ void cp_async_wait(int pending) {
    if (pending)
        asm volatile("cp.async.wait_group 1;" ::: "memory");
    else
        asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Place of a row's first element behind a 16-byte boundary, in elements.
template <typename T>
__device__ __forceinline__ int phase_of(const T* p) {
    return (int)((reinterpret_cast<uintptr_t>(p) / sizeof(T)) % (16 / sizeof(T)));
}

// Fills a staged row up to whole groups: no mass beside any logit above it, and no infinities in differences.
constexpr float PAD = -1e30f;

// All threads: begins the copy of src[0, n) to dst[P, P + n) (dst starts on 16 bytes, 0 <= P < 8).  16 bytes at a time
// where src lies P elements behind a 16-byte boundary too, 4 where it lies so behind a 4-byte boundary, else one by one.  Of bf16, the 4
// bytes that hold src's first or last element may hold one of a neighbour: it is copied too.  Then
// cp_async_wait_all, a barrier, end_row and a barrier.
template <typename T, int THREADS>
__device__ __forceinline__ void stage_row(T* dst, const T* src, int n, int P) {
    constexpr int VEC = 16 / sizeof(T), W = 4 / sizeof(T);
    const int tid = threadIdx.x, end = P + n;
    const T* base = src - P;
    if (n <= 0) return;
    if (phase_of(src) == P % VEC) {
        const int first = (P + VEC - 1) / VEC, last = end / VEC;  // whole vectors
#pragma unroll 4
        for (int j = first + tid; j < last; j += THREADS) cp_async16(dst + j * VEC, base + j * VEC);
        // words of the less than VEC elements in front, and of those behind
        const int head_end = min(first * VEC, end), tail = max(last * VEC, head_end), w = P / W + tid;
        if (w * W < head_end) cp_async4(dst + w * W, base + w * W);
        const int q = tid - (THREADS > 32 ? 32 : 16);  // (other threads than those of the head)
        if (q >= 0 && tail + q * W < end) cp_async4(dst + tail + q * W, base + tail + q * W);
    } else if ((phase_of(src) - P) % W == 0) {
#pragma unroll 8
        for (int w = P / W + tid; w * W < end; w += THREADS) cp_async4(dst + w * W, base + w * W);
    } else {
        for (int i = tid; i < n; i += THREADS * 8) {
            T x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u * THREADS < n) x[u] = src[i + u * THREADS];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u * THREADS < n) dst[P + i + u * THREADS] = x[u];
        }
    }
}
// `pad` in front of a staged row and behind it up to a multiple of G elements.
template <typename T, int G>
__device__ __forceinline__ void end_row(T* dst, int n, int P, float pad) {
    const int tid = threadIdx.x, end = P + n, padded = (end + G - 1) / G * G;
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
// The elements of [i, i + G) that lie in [lo, hi) to out (out + i lies on a multiple of G elements).
template <typename T, int G>
__device__ __forceinline__ void put_at(T* out, int i, int lo, int hi, const float (&x)[G]) {
    if (i >= lo && i + G <= hi) {
        put<G>(out + i, x);
    } else {
#pragma unroll
        for (int e = 0; e < G; ++e)
            if (i + e >= lo && i + e < hi) out[i + e] = from_f<T>(x[e]);
    }
}

// ------------------------------------------------------------------ a warp's part of a row (see row_parts.cuh)
// The words of the less than 16 bytes in front of the part's whole vectors, and of those behind.
template <typename T, int G, int WARPS>
__device__ __forceinline__ void stage_ends(T* dst, const T* src, const Part<G, WARPS>& p) {
    constexpr int VEC = 16 / sizeof(T), W = 4 / sizeof(T);
    const int lane = threadIdx.x & 31, b = p.first(), f = p.last();
    const T* base = src - p.P;
    if ((b | f) % VEC && b < f) {
        const int head_end = min((b + VEC - 1) / VEC * VEC, f), tail = max(f / VEC * VEC, head_end), w = b / W + lane;
        if (w * W < head_end) cp_async4(dst + w * W, base + w * W);
        if (tail + lane * W < f) cp_async4(dst + tail + lane * W, base + tail + lane * W);
    }
}
// Begins the copy of the warp's part of a slice at src.  16 bytes at a time where src lies P elements behind a 16-byte boundary
// too, 4 where it lies so behind a 4-byte boundary, else one by one.  Of bf16, the 4 bytes that hold the slice's first or last element may
// hold one of a neighbour: it is copied too (and covered by end_part).
template <typename T, int G, int WARPS>
__device__ __forceinline__ void stage_part(T* dst, const T* src, const Part<G, WARPS>& p) {
    constexpr int VEC = 16 / sizeof(T), W = 4 / sizeof(T);
    const int lane = threadIdx.x & 31, b = p.first(), f = p.last();
    const T* base = src - p.P;
    if (f <= b) return;
    if (phase_of(src) == p.P % VEC) {
        const int first = (b + VEC - 1) / VEC, last = f / VEC;  // whole vectors
#pragma unroll 4
        for (int j = first + lane; j < last; j += 32) cp_async16(dst + j * VEC, base + j * VEC);
        stage_ends(dst, src, p);
    } else if ((phase_of(src) - p.P) % W == 0) {
#pragma unroll 8
        for (int w = b / W + lane; w * W < f; w += 32) cp_async4(dst + w * W, base + w * W);
    } else {
        for (int e = b + lane; e < f; e += 32 * 8) {
            T x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (e + u * 32 < f) x[u] = base[e + u * 32];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (e + u * 32 < f) dst[e + u * 32] = x[u];
        }
    }
}
// `pad` in the places of the warp's groups that are not the row's.  (Fewer than G + 8 of them; the copies have arrived.)
template <typename T, int G, int WARPS>
__device__ __forceinline__ void end_part(T* dst, const Part<G, WARPS>& p, float pad) {
    const int lane = threadIdx.x & 31, b = p.first(), f = max(p.last(), p.j0 * G);
    if (p.j0 * G + lane < min(b, p.j1 * G)) dst[p.j0 * G + lane] = from_f<T>(pad);
    if (f + lane < p.j1 * G) dst[f + lane] = from_f<T>(pad);
    __syncwarp();
}
// f(j, whole) for the warp's groups, one a lane: those that are the row's in whole first, in a loop without a condition.
template <int G, int WARPS, typename F>
__device__ __forceinline__ void each_group(const Part<G, WARPS>& p, F&& f) {
    const int lane = threadIdx.x & 31, inner = p.inner(), outer = p.outer();
#pragma unroll 4
    for (int j = inner + lane; j < outer; j += 32) f(j, std::true_type());
    // of the others, at most two hold some of the row: one in front, one behind
    if (inner > p.j0 && lane == 0) f(inner - 1, std::false_type());
    if (outer < p.j1 && lane == 1) f(outer, std::false_type());
}
// out[lo, hi) = 0 by a warp.
template <typename T>
__device__ __forceinline__ void put_zeros(T* out, int lo, int hi) {
    constexpr int G = 16 / sizeof(T);
    const float zero[G] = {};
    const int lane = threadIdx.x & 31, Pg = (phase_of(out) + lo) % G;
    for (int e = lo - Pg + lane * G; e < hi; e += 32 * G) put_at<T, G>(out, e, lo, hi, zero);
}

// ------------------------------------------------------------------ sums of exponentials
// 2^{(from - to) c}; zero where nothing was summed, 1 where both are infinite.  (to >= from)
__device__ __forceinline__ float rescale(float from, float to, float c) {
    return from == -INFINITY ? 0.f : from == to ? 1.f : ex2((from - to) * c);
}

// A sum z of 2^{(x - m) c}, where m is within reach of its largest x (z neither overflows nor vanishes).
struct Mass {
    float m, z;
    __device__ __forceinline__ static Mass none() { return {-INFINITY, 0.f}; }
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
    float ms, mt, zs, zt, as, at;
    __device__ __forceinline__ static Pair none() { return {-INFINITY, -INFINITY, 0.f, 0.f, 0.f, 0.f}; }
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

// Four values' sums at once: lane i gets the sum of v[i / 8].
__device__ __forceinline__ float sums_of_warp(const float (&v)[4]) {
    const int lane = threadIdx.x & 31;
    const bool up = lane & 16, mid = lane & 8;
    const float a = (up ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[2], 16);
    const float b = (up ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, up ? v[1] : v[3], 16);
    float r = (mid ? b : a) + __shfl_xor_sync(0xffffffffu, mid ? a : b, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
    return r;
}

// One float of a warp's sums to its place in this CTA, or in CTA `to` of several (which have waited for one another's start).
__device__ __forceinline__ void post_float(float* place, int ctas, int to, float v) {
    if (ctas == 1)
        *place = v;
    else
        remote_store(remote_smem(place, to), v);
}
// A warp's sums to its place of `slots` (shared memory for ctas x WARPS of them) in all CTAs of the row; a pair's as each lane's
// share.
template <int WARPS>
__device__ __forceinline__ void post(const Pair& x, Pair* slots, int ctas, int rank) {
    const int lane = threadIdx.x & 31, to = lane & 7, which = lane >> 3;
    const float v[4] = {x.zs, x.zt, x.as, x.at};
    const float sum = sums_of_warp(v);
    if (to < ctas) {
        float* f = reinterpret_cast<float*>(slots + rank * WARPS + (threadIdx.x >> 5));
        post_float(f + 2 + which, ctas, to, sum);
        if (which < 2) post_float(f + which, ctas, to, which ? x.mt : x.ms);
    }
}
template <int WARPS>
__device__ __forceinline__ void post(const Mass& x, Mass* slots, int ctas, int rank) {
    const int lane = threadIdx.x & 31;
    if (lane < ctas) {
        float* f = reinterpret_cast<float*>(slots + rank * WARPS + (threadIdx.x >> 5));
        post_float(f, ctas, lane, x.m);
        post_float(f + 1, ctas, lane, x.z);
    }
}
// All threads of the row: what was posted before is there after it.  In a cluster, none touches the others' shared memory later.
__device__ __forceinline__ void posted(int ctas) {
    if (ctas == 1) {
        __syncthreads();
    } else {
        cluster_barrier();
    }
}
// The row's sums from its warps', the same bits in every warp that asks.
__device__ __forceinline__ Mass collect(const Mass* slots, int count, float c) {
    const int lane = threadIdx.x & 31;
    Mass top = Mass::none();
    for (int j = lane; j < count; j += 32) slots[j].raise(top);
    top.share();
    float z = 0.f;
    for (int j = lane; j < count; j += 32) z += slots[j].against(top, c).z;
    return {top.m, sum_of_warp(z)};
}
__device__ __forceinline__ Pair collect(const Pair* slots, int count, float c) {
    const int lane = threadIdx.x & 31;
    Pair r = Pair::none();
    for (int j = lane; j < count; j += 32) slots[j].raise(r);
    r.share();
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j = lane; j < count; j += 32) {
        const Pair x = slots[j].against(r, c);
        v[0] += x.zs, v[1] += x.zt, v[2] += x.as, v[3] += x.at;
    }
    const float sum = sums_of_warp(v);
    r.zs = __shfl_sync(0xffffffffu, sum, 0);
    r.zt = __shfl_sync(0xffffffffu, sum, 8);
    r.as = __shfl_sync(0xffffffffu, sum, 16);
    r.at = __shfl_sync(0xffffffffu, sum, 24);
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

// Clusters of `ctas` CTAs that rows are dealt to: no more than run at once.
template <auto Kernel>
inline cudaError_t resident_clusters(int ctas, int threads, int per_sm, size_t smem, int64_t rows, int* clusters) {
    const int sms = device_sm_count();
    *clusters = (int)std::min<int64_t>(rows, std::max(1, sms * per_sm / ctas));
    if (ctas <= 2 || rows * ctas * 2 <= (int64_t)sms * per_sm) return cudaSuccess;
    // Larger clusters lie within groups of SMs that they may not fill.  The last answer is kept: a loop asks for one shape.
    static std::atomic<uint64_t> last{0};  // device, shared memory, CTAs; then the answer
    int dev = 0, most = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t asked = (((uint64_t)(dev + 1) << 24 | smem) << 4 | (uint64_t)ctas) << 16, known = last.load(std::memory_order_relaxed);
    if ((known & ~(uint64_t)0xffff) == asked) {
        most = (int)(known & 0xffff);
    } else {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(sms * per_sm / ctas * ctas);
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = ctas;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&most, Kernel, &cfg);
        if (e != cudaSuccess) return e;
        last.store(asked | (uint64_t)std::min(most, 0xffff), std::memory_order_relaxed);
    }
    if (most > 0) *clusters = std::min(*clusters, most);
    return cudaSuccess;
}

struct DistillArgs {
    const void *s, *t;       // student's and teacher's rows
    int64_t ld_s, ld_t, ld_g;
    const float* weight;     // [rows] or null
    float* loss;             // [rows] or null
    void* grad;              // rows, or null
    int rows, V, ctas, slice;
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
    int rows, V, k, ctas, slice, cap;
    float temperature;
    // rows of a scoring forward (null: row r of x is row r of the outputs): row r holds the distribution of position
    // at[r].y + 1 of image at[r].x, and goes to row at[r].x * T + at[r].y if that position lies behind the image's prefix
    const int2* at;
    const int32_t* prefix_len;
    int T;
};
cudaError_t launch_topk(const TopkArgs& a, int rows, int dtype, Stream& s);
// empty lists for the positions of the images' prefixes (a.prefix_len, a.T)
cudaError_t launch_topk_clear(const TopkArgs& a, int batch, Stream& s);

struct TokenArgs {
    const void* x;
    int64_t ld, ld_g;
    const int32_t* tokens;   // [rows]
    const float* weight;     // [rows] or null; 0: the row is left out
    const float *advantage, *old_logp, *ref;  // [rows]: the policy's loss; null: none, its own, no KL term
    const float *d_logp, *d_entropy;          // [rows]: the gradient of these; null: the policy's, none
    float *loss, *logp, *entropy;             // [rows] or null
    void* grad;              // rows, or null
    float4* stats;           // [rows] or null: m, z (see TokenSums), the mass of the others, what the rounding of logp left
    int rows, V, ctas, slice, tiles;  // tiles: slices that a CTA takes in turn (then ctas is 1)
    int summed;                       // logp is for sums over many rows
    float temperature, low, high, dual, kl, bonus;
    // rows of a scoring forward (see TopkArgs); tokens, logp and entropy are [batch][T] then
    const int2* at;
    const int32_t* prefix_len;
    int T;
};
cudaError_t launch_token(const TokenArgs& a, int rows, int dtype, Stream& s);

// The gradient of slope log q_token from a row's sums, the last rows first: those that were summed last may still be in L2.
struct SpreadArgs {
    const void* x;
    void* grad;
    int64_t ld, ld_g;
    const int32_t* tokens;  // [rows]
    const float* slope;     // [rows]; 0: the row is left out
    const float4* stats;    // [rows]
    int rows, V, parts, part;
    float temperature;
};
cudaError_t launch_spread(const SpreadArgs& a, int rows, int dtype, Stream& s);

struct PairArgs {
    const int32_t *offsets, *tokens;  // [2 pairs + 1], [rows]
    const float *logp, *ref, *weight, *pair_weight;  // [rows], [rows] or null, [rows] or null, [pairs] or null
    const float4* stats;     // [rows]
    float *loss, *sums;      // [pairs], [2 pairs]; null: not wanted
    float* slope;            // [rows] or null
    int rows, V, pairs, kind, interleaved;
    bool early;              // the kernel before triggers late (see pdl_wait)
    float beta, smoothing, margin;
};
// directly behind launch_token, which makes logp
cudaError_t launch_pairs(const PairArgs& a, Stream& s);

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
