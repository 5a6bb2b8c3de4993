// The norm of many arrays as one vector, and their scaling by it.
//
// Two kernels: k_norm reads every element once and leaves a part a CTA, k_clip joins the parts, has the norm and the factor
// min(1, limit / (norm + 1e-6)), and scales.  What has to be scaled is read a second time, which bounds it; the last that k_norm read is the first
// that k_clip does, so that arrays within L2 come from there.  Arrays are cut into chunks of 64 KB from a 16-byte boundary on, dealt to two CTAs of 512
// threads an SM; a thread has its eight vectors of a chunk on their way at once.  Sums of a chunk are in fp32, of chunks in 64 bits.  Measured: 343
// million fp32 elements into other arrays 670 us (0.95 of two readings and a writing at a copy's rate), 110 million bf16 below the limit 40 us (0.85).
#include "clip.cuh"

namespace hbsjd {

namespace {

constexpr int CLIP_THREADS = 512, CLIP_VECTORS = 8;             // a chunk: vectors of 16 bytes a thread
constexpr int CHUNK = CLIP_THREADS * CLIP_VECTORS * 16;         // bytes

// A launch's arrays, in its parameters: nothing is copied to the device, and a captured call needs no memory of the host's.
template <int N>
struct ClipList {
    const void* in[N];
    void* out[N];
    int64_t n[N];
    int32_t chunk[N + 1];  // first chunk of an array
    uint8_t wide[N];       // fp32
    int count;
};

// An array's chunk: vectors of 16 bytes from `base`, of which elements [lo, hi) (from base) are the array's.
template <typename T>
struct Chunk {
    const T* base;
    T* out;
    int lo, hi;
    bool alike;  // out lies as `in` does behind a 16-byte boundary
    template <typename L>
    __device__ __forceinline__ Chunk(const L& list, int i, int at) {
        constexpr int VEC = 16 / sizeof(T), E = CHUNK / sizeof(T);
        const T* in = (const T*)list.in[i];
        const int P = phase_of(in);
        const int64_t from = (int64_t)at * E - P;  // of the array; below 0 for what lies in front of it
        base = in + from;
        out = (T*)list.out[i] + from;
        lo = from < 0 ? (int)-from : 0;
        hi = (int)min((int64_t)E, list.n[i] - from);
        alike = phase_of((const T*)list.out[i]) == P;
        static_assert(VEC * CLIP_THREADS * CLIP_VECTORS == E, "a chunk is a round of the CTA");
    }
    // elements of vector j that are the array's
    __device__ __forceinline__ bool whole(int j) const { return j * VEC() >= lo && (j + 1) * VEC() <= hi; }
    __device__ __forceinline__ static constexpr int VEC() { return 16 / sizeof(T); }
    __device__ __forceinline__ uint4 load(int j, bool last = false) const {
        // (for the last time: not as what no one writes, since a gradient may be scaled in its place)
        if (whole(j)) return last ? reinterpret_cast<const uint4*>(base)[j] : __ldg(reinterpret_cast<const uint4*>(base) + j);
        uint4 v = {0, 0, 0, 0};
        T* x = reinterpret_cast<T*>(&v);
#pragma unroll
        for (int e = 0; e < VEC(); ++e)
            if (j * VEC() + e >= lo && j * VEC() + e < hi) x[e] = base[j * VEC() + e];
        return v;
    }
};

__device__ __forceinline__ void values(const uint4& v, float (&x)[4], float) {
    x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void values(const uint4& v, float (&x)[8], bf16) {
    unpack(v.x, x[0], x[1]);
    unpack(v.y, x[2], x[3]);
    unpack(v.z, x[4], x[5]);
    unpack(v.w, x[6], x[7]);
}

// The array of a chunk.
template <typename L>
__device__ __forceinline__ int array_of(const L& list, int chunk) {
    int lo = 0, hi = list.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (list.chunk[mid] <= chunk)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// A thread's sum of squares of a chunk.  In 32 bits where these neither overflow nor vanish there, else in 64.
template <typename T, typename L>
__device__ __forceinline__ double squares(const L& list, int i, int at) {
    constexpr int VEC = 16 / sizeof(T);
    const Chunk<T> c(list, i, at);
    uint4 v[CLIP_VECTORS];
#pragma unroll
    for (int u = 0; u < CLIP_VECTORS; ++u) v[u] = c.load(u * CLIP_THREADS + threadIdx.x);
    f32x2 s = both(0.f);
    uint32_t any = 0;
#pragma unroll
    for (int u = 0; u < CLIP_VECTORS; ++u) {
        float x[VEC];
        values(v[u], x, T());
        any |= v[u].x | v[u].y | v[u].z | v[u].w;
#pragma unroll
        for (int e = 0; e < VEC; e += 2) s = fma2(both(x[e], x[e + 1]), both(x[e], x[e + 1]), s);
    }
    const float sum = sum2(s);
    if ((sum > 1e-26f && sum < 1e30f) || !(any << 1)) return sum;
    double wide = 0.0;
#pragma unroll
    for (int u = 0; u < CLIP_VECTORS; ++u) {
        float x[VEC];
        values(v[u], x, T());
#pragma unroll
        for (int e = 0; e < VEC; ++e) wide = fma((double)x[e], (double)x[e], wide);
    }
    return wide;
}
// A thread's largest magnitude of a chunk, as bits: those of NaN are above all others.
template <typename T, typename L>
__device__ __forceinline__ uint32_t largest(const L& list, int i, int at) {
    constexpr int VEC = 16 / sizeof(T);
    const Chunk<T> c(list, i, at);
    uint4 v[CLIP_VECTORS];
#pragma unroll
    for (int u = 0; u < CLIP_VECTORS; ++u) v[u] = c.load(u * CLIP_THREADS + threadIdx.x);
    uint32_t most = 0;
#pragma unroll
    for (int u = 0; u < CLIP_VECTORS; ++u) {
        float x[VEC];
        values(v[u], x, T());
#pragma unroll
        for (int e = 0; e < VEC; ++e) most = max(most, __float_as_uint(x[e]) & 0x7fffffffu);
    }
    return most;
}

// The block's sum (or maximum), in every thread of warp 0.
__device__ __forceinline__ double join(double v, bool max_norm, double* parts) {
    const int lane = threadIdx.x & 31;
    const auto with = [&](double x, double y) { return !max_norm ? x + y : y > x || y != y ? y : x; };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = with(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (lane == 0) parts[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < CLIP_THREADS / 32 ? parts[lane] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = with(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

template <int N>
__global__ void __launch_bounds__(CLIP_THREADS, 2) k_norm(const __grid_constant__ ClipList<N> list, int chunks, int max_norm, double* parts) {
    __shared__ double shared[CLIP_THREADS / 32];
    pdl_wait();
    pdl_trigger();
    double sum = 0.0;
    uint32_t most = 0;
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int i = array_of(list, c), at = c - list.chunk[i];
        if (max_norm)
            most = max(most, list.wide[i] ? largest<float>(list, i, at) : largest<bf16>(list, i, at));
        else
            sum += list.wide[i] ? squares<float>(list, i, at) : squares<bf16>(list, i, at);
    }
    const double v = join(max_norm ? (double)__uint_as_float(most) : sum, max_norm, shared);
    if (threadIdx.x == 0) parts[blockIdx.x] = v;
}

template <typename T, typename L>
__device__ __forceinline__ void scaled(const L& list, int i, int at, float f) {
    constexpr int VEC = 16 / sizeof(T);
    const Chunk<T> c(list, i, at);
    uint4 v[CLIP_VECTORS];
#pragma unroll
    for (int u = 0; u < CLIP_VECTORS; ++u) v[u] = c.load(u * CLIP_THREADS + threadIdx.x, true);
#pragma unroll
    for (int u = 0; u < CLIP_VECTORS; ++u) {
        const int j = u * CLIP_THREADS + threadIdx.x;
        if (f != 1.f) {  // (else the same bits, of NaN too)
            float x[VEC];
            values(v[u], x, T());
            if constexpr (VEC == 4)
                v[u] = make_uint4(__float_as_uint(x[0] * f), __float_as_uint(x[1] * f), __float_as_uint(x[2] * f), __float_as_uint(x[3] * f));
            else
                v[u] = make_uint4(pack(x[0] * f, x[1] * f), pack(x[2] * f, x[3] * f), pack(x[4] * f, x[5] * f), pack(x[6] * f, x[7] * f));
        }
        if (c.alike && c.whole(j)) {
            __stcs(reinterpret_cast<uint4*>(c.out) + j, v[u]);
        } else {
            const T* x = reinterpret_cast<const T*>(&v[u]);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (j * VEC + e >= c.lo && j * VEC + e < c.hi) c.out[j * VEC + e] = x[e];
        }
    }
}

template <int N>
__global__ void __launch_bounds__(CLIP_THREADS, 2) k_clip(const __grid_constant__ ClipList<N> list, int chunks, int max_norm, const double* parts,
                                                          int count, float limit, int copy, float* norm) {
    __shared__ double shared[CLIP_THREADS / 32];
    __shared__ float factor;
    pdl_wait();
    pdl_trigger();
    double v = 0.0;
    for (int i = threadIdx.x; i < count; i += CLIP_THREADS) {
        const double x = __ldcg(parts + i);
        v = !max_norm ? v + x : x > v || x != x ? x : v;
    }
    v = join(v, max_norm, shared);
    if (threadIdx.x == 0) {
        if (!max_norm) v = sqrt(v);
        if (norm && blockIdx.x == 0) *norm = (float)v;
        const double f = limit / (v + 1e-6);
        factor = isfinite((float)v) && f < 1.0 ? (float)f : 1.f;  // (a norm that is no number, as it is given out, scales nothing)
    }
    __syncthreads();
    const float f = factor;
    if (f == 1.f && !copy) return;
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int c = chunks - 1 - k, i = array_of(list, c), at = c - list.chunk[i];
        if (list.wide[i])
            scaled<float>(list, i, at, f);
        else
            scaled<bf16>(list, i, at, f);
    }
}

template <int N>
int fill(ClipList<N>& list, const ClipArray* arrays, int count) {
    int64_t chunks = 0;
    for (int i = 0; i < count; ++i) {
        const ClipArray& x = arrays[i];
        list.in[i] = x.in;
        list.out[i] = x.out;
        list.n[i] = x.n;
        list.wide[i] = x.bytes == 4;
        list.chunk[i] = (int32_t)chunks;
        chunks += ((int64_t)((uintptr_t)x.in % 16) + x.n * x.bytes + CHUNK - 1) / CHUNK;
    }
    list.chunk[count] = (int32_t)chunks;
    list.count = count;
    return (int)chunks;
}

// CTAs of a launch, two an SM; each of k_norm's leaves a part
int norm_ctas(int chunks) { return std::min(chunks, std::min(CLIP_PARTS, 2 * device_sm_count())); }

template <int N>
cudaError_t run_clip(const ClipArray* arrays, int count, const ClipArgs& a, Stream& s) {
    cudaError_t e = cudaSuccess;
    const int launches = (count + N - 1) / N;
    int parts = 0;
    ClipList<N> list;
    for (int l = 0; l < launches && e == cudaSuccess; ++l) {
        const int chunks = fill(list, arrays + l * N, std::min(N, count - l * N)), ctas = norm_ctas(chunks);
        e = launch_k(k_norm<N>, dim3((unsigned)ctas), dim3(CLIP_THREADS), 0, s, list, chunks, a.max_norm, a.parts + parts);
        parts += ctas;
    }
    for (int l = launches - 1; l >= 0 && e == cudaSuccess; --l) {
        if (launches > 1) fill(list, arrays + l * N, std::min(N, count - l * N));
        const int chunks = list.chunk[list.count];
        // (nothing to scale: one CTA joins the parts)
        const int ctas = a.scale ? norm_ctas(chunks) : 1;
        if (!a.scale && l) continue;
        e = launch_k(k_clip<N>, dim3((unsigned)ctas), dim3(CLIP_THREADS), 0, s, list, a.scale ? chunks : 0, a.max_norm, (const double*)a.parts, parts, a.limit,
                     a.copy, l ? nullptr : a.norm);
    }
    return e;
}

}  // namespace

int clip_launches(int count) { return count <= CLIP_FEW ? 1 : (count + CLIP_MANY - 1) / CLIP_MANY; }

int64_t clip_chunks(const ClipArray* arrays, int count) {
    int64_t chunks = 0;
    for (int i = 0; i < count; ++i) chunks += (arrays[i].n * arrays[i].bytes + 16 + CHUNK - 1) / CHUNK;
    return chunks;
}

cudaError_t launch_clip(const ClipArray* arrays, int count, const ClipArgs& a, Stream& s) {
    return count <= CLIP_FEW ? run_clip<CLIP_FEW>(arrays, count, a, s) : run_clip<CLIP_MANY>(arrays, count, a, s);
}

}  // namespace hbsjd
