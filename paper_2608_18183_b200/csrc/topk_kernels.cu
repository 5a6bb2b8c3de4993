// The K largest logits of a row, in order, and the logarithm of the mass of all others: what of a teacher's distribution is
// stored for a student.
//
// One CTA (or a cluster, see below) holds a row in shared memory.  Selection: a thread keeps the maxima of its own groups of
// entries; a key that K of these maxima reach is a lower bound for the K-th largest entry and close to it (512 groups of 32 of
// 16384 normal entries: 68 candidates for K = 64).  It comes from histograms of 256 bins over the maxima's keys, which narrow
// to one bin until few maxima are too many.  One more pass collects the candidates and sums the exponentials of all others
// against the bound, the candidates are ranked by counting or sorted, and those behind the K-th join the sum.  No difference
// of masses is taken: the rest keeps its digits however small it is.  Candidates that do not fit (an order of the row that puts
// the largest into few groups, ties without end) are narrowed by histograms over the entries themselves.
// A row is read from HBM once, which bounds the kernel.  The CTAs of a cluster select from their slices; the first merges the lists.
#include "logit_rows.cuh"

namespace hbsjd {

namespace {

constexpr int BINS = 256;
constexpr uint32_t LOWEST_KEY = 0x00800000u;  // of the lowest finite value; -inf and NaN lie below

// Order of the values as whole numbers; -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
// Larger value first, then the lower index.
__device__ __forceinline__ unsigned long long rank_key(float x, int index) {
    return (unsigned long long)key_of(x) << 32 | (0xffffffffu - (uint32_t)index);
}

// A bound for the `want`-th largest of the keys that visit(f) hands to f: all threads get a key that at least `want` keys reach,
// and at most `limit` if that can be had; else the want-th largest itself.  No key lies beyond hi, and at least `want` reach lo.
template <int THREADS, typename Visit>
__device__ __forceinline__ uint32_t bound_key(uint32_t lo, uint32_t hi, int want, int limit, uint32_t* hist,
                                              Visit&& visit) {
    const int lane = threadIdx.x & 31;
    int more = 0;
    while (true) {
        const int shift = max(0, 24 - __clz(hi - lo));  // (hi - lo) >> shift < BINS
        for (int i = threadIdx.x; i < BINS; i += THREADS) hist[i] = 0;
        __syncthreads();
        visit([&](uint32_t key) {
            if (key >= lo && key <= hi) atomicAdd(&hist[(key - lo) >> shift], 1u);
        });
        __syncthreads();
        if (threadIdx.x < 32) {  // bins from the top, eight per lane
            uint32_t h[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += h[i] = hist[BINS - 1 - (lane * 8 + i)];
            uint32_t upto = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            const uint32_t reach = __ballot_sync(0xffffffffu, (int)upto + more >= want);
            if (lane == (reach ? __ffs(reach) - 1 : 31)) {
                int before = (int)(upto - sum) + more, bin = 0, inside = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (before < want) {
                        bin = BINS - 1 - (lane * 8 + i);
                        inside = (int)h[i];
                        before += inside;
                    }
                hist[BINS] = bin;
                hist[BINS + 1] = before;   // keys that reach the bin
                hist[BINS + 2] = inside;
            }
        }
        __syncthreads();
        const int total = (int)hist[BINS + 1], inside = (int)hist[BINS + 2];
        const uint32_t start = lo + (hist[BINS] << shift);
        if (total <= limit || shift == 0) return start;
        more = total - inside;
        hi = min(hi, start + ((1u << shift) - 1));
        lo = start;
    }
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) k_topk(TopkArgs a, int cap) {
    constexpr int G = 16 / sizeof(T), WARPS = THREADS / 32, SETS = 4;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Mass slots[ROW_CTAS], slots_all[WARPS];  // the slices' rests; the warps' of what no list keeps
    __shared__ uint32_t hist[BINS + 3], red[2][WARPS];
    __shared__ float sums[WARPS];
    __shared__ int found;
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, k = a.k;
    const int64_t row = blockIdx.x / a.ctas;
    int64_t to = row;
    if (a.at) {
        const int2 at = __ldcg(a.at + row);
        if (at.x < 0 || at.y < a.prefix_len[at.x]) return;
        to = (int64_t)at.x * a.T + at.y;
    }
    if (a.ctas > 1) cluster_arrive();
    const int rank = blockIdx.x % a.ctas, v0 = rank * a.slice, n = max(0, min(a.slice, a.V - v0));
    const T* src = (const T*)a.x + row * a.ld + v0;
    const int P = phase_of(src), groups = (P + n + G - 1) / G;
    T* xs = (T*)smem;
    unsigned long long* cand = (unsigned long long*)(smem + (a.slice + 16) * sizeof(T));
    unsigned long long* lists = cand + cap;  // [ctas][k], several CTAs only
    stage_row<T, THREADS>(xs, src, n, P);
    if (tid == 0) found = 0;
    cp_async_wait_all();
    __syncthreads();
    if ((P + n) % G || P) {
        end_row<T, G>(xs, n, P, -INFINITY);
        __syncthreads();
    }

    // ---- a bound that at least k entries reach
    uint32_t thr = LOWEST_KEY;
    uint32_t top = 0;
    if (n > cap) {
        float best[SETS];
#pragma unroll
        for (int i = 0; i < SETS; ++i) best[i] = -INFINITY;
        for (int j0 = tid; j0 < groups; j0 += THREADS * SETS) {
#pragma unroll
            for (int u = 0; u < SETS; ++u) {
                const int j = j0 + u * THREADS;
                if (j < groups) {
                    float x[G];
                    get<G>(xs + j * G, x);
#pragma unroll
                    for (int i = 0; i < G; ++i) best[u] = fmaxf(best[u], x[i]);
                }
            }
        }
        int sets = SETS;
        if (k * 4 <= THREADS) {  // enough threads: one set each
            best[0] = fmaxf(fmaxf(best[0], best[1]), fmaxf(best[2], best[3]));
            sets = 1;
        }
        uint32_t key[SETS], lo = 0xffffffffu;
        int filled = 0;
#pragma unroll
        for (int i = 0; i < SETS; ++i) {
            key[i] = key_of(best[i]);
            if (i < sets && key[i] >= LOWEST_KEY) {
                lo = min(lo, key[i]);
                top = max(top, key[i]);
                ++filled;
            }
        }
        lo = __reduce_min_sync(0xffffffffu, lo);
        top = __reduce_max_sync(0xffffffffu, top);
        filled = __reduce_add_sync(0xffffffffu, filled);
        if (lane == 0) {
            red[0][wid] = lo;
            red[1][wid] = top;
            hist[wid] = filled;
        }
        __syncthreads();
        lo = __reduce_min_sync(0xffffffffu, red[0][lane % WARPS]);
        top = __reduce_max_sync(0xffffffffu, red[1][lane % WARPS]);
        filled = __reduce_add_sync(0xffffffffu, lane < WARPS ? hist[lane % WARPS] : 0);
        __syncthreads();  // (hist is cleared next)
        if (filled >= k)
            thr = bound_key<THREADS>(lo, top, k, k + max(16, k / 4), hist, [&](auto&& f) {
#pragma unroll
                for (int i = 0; i < SETS; ++i)
                    if (i < sets) f(key[i]);
            });
    }
    // ---- candidates, and the mass of all others against the bound
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    const f32x2 c2 = both(c);
    float z, t;
    bool tied = false;  // too many entries equal the k-th: only those beyond it are candidates yet
    int reach = 0;      // (if so) the entries that reach it
    while (true) {
        t = value_of(thr);
        const f32x2 o = both(-t);
        f32x2 z2 = both(0.f);
        for (int j = tid; j < groups; j += THREADS) {
            float x[G];
            get<G>(xs + j * G, x);
            float most = x[0];
#pragma unroll
            for (int i = 1; i < G; ++i) most = fmaxf(most, x[i]);
            if (most >= t) {
#pragma unroll
                for (int i = 0; i < G; ++i)
                    if (x[i] >= t) {
                        if (!tied || x[i] > t) {
                            const int p = atomicAdd(&found, 1);
                            if (p < cap) cand[p] = rank_key(x[i], v0 + j * G + i - P);
                        }
                        x[i] = -INFINITY;
                    }
            }
            if (a.rest) {
#pragma unroll
                for (int i = 0; i < G; i += 2) z2 = add2(z2, ex2(mul2(add2(both(x[i], x[i + 1]), o), c2)));
            }
        }
        z = sum2(z2);
        __syncthreads();
        if (found <= cap) break;
        // the entries that reach the bound, narrowed until they fit; the k-th largest itself if they never do
        __syncthreads();
        if (tid == 0) found = 0;
        thr = bound_key<THREADS>(thr, top, k, cap, hist, [&](auto&& f) {
            for (int j = tid; j < groups; j += THREADS) {
                float x[G];
                get<G>(xs + j * G, x);
#pragma unroll
                for (int i = 0; i < G; ++i)
                    if (x[i] > -INFINITY) f(key_of(x[i]));
            }
        });
        // (where more than cap entries reach it still, it is the k-th largest: fewer than k lie above)
        reach = 0;
        const float u = value_of(thr);
        for (int j = tid; j < groups; j += THREADS) {
            float x[G];
            get<G>(xs + j * G, x);
#pragma unroll
            for (int i = 0; i < G; ++i) reach += x[i] >= u;
        }
        reach = __reduce_add_sync(0xffffffffu, reach);
        if (lane == 0) red[0][wid] = reach;
        __syncthreads();
        reach = __reduce_add_sync(0xffffffffu, lane < WARPS ? red[0][lane % WARPS] : 0);
        tied = reach > cap;
        __syncthreads();
    }
    int count = found;
    if (tied) {  // the first of the tied entries, by index
        for (int e0 = 0; e0 < P + n && count < k; e0 += THREADS) {
            const int e = e0 + tid;
            const bool is = e < P + n && to_f<T>(xs[e]) == t;
            const uint32_t b = __ballot_sync(0xffffffffu, is);
            if (lane == 0) red[0][wid] = __popc(b);
            __syncthreads();
            int place = count + __popc(b & ((1u << lane) - 1)), all = 0;
            for (int w = 0; w < WARPS; ++w) {
                if (w < wid) place += red[0][w];
                all += red[0][w];
            }
            if (is && place < k) cand[place] = rank_key(t, v0 + e - P);
            count = min(k, count + all);
            __syncthreads();
        }
        if (tid == 0) z += (float)(reach - count);  // those that were not taken
    }
    __syncthreads();

    // ---- order
    float* values = a.values + to * k;
    int32_t* indices = a.indices + to * k;
    const auto place = [&](int r, unsigned long long key) {
        if (a.ctas == 1) {
            values[r] = key ? value_of((uint32_t)(key >> 32)) : -INFINITY;
            indices[r] = key ? (int32_t)(0xffffffffu - (uint32_t)key) : -1;
        } else {
            remote_store(remote_smem(lists + rank * k + r, 0), key);
        }
    };
    if (a.ctas > 1) cluster_wait();  // every CTA of the row runs
    const unsigned long long* sorted = cand;
    if ((int64_t)count * count <= 128 * THREADS) {
        int per = 1;  // threads per candidate
        while (per < 32 && per * 2 * count <= THREADS) per *= 2;
        const int i = tid / per;
        const unsigned long long key = i < count ? cand[i] : 0;
        int r = 0;
        for (int j = tid % per; j < count; j += per) r += cand[j] > key;
        for (int o = 1; o < per; o <<= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
        // (cand holds 1024 or more, count is at most 256: the atomics' order ends here)
        if (i < count && tid % per == 0) cand[512 + r] = key;
        sorted = cand + 512;
        __syncthreads();
    } else {
        int size = 1;
        while (size < count) size *= 2;
        for (int i = count + tid; i < size; i += THREADS) cand[i] = 0;
        for (int span = 2; span <= size; span *= 2)
            for (int o = span / 2; o > 0; o /= 2) {
                __syncthreads();
                for (int p = tid; p < size / 2; p += THREADS) {
                    const int i = 2 * o * (p / o) + p % o;
                    const unsigned long long x = cand[i], y = cand[i + o];
                    if ((x < y) == ((i & span) == 0)) {
                        cand[i] = y;
                        cand[i + o] = x;
                    }
                }
            }
        __syncthreads();
    }
    // (where every entry is a candidate, none was summed yet, and the bound is no entry)
    if (thr == LOWEST_KEY && count > k) t = value_of((uint32_t)(sorted[k - 1] >> 32));
    for (int i = tid; i < max(count, k); i += THREADS)
        if (i < k)
            place(i, i < count ? sorted[i] : 0);
        else  // a candidate behind the k-th
            z += ex2((value_of((uint32_t)(sorted[i] >> 32)) - t) * c);

    // ---- the rest
    Mass rest = {t, 0.f};
    if (a.rest) {
        z = sum_of_warp(z);
        if (lane == 0) sums[wid] = z;
        __syncthreads();
        rest.z = sum_of_warp(lane < WARPS ? sums[lane % WARPS] : 0.f);
        // NaN in the row, or all of the rest far off the bound: again, against its largest and passing NaN over
        if (!(rest.z > 1e-20f && rest.z < 1e20f)) {
            const auto each = [&](auto&& f) {
                for (int j = tid; j < groups; j += THREADS) {
                    float x[G];
                    get<G>(xs + j * G, x);
#pragma unroll
                    for (int i = 0; i < G; ++i)
                        if (x[i] < value_of(thr)) f(x[i], 1.f);
                }
                for (int i = k + tid; i < count; i += THREADS) f(value_of((uint32_t)(sorted[i] >> 32)), 1.f);
                if (tied && tid == 0 && reach > count) f(t, (float)(reach - count));
            };
            float m = -INFINITY;
            each([&](float x, float) { m = fmaxf(m, x); });
            m = max_of_warp(m);
            __syncthreads();
            if (lane == 0) sums[wid] = m;
            __syncthreads();
            m = max_of_warp(sums[lane % WARPS]);
            z = 0.f;
            const float o = m == -INFINITY ? 0.f : m;
            each([&](float x, float times) { z += x == m ? times : times * ex2((x - o) * c); });
            z = sum_of_warp(z);
            __syncthreads();
            if (lane == 0) sums[wid] = z;
            __syncthreads();
            rest = {m, m == -INFINITY ? 0.f : sum_of_warp(lane < WARPS ? sums[lane % WARPS] : 0.f)};
        }
    }
    if (a.ctas > 1) {
        if (tid == 0) {
            const uint32_t place = remote_smem(&slots[rank], 0);
            remote_store(place, rest.m);
            remote_store(place + 4, rest.z);
        }
        posted(a.ctas);
        if (rank) return;
        // the lists of all slices: an entry's place is its own list's and, for each other, the entries that come first
        Mass mine = Mass::none();
        int valid = 0;
        for (int i = tid; i < a.ctas * k; i += THREADS) {
            const unsigned long long key = lists[i];
            if (!key) continue;
            ++valid;
            int r = i % k;
            for (int l = 0; l < a.ctas; ++l) {
                if (l == i / k) continue;
                const unsigned long long* list = lists + l * k;
                int first = 0, last = k;  // entries before `first` are larger, those from `last` on are not
                while (first < last) {
                    const int mid = (first + last) / 2;
                    if (list[mid] > key)
                        first = mid + 1;
                    else
                        last = mid;
                }
                r += first;
            }
            if (r < k) {
                values[r] = value_of((uint32_t)(key >> 32));
                indices[r] = (int32_t)(0xffffffffu - (uint32_t)key);
            } else {
                mine = merge(mine, {value_of((uint32_t)(key >> 32)), 1.f}, c);
            }
        }
        valid = __reduce_add_sync(0xffffffffu, valid);
        if (lane == 0) red[0][wid] = valid;
        if (tid < a.ctas) mine = merge(mine, slots[tid], c);
        Mass all = mine;
        all.share();
        all.z = sum_of_warp(mine.against(all, c).z);
        if (lane == 0) slots_all[wid] = all;
        __syncthreads();
        mine = lane < WARPS ? slots_all[lane] : Mass::none();
        rest = mine;
        rest.share();
        rest.z = sum_of_warp(mine.against(rest, c).z);
        valid = __reduce_add_sync(0xffffffffu, lane < WARPS ? red[0][lane % WARPS] : 0);
        for (int i = valid + tid; i < k; i += THREADS) {
            values[i] = -INFINITY;
            indices[i] = -1;
        }
    }
    if (a.rest && tid == 0)
        a.rest[to] = rest.z == 0.f ? -INFINITY : fmaf(rest.m, inv_tau, LN2 * log2f(rest.z));
}

template <typename T>
cudaError_t run_topk(const TopkArgs& a, int rows, Stream& s) {
    constexpr int G = 16 / sizeof(T);
    int cap = 1024;
    while (cap < 4 * a.k) cap *= 2;
    const size_t smem = (a.slice + 16) * sizeof(T) + cap * 8 + (a.ctas > 1 ? (size_t)a.ctas * a.k * 8 : 0);
    const auto run = [&](auto threads) {
        constexpr int THREADS = decltype(threads)::value;
        const cudaError_t e = allow_row_smem<k_topk<T, THREADS>>();
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_topk<T, THREADS>, dim3((unsigned)rows * a.ctas), dim3(THREADS), smem, s, a.ctas, a, cap);
    };
    // at least eight groups a thread, and two maxima per entry of the list
    if (a.slice <= 8 * 128 * G && a.k <= 256) return run(std::integral_constant<int, 128>());
    if (a.slice <= 8 * 256 * G && a.k <= 512) return run(std::integral_constant<int, 256>());
    return run(std::integral_constant<int, 512>());
}

}  // namespace

cudaError_t launch_topk(const TopkArgs& args, int rows, int dtype, Stream& s) {
    TopkArgs a = args;
    const RowSplit sp = split_row(rows, a.V, dtype ? 2 : 4, device_sm_count());
    a.ctas = sp.ctas, a.slice = sp.slice;
    return dtype ? run_topk<bf16>(a, rows, s) : run_topk<float>(a, rows, s);
}

}  // namespace hbsjd
