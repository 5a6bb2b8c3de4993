// The K largest logits of a row, in order, and the logarithm of the mass of all others: what of a teacher's distribution is
// stored for a student.
//
// A CTA (or a cluster, see below) holds a row in shared memory.  Selection: a thread keeps the maximum of its own entries (or four, of
// parts of them); a key that k of these maxima reach is a lower bound for the k-th largest entry and close to it (256 maxima of 64
// of 16384 normal entries: 84 candidates for k = 64).  It comes from histograms of 256 bins over the maxima's keys, which narrow
// to one bin until few maxima are too many.  One more pass marks the groups with candidates and sums the exponentials of all others
// against the bound; the candidates go into bins over their own range, and those of one bin are counted against one another.  No
// difference of masses is taken: the rest keeps its digits however small it is.  Candidates that do not fit (an order of the row that
// puts the largest into few threads' entries, ties without end) are narrowed by histograms over the entries themselves.
// A row is read from HBM once; the barriers between these steps and their latency bound the kernel (three CTAs an SM, 14000 cycles
// a row of 16384 fp32, of which HBM would need 8500).  The next row is fetched while the list is put in order.  The CTAs of
// a cluster select from their slices; the first merges the lists.
#include "logit_rows.cuh"

namespace hbsjd {

namespace {

constexpr int BINS = 256;  // (eight per lane of the warp that scans them)
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
// and at most `limit` if that can be had; else the want-th largest itself.  No key lies beyond hi, and at least `want` reach lo.  The
// bins are clear, and all threads have met since.
template <int THREADS, typename Visit>
__device__ __forceinline__ uint32_t bound_key(uint32_t lo, uint32_t hi, int want, int limit, uint32_t* hist,
                                              Visit&& visit) {
    const int lane = threadIdx.x & 31;
    int more = 0;
    while (true) {
        const int shift = max(0, 24 - __clz(hi - lo));  // (hi - lo) >> shift < BINS
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
        for (int i = threadIdx.x; i < BINS; i += THREADS) hist[i] = 0;
        __syncthreads();
        more = total - inside;
        hi = min(hi, start + ((1u << shift) - 1));
        lo = start;
    }
}

constexpr int ALONE_SM = 160 * 1024;  // (lists and candidates of 1024 need 48 KB beside the row)

// CTAs of an SM, at most: three of 256 threads, which is what rows of 16384 fp32 leave room for, with the registers that they may
// have then (lists of 64 from 8192 such rows: 138 us, with 40 registers 148).
template <int THREADS>
constexpr int topk_ctas() {
    return THREADS == 256 ? 3 : THREADS == 32 ? 32 : 1536 / THREADS;
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, topk_ctas<THREADS>()) k_topk(TopkArgs a) {
    constexpr int G = 16 / sizeof(T), WARPS = THREADS / 32, SETS = 4;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ Mass rests[ROW_CTAS];  // of the slices
    __shared__ uint32_t hist[BINS + 3], red[3][WARPS];
    __shared__ float sums[WARPS];
    __shared__ int found, bad, big;        // candidates; a sum that is no number; one that is far from zero
    __shared__ uint32_t least_key, top_key;  // of the candidates
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, k = a.k, cap = a.cap;
    const int rank = blockIdx.x % a.ctas, v0 = rank * a.slice, n = max(0, min(a.slice, a.V - v0)), step = gridDim.x / a.ctas;
    const float inv_tau = 1.f / a.temperature, c = LOG2E * inv_tau;
    const f32x2 c2 = both(c);
    T* xs = (T*)smem;
    unsigned long long* cand = (unsigned long long*)(smem + (a.slice + 16) * sizeof(T));  // [cap]
    unsigned long long* other = cand + cap;   // [cap]
    unsigned long long* lists = other + cap;  // [ctas][k], several CTAs only
    if (tid == 0) {
        found = bad = big = 0;
        least_key = 0xffffffffu, top_key = 0;
    }
    if (a.ctas > 1) cluster_barrier();  // every CTA of the rows runs
    const auto source = [&](int row) { return (const T*)a.x + (int64_t)row * a.ld + v0; };
    // where a row's results go, -1: nowhere
    const auto target = [&](int row) -> int64_t {
        if (row >= a.rows) return -1;
        if (!a.at) return row;
        const int2 at = __ldcg(a.at + row);
        return at.x < 0 || at.y < __ldg(a.prefix_len + at.x) ? -1 : (int64_t)at.x * a.T + at.y;
    };
    int row = blockIdx.x / a.ctas;
    int64_t to = target(row);
    if (to >= 0) stage_row<T, THREADS>(xs, source(row), n, phase_of(source(row)));
    for (; row < a.rows; row += step) {
        const int64_t to1 = target(row + step);
        bool fetched = to1 < 0;
        const auto fetch = [&] {
            if (!fetched) stage_row<T, THREADS>(xs, source(row + step), n, phase_of(source(row + step)));
            fetched = true;
        };
        if (to < 0) {  // (all CTAs of the row)
            fetch();
            to = to1;
            continue;
        }
        const int P = phase_of(source(row)), groups = (P + n + G - 1) / G;
        cp_async_wait_all();
        for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;
        __syncthreads();
        if ((P + n) % G || P) {
            end_row<T, G>(xs, n, P, -INFINITY);
            __syncthreads();
        }
        const auto each = [&](auto&& f) {
#pragma unroll 4
            for (int j = tid; j < groups; j += THREADS) {
                float x[G];
                get<G>(xs + j * G, x);
                f(x, j);
            }
        };

        // ---- a bound that at least k entries reach
        uint32_t thr = LOWEST_KEY, top = 0;
        if (n > cap) {
            float best[SETS];
#pragma unroll
            for (int i = 0; i < SETS; ++i) best[i] = -INFINITY;
            int j = tid;
            for (; j + (SETS - 1) * THREADS < groups; j += THREADS * SETS) {
#pragma unroll
                for (int u = 0; u < SETS; ++u) {
                    float x[G];
                    get<G>(xs + (j + u * THREADS) * G, x);
#pragma unroll
                    for (int i = 0; i < G; ++i) best[u] = fmaxf(best[u], x[i]);
                }
            }
#pragma unroll
            for (int u = 0; u < SETS - 1; ++u)
                if (j + u * THREADS < groups) {
                    float x[G];
                    get<G>(xs + (j + u * THREADS) * G, x);
#pragma unroll
                    for (int i = 0; i < G; ++i) best[u] = fmaxf(best[u], x[i]);
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
                red[2][wid] = filled;
            }
            __syncthreads();
            lo = __reduce_min_sync(0xffffffffu, red[0][lane % WARPS]);
            top = __reduce_max_sync(0xffffffffu, red[1][lane % WARPS]);
            filled = __reduce_add_sync(0xffffffffu, lane < WARPS ? red[2][lane % WARPS] : 0);
            if (filled >= k)
                thr = bound_key<THREADS>(lo, top, k, k + max(16, k / 4), hist, [&](auto&& f) {
#pragma unroll
                    for (int i = 0; i < SETS; ++i)
                        if (i < sets) f(key[i]);
                });
        }
        // ---- candidates, and the mass of all others against the bound
        bool tied = false;  // too many entries equal the k-th: only those beyond it are candidates yet
        int reach = 0;      // (if so) the entries that reach it
        while (true) {
            const float t = value_of(thr);
            const f32x2 o = both(-t);
            f32x2 z2 = both(0.f);
            // A group that reaches the bound is only marked: some lane of a warp has one in half of the steps and more.
            uint32_t marks = 0;
            int step_no = 0;
            each([&](const float(&x)[G], int) {
                float most = x[0];
#pragma unroll
                for (int i = 1; i < G; ++i) most = fmaxf(most, x[i]);
                if (most >= t) marks |= 1u << step_no;
                ++step_no;
                if (a.rest) {
                    f32x2 e = both(0.f);
#pragma unroll
                    for (int i = 0; i < G; i += 2) e = add2(e, ex2(mul2(add2(both(x[i], x[i + 1]), o), c2)));
                    if (!(most >= t)) z2 = add2(z2, e);
                }
            });
            float z = sum2(z2);
            // The marked groups of a warp, a lane each, from a list of its own (in `other`, which is free here).
            uint16_t* list = (uint16_t*)other + wid * 64;
            for (int listed = 0;;) {
                uint32_t more = __ballot_sync(0xffffffffu, marks != 0);
                while (more && listed < 32) {
                    if (marks) list[listed + __popc(more & ((1u << lane) - 1))] = (uint16_t)(tid + (__ffs(marks) - 1) * THREADS);
                    marks &= marks - 1;
                    listed += __popc(more);
                    more = __ballot_sync(0xffffffffu, marks != 0);
                }
                if (!listed) break;
                __syncwarp();
                const int take = min(listed, 32);
                listed -= take;
                if (lane < take) {
                    const int j = list[listed + lane];
                    float x[G], lo = INFINITY, hi = -INFINITY;
                    get<G>(xs + j * G, x);
                    int some = 0;
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const bool in = x[i] >= t, kept = in && (!tied || x[i] > t);
                        if (!in) z += ex2((x[i] - t) * c);
                        some += kept;
                        lo = kept ? fminf(lo, x[i]) : lo;
                        hi = kept ? fmaxf(hi, x[i]) : hi;
                    }
                    if (some) {
                        int p = atomicAdd(&found, some);
                        atomicMin(&least_key, key_of(lo));
                        atomicMax(&top_key, key_of(hi));
#pragma unroll
                        for (int i = 0; i < G; ++i)
                            if (x[i] >= t && (!tied || x[i] > t)) {
                                if (p < cap) cand[p] = rank_key(x[i], v0 + j * G + i - P);
                                ++p;
                            }
                    }
                }
                __syncwarp();
            }
            z = sum_of_warp(z);
            if (lane == 0) {
                sums[wid] = z;
                if (!(z < 1e20f)) bad = 1;
                if (z > 1e-20f) big = 1;
            }
            for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;  // (for the order; the bound's were read before threads last met)
            __syncthreads();
            if (found <= cap) break;
            // the entries that reach the bound, narrowed until they fit; the k-th largest itself if they never do
            __syncthreads();
            if (tid == 0) {
                found = bad = big = 0;
                least_key = 0xffffffffu, top_key = 0;
            }
            thr = bound_key<THREADS>(thr, top, k, cap, hist, [&](auto&& f) {
                each([&](const float(&x)[G], int) {
#pragma unroll
                    for (int i = 0; i < G; ++i)
                        if (x[i] > -INFINITY) f(key_of(x[i]));
                });
            });
            // (where more than cap entries reach it still, it is the k-th largest: fewer than k lie above)
            reach = 0;
            const float u = value_of(thr);
            each([&](const float(&x)[G], int) {
#pragma unroll
                for (int i = 0; i < G; ++i) reach += x[i] >= u;
            });
            reach = __reduce_add_sync(0xffffffffu, reach);
            if (lane == 0) red[0][wid] = reach;
            __syncthreads();
            reach = __reduce_add_sync(0xffffffffu, lane < WARPS ? red[0][lane % WARPS] : 0);
            tied = reach > cap;
            __syncthreads();
        }
        int count = found;
        float t = value_of(thr), zr = -1.f;  // reference of the sum; the sum itself where it was taken again
        if (a.rest && (bad || !(big || thr == LOWEST_KEY))) {
            // NaN in the row, or all others far off the bound: again, against their largest and passing NaN over
            const float least = t;
            float m = -INFINITY, z = 0.f;
            each([&](const float(&x)[G], int) {
#pragma unroll
                for (int i = 0; i < G; ++i)
                    if (x[i] < least) m = fmaxf(m, x[i]);
            });
            m = max_of_warp(m);
            __syncthreads();
            if (lane == 0) sums[wid] = m;
            __syncthreads();
            m = max_of_warp(sums[lane % WARPS]);
            if (m > -INFINITY) {
                each([&](const float(&x)[G], int) {
#pragma unroll
                    for (int i = 0; i < G; ++i)
                        if (x[i] < least) z += ex2((x[i] - m) * c);
                });
                t = m;
            }
            z = sum_of_warp(z);
            __syncthreads();
            if (lane == 0) sums[wid] = z;
            __syncthreads();
            zr = sum_of_warp(lane < WARPS ? sums[lane % WARPS] : 0.f);
            if (tied && zr > 0.f) zr *= rescale(t, least, c);  // (the tied entries join it)
            if (tied) t = least;
        }
        if (tied) {  // the first of the tied entries, by index
            const float u = value_of(thr);
            for (int e0 = 0; e0 < P + n && count < k; e0 += THREADS) {
                const int e = e0 + tid;
                const bool is = e < P + n && to_f<T>(xs[e]) == u;
                const uint32_t b = __ballot_sync(0xffffffffu, is);
                if (lane == 0) red[0][wid] = __popc(b);
                __syncthreads();
                int place = count + __popc(b & ((1u << lane) - 1)), all = 0;
                for (int w = 0; w < WARPS; ++w) {
                    if (w < wid) place += red[0][w];
                    all += red[0][w];
                }
                if (is && place < k) cand[place] = rank_key(u, v0 + e - P);
                count = min(k, count + all);
                __syncthreads();
            }
        }
        if (tied) {
            if (tid == 0) least_key = thr, top_key = max(top_key, thr);
            for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;
            __syncthreads();
        }
        fetch();  // the row is read

        // ---- order
        // By bins over the candidates' keys (and tokens, where all are equal): what is in a higher bin comes first, those of one bin
        // are counted against one another.
        if (count > 1) {
            const uint32_t least = least_key;
            const auto place_of = [&](unsigned long long key) {  // value, then token, in the bits that differ
                return (unsigned long long)((uint32_t)(key >> 32) - least) << 17 | ((uint32_t)key & 0x1ffffu);
            };
            const int shift = max(0, 64 - __clzll((unsigned long long)(top_key - least) << 17 | 0x1ffffu) - 8);
            for (int q = tid; q < count; q += THREADS) atomicAdd(&hist[place_of(cand[q]) >> shift], 1u);
            __syncthreads();
            if (tid < 32) {  // how many are in higher bins; eight bins per lane, from the top
                uint32_t h[8], sum = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += h[i] = hist[BINS - 1 - (lane * 8 + i)];
                uint32_t upto = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += x;
                }
                upto -= sum;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    hist[BINS - 1 - (lane * 8 + i)] = upto;
                    upto += h[i];
                }
            }
            __syncthreads();
            for (int q = tid; q < count; q += THREADS) {
                const unsigned long long key = cand[q];
                other[atomicAdd(&hist[place_of(key) >> shift], 1u)] = key;
            }
            __syncthreads();
            for (int q = tid; q < count; q += THREADS) {
                const unsigned long long key = other[q];
                const int bin = (int)(place_of(key) >> shift), first = bin == BINS - 1 ? 0 : (int)hist[bin + 1], last = (int)hist[bin];
                int r = first;
                for (int j = first; j < last; ++j) r += other[j] > key;
                cand[r] = key;
            }
        }
        __syncthreads();  // (with one candidate, too: what is reset below was read)
        const unsigned long long* sorted = cand;
        if (tid == 0) {
            found = bad = big = 0;
            least_key = 0xffffffffu, top_key = 0;
        }
        float* values = a.values + to * k;
        int32_t* indices = a.indices + to * k;
        for (int i = tid; i < k; i += THREADS) {
            const unsigned long long key = i < count ? sorted[i] : 0;
            if (a.ctas == 1) {
                values[i] = key ? value_of((uint32_t)(key >> 32)) : -INFINITY;
                indices[i] = key ? (int32_t)(0xffffffffu - (uint32_t)key) : -1;
            } else {
                remote_store(remote_smem(lists + rank * k + i, 0), key);
            }
        }
        // ---- the rest: the sum over the row, and the candidates behind the k-th, against the largest
        Mass rest = {t, 0.f};
        if (wid == 0 && a.rest) {
            rest.z = zr >= 0.f ? zr : sum_of_warp(lane < WARPS ? sums[lane % WARPS] : 0.f);
            if (tied) rest.z += (float)(reach - count);
            if (count > k) {
                const float m = value_of((uint32_t)(sorted[k] >> 32));
                float z = 0.f;
                for (int i = k + lane; i < count; i += 32) {
                    const float x = value_of((uint32_t)(sorted[i] >> 32));
                    z += x == m ? 1.f : ex2((x - m) * c);
                }
                if (rest.z > 0.f) rest.z *= rescale(t, m, c);
                rest = {m, sum_of_warp(z) + rest.z};
            }
            if (rest.z == 0.f) rest.m = -INFINITY;
        }
        if (a.ctas == 1) {
            if (a.rest && tid == 0) a.rest[to] = rest.z == 0.f ? -INFINITY : fmaf(rest.m, inv_tau, LN2 * lg2(rest.z));
        } else {
            if (tid == 0) {
                const uint32_t place = remote_smem(&rests[rank], 0);
                remote_store(place, rest.m);
                remote_store(place + 4, rest.z);
            }
            posted(a.ctas);
            if (rank == 0) {
                // the lists of all slices: an entry's place is its own list's and, for each other, the entries that come first
                Mass mine = tid < a.ctas ? rests[tid] : Mass::none();
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
                Mass all = mine;
                all.share();
                all.z = sum_of_warp(mine.against(all, c).z);
                if (lane == 0) {
                    red[0][wid] = valid;
                    red[1][wid] = __float_as_uint(all.m);
                    sums[wid] = all.z;
                }
                __syncthreads();
                mine = lane < WARPS ? Mass{__uint_as_float(red[1][lane % WARPS]), sums[lane % WARPS]} : Mass::none();
                rest = mine;
                rest.share();
                rest.z = sum_of_warp(mine.against(rest, c).z);
                valid = __reduce_add_sync(0xffffffffu, lane < WARPS ? red[0][lane % WARPS] : 0);
                for (int i = valid + tid; i < k; i += THREADS) {
                    values[i] = -INFINITY;
                    indices[i] = -1;
                }
                if (a.rest && tid == 0) a.rest[to] = rest.z == 0.f ? -INFINITY : fmaf(rest.m, inv_tau, LN2 * lg2(rest.z));
            }
            // (the others' lists of the next row are to wait for these)
            cluster_barrier();
        }
        to = to1;
    }
}

// One CTA per image: empty lists for its prefix.
__global__ void k_topk_clear(TopkArgs a) {
    pdl_wait();
    pdl_trigger();
    const int64_t first = (int64_t)blockIdx.x * a.T;
    const int len = min(a.prefix_len[blockIdx.x], a.T);
    for (int64_t i = threadIdx.x; i < (int64_t)len * a.k; i += blockDim.x) {
        a.values[first * a.k + i] = -INFINITY;
        a.indices[first * a.k + i] = -1;
    }
    for (int i = threadIdx.x; i < len && a.rest; i += blockDim.x) a.rest[first + i] = -INFINITY;
}

template <typename T>
cudaError_t run_topk(TopkArgs& a, Stream& s) {
    constexpr int G = 16 / sizeof(T);
    a.cap = 512;
    while (a.cap < 2 * a.k) a.cap *= 2;
    const size_t smem = (a.slice + 16) * sizeof(T) + a.cap * 16 + (a.ctas > 1 ? (size_t)a.ctas * a.k * 8 : 0);
    const auto run = [&](auto threads) {
        constexpr int THREADS = decltype(threads)::value;
        cudaError_t e = allow_row_smem<k_topk<T, THREADS>>();
        if (e != cudaSuccess) return e;
        const int per_sm = std::max(1, std::min<int>(topk_ctas<THREADS>(), 227 * 1024 / (smem + 1024 + 1600)));  // (1 KB is the system's)
        int clusters = 0;
        e = resident_clusters<k_topk<T, THREADS>>(a.ctas, THREADS, per_sm, smem, a.rows, &clusters);
        if (e != cudaSuccess) return e;
        return launch_kc(true, k_topk<T, THREADS>, dim3((unsigned)clusters * a.ctas), dim3(THREADS), smem, s, a.ctas, a);
    };
    // Many rows: at most eighteen groups a thread (256 threads for the largest slice), as for the divergences (lists of 64 from 8192 rows of
    // 16384 fp32: 148 us with 256 threads, 185 with 512; from 16384 rows of 1000: 72 with one warp, 103 with four), and two
    // maxima per entry of the list.  Few rows: what is fastest for one (of 1000, lists of 64: 5 us with 256 threads, 7.6 with 64).
    const bool many = (int64_t)a.rows * a.ctas > device_sm_count();
    constexpr int MOST = 18;
    const int per = (many ? MOST : 4) * G;
    // (a thread marks its groups in the bits of a word; the row's place behind 16 bytes may take one more)
    static_assert(MOST < 32 && ALONE_SM >= SHARED_SM && ALONE_SM / 16 + 2 <= 32 * 512 && MAX_LOGIT_V / ROW_CTAS / G + 2 <= 32 * 512,
                  "512 threads have at most 32 groups each");
    if (many && a.slice <= 32 * per && a.k <= 64) return run(std::integral_constant<int, 32>());
    if (many && a.slice <= 64 * per && a.k <= 128) return run(std::integral_constant<int, 64>());
    if (many && a.slice <= 128 * per && a.k <= 256) return run(std::integral_constant<int, 128>());
    if (a.slice <= 256 * per && a.k <= 512) return run(std::integral_constant<int, 256>());
    return run(std::integral_constant<int, 512>());
}

}  // namespace

cudaError_t launch_topk_clear(const TopkArgs& a, int batch, Stream& s) {
    return launch_k(k_topk_clear, dim3(batch), dim3(512), 0, s, a);
}

cudaError_t launch_topk(const TopkArgs& args, int rows, int dtype, Stream& s) {
    TopkArgs a = args;
    // Few rows have an SM each, and one CTA to each as long as it holds them: joining lists costs more than it saves (a row of 16384 fp32,
    // lists of 64, on 1, 2, 4, 8 CTAs: 7.3, 8.6, 8.2, 20.6 us).
    const int sms = device_sm_count();
    const RowSplit sp = split_row(rows, a.V, dtype ? 2 : 4, sms, rows <= sms ? ALONE_SM : SHARED_SM, false);
    a.rows = rows, a.ctas = sp.ctas, a.slice = sp.slice;
    return dtype ? run_topk<bf16>(a, s) : run_topk<float>(a, s);
}

}  // namespace hbsjd
