// The K largest logits of each row, ids and values, falling, the lowest index first among equals.
//
// A row is read once.  A sample of it (16384 values in 128-byte runs spread over the row, which L2 still has when the pass
// behind comes to them, as that leaves L2 first: load_once) yields a cut: each of the 512 (short rows: 256) threads keeps its
// share's maximum, and the K-th largest of those maxima has K values of the row at or above it, whatever the row looks like.
// The pass keeps what is not below the cut -- some 10 K of 151936 values -- in shared memory, one compare for four values.
// The K best of those are found by a histogram of their keys, 256 bins over the range that they span, narrowed to the bin
// that holds the K-th until it is decided, and put in order by counting.  A row that overfills the list (long ties, a sample
// that says nothing about the row) is selected exactly instead, by four passes over the digits of the key and one that
// collects in order of index.  The key is the value's bits in an order of whole numbers: NaN below everything, -0 equal to 0.
//
// The reading bounds it where the rows are many and long: 2048 rows of 151936, the 64 best, 222 us or 0.86 of the measured
// copy rate.  Few or short rows are a chain of steps, each a meeting of the block: one row 9 us, 32 rows 17.
//
// With few rows a cluster of up to eight blocks shares one, each a slice with a cut of its own, and the first block selects
// among what they kept.
#include <math.h>

#include "sm100.cuh"

namespace toplogits {

constexpr int MAX_TOP = 128;
constexpr int MAX_CLUSTER = 8;
constexpr int RUN = 32, SAMPLE_RUNS = 512; // values of a sampled run, runs of a sample

// T: threads of a block.
template <int T>
constexpr int LIST = 8 * T;                // candidates that a block holds
template <int T>
constexpr int SENT = LIST<T> / MAX_CLUSTER;    // of them, those that a block of a cluster sends as they are

__device__ __forceinline__ uint32_t key_of(float v) {
    uint32_t b = __float_as_uint(v);
    if (b == 0x80000000u) b = 0;
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

template <int T>
struct Shared {
    uint32_t key[LIST<T>], idx[LIST<T>];
    uint32_t best_key[MAX_TOP], best_idx[MAX_TOP];
    int hist[256];
    int part[2][T / 32];
    int count, found, bin, above;
    uint32_t low, high;
    int sent[MAX_CLUSTER];                 // behind it, with clusters: what the blocks sent, [MAX_CLUSTER][SENT<T>] keys, then indices
};

// The bin that holds the need-th largest of the values counted in s.hist, and how many lie in bins above it: s.bin, s.above.
// A warp's work; 1 <= need <= their number.
template <int T>
__device__ __forceinline__ void find_bin(Shared<T>& s, int need) {
    const int lane = threadIdx.x & 31;
    int n[8], sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += n[i] = s.hist[255 - lane * 8 - i];       // lane 0 has the highest bins
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    int above = upto - sum;
    if (above < need && need <= upto) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (above < need && need <= above + n[i]) {
                s.bin = 255 - lane * 8 - i;
                s.above = above;
            }
            above += n[i];
        }
    }
}
template <int T>
__device__ __forceinline__ void clear_bins(Shared<T>& s) {
    for (int i = threadIdx.x; i < 256; i += T) s.hist[i] = 0;
}
// Bits of the differences from `low` behind the eight that number the bins of [low, high].
__device__ __forceinline__ int bin_shift(uint32_t low, uint32_t high) { return max(0, 24 - __clz(high - low)); }

struct Cut {
    uint32_t low;                          // the values above the bin are the (need at the start - need) largest
    int need;                              // still to come from the bin that starts at `low`
    bool exact;                            // it holds just as many
};
// Narrows [low, high] to the bin that holds the need-th largest of the values value(j, v), j < n (false: no value), until it
// is decided or the bins are 2^stop wide.
template <int T, typename F>
__device__ __forceinline__ Cut narrow(Shared<T>& s, int n, F value, uint32_t low, uint32_t high, int need, int stop) {
    int shift = bin_shift(low, high);
    uint32_t span = high - low;
    for (;;) {
        clear_bins(s);
        __syncthreads();
        for (int j = threadIdx.x; j < n; j += T) {
            uint32_t v;
            if (value(j, v) && v >= low && v - low <= span) atomicAdd(&s.hist[(v - low) >> shift], 1);
        }
        __syncthreads();
        if (threadIdx.x < 32) find_bin(s, need);
        __syncthreads();
        need -= s.above;
        low += (uint32_t)s.bin << shift;
        const bool exact = s.hist[s.bin] == need;
        __syncthreads();                   // all of this has been read before the next pass writes it
        if (exact || shift <= stop) return {low, need, exact};
        span = (1u << shift) - 1u;
        shift = max(0, shift - 8);
    }
}

// The k best of the n <= LIST<T> entries of keys / idxs, whose keys lie in [low, high]: to best_key / best_idx in any order.
// Returns how many (min(n, k)).
template <int T>
__device__ int select(Shared<T>& s, const uint32_t* keys, const uint32_t* idxs, int n, int k, uint32_t low, uint32_t high) {
    const int tid = threadIdx.x;
    if (tid == 0) s.found = 0;
    Cut cut = {0, 0, true};                // taken: all
    uint32_t least = 0;                    // of the entries that equal the cut: those whose index, inverted, is not less
    if (n > k) {
        cut = narrow(s, n, [&](int j, uint32_t& v) { v = keys[j]; return true; }, low, high, k, 0);
        if (!cut.exact)                    // one key, more often than needed
            least = narrow(s, n, [&](int j, uint32_t& v) { v = ~idxs[j]; return keys[j] == cut.low; }, 0u, ~0u, cut.need, 0).low;
    }
    __syncthreads();
    for (int j = tid; j < n; j += T)
        if (keys[j] > cut.low || (keys[j] == cut.low && ~idxs[j] >= least)) {
            const int at = atomicAdd(&s.found, 1);
            s.best_key[at] = keys[j];
            s.best_idx[at] = idxs[j];
        }
    __syncthreads();
    return min(n, k);
}

// What comes so leaves L2 first, and the runs of the sample are still there when the pass comes to them (512 rows of 151936:
// 356 MB read from HBM without it, 315 with it, of 311; a tenth of the time of 2048 rows).
__device__ __forceinline__ float4 load_once(const float4* p) {
    float4 x;
    asm volatile("ld.global.cs.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "l"(p) : "memory");
    return x;
}
// Calls f4(four values, the first one's index) for the values [lo, hi) of the row, 16 bytes at a time where the alignment
// allows it, and f(value, index) for the rest.
template <int T, typename F4, typename F>
__device__ __forceinline__ void for_values(const float* row, int lo, int hi, F4 f4, F f) {
    const int tid = threadIdx.x;
    const int skew = (int)((4 - ((reinterpret_cast<uintptr_t>(row + lo) >> 2) & 3)) & 3);
    const int v0 = min(lo + skew, hi), nv = (hi - v0) / 4;
    if (tid < v0 - lo) f(row[lo + tid], lo + tid);
    const float4* vec = reinterpret_cast<const float4*>(row + v0);
    int i = tid;
    for (; i + 3 * T < nv; i += 4 * T) {
        float4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = load_once(vec + i + j * T);
#pragma unroll
        for (int j = 0; j < 4; ++j) f4(x[j], v0 + 4 * (i + j * T));
    }
    for (; i < nv; i += T) f4(vec[i], v0 + 4 * i);
    const int rest = v0 + 4 * nv + tid;
    if (rest < hi) f(row[rest], rest);
}
template <int T, typename F>
__device__ __forceinline__ void for_values(const float* row, int lo, int hi, F f) {
    for_values<T>(row, lo, hi, [&](const float4& x, int at) {
        f(x.x, at);
        f(x.y, at + 1);
        f(x.z, at + 2);
        f(x.w, at + 3);
    }, f);
}

// Exact selection of the k best of [lo, hi), k <= hi - lo, whatever the values: the k-th largest key digit by digit, then
// what is above it and, in order of index, as many of its equals as are missing.
template <int T>
__device__ void select_exact(Shared<T>& s, const float* row, int lo, int hi, int k) {
    const int tid = threadIdx.x;
    int turn = 0;
    uint32_t prefix = 0;
    int need = k;                              // still to come from values that share the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        clear_bins(s);
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        uint32_t last = 0;                     // a thread adds a run of one digit at once: rows of equal values meet in one bin
        int run = 0;
        for_values<T>(row, lo, hi, [&](float v, int) {
            const uint32_t key = key_of(v), digit = (key >> shift) & 255u;
            if ((key & mask) != prefix) return;
            if (digit != last && run > 0) {
                atomicAdd(&s.hist[last], run);
                run = 0;
            }
            last = digit;
            ++run;
        });
        if (run > 0) atomicAdd(&s.hist[last], run);
        __syncthreads();
        if (tid < 32) find_bin(s, need);
        __syncthreads();
        prefix |= (uint32_t)s.bin << shift;
        need -= s.above;
        __syncthreads();
    }
    if (tid == 0) s.found = 0;
    __syncthreads();
    for_values<T>(row, lo, hi, [&](float v, int at) {
        const uint32_t key = key_of(v);
        if (key > prefix) {
            const int j = atomicAdd(&s.found, 1);
            s.best_key[j] = key;
            s.best_idx[j] = (uint32_t)at;
        }
    });
    __syncthreads();
    int done = 0;
    const int above = k - need;
    for (int base = lo; base < hi && done < need; base += T) {
        const int at = base + tid;
        const bool eq = at < hi && key_of(row[at]) == prefix;
        const unsigned mask = __ballot_sync(0xffffffffu, eq);
        const int warp = tid >> 5, lane = tid & 31;
        if (lane == 0) s.part[turn][warp] = __popc(mask);
        __syncthreads();
        int before = done, all = 0;
        for (int i = 0; i < (T / 32); ++i) {
            const int n = s.part[turn][i];
            if (i < warp) before += n;
            all += n;
        }
        before += __popc(mask & ((1u << lane) - 1u));
        if (eq && before < need) {
            s.best_key[above + before] = prefix;
            s.best_idx[above + before] = (uint32_t)at;
        }
        done += all;
        turn ^= 1;
    }
    __syncthreads();
}

template <int T, int BLOCKS>
__global__ void __launch_bounds__(T, BLOCKS) top_logits_kernel(int V, const float* logits, int K, int cluster, int32_t* ids, float* values) {
    extern __shared__ __align__(16) unsigned char raw[];
    constexpr int FAN = T / MAX_TOP;
    Shared<T>& s = *reinterpret_cast<Shared<T>*>(raw);
    uint32_t* sent_key = reinterpret_cast<uint32_t*>(&s + 1);
    uint32_t* sent_idx = sent_key + LIST<T>;
    const int tid = threadIdx.x, rank = (int)blockIdx.x % cluster;
    const size_t r = blockIdx.x / cluster;
    const float* row = logits + r * V;
    const int lo = (int)((long)rank * V / cluster), hi = (int)((long)(rank + 1) * V / cluster), n_slice = hi - lo;
    const int k = min(K, n_slice);
    if (tid == 0) {
        s.count = 0;
        s.low = ~0u;
        s.high = 0;
    }
    pdl_trigger();
    if (cluster > 1) sm100::cluster_arrive();                  // met before the first store to another block
    __syncthreads();
    pdl_wait();
    float cut = -INFINITY;
    bool exact = false;
    if (n_slice > LIST<T>) {
        // runs of 32 values, eight lanes (16 bytes each) to a run, a third of the slice at most: apart by more than a run,
        // whatever their starts' rounding, so that no value is counted twice
        const int runs = min((n_slice - RUN) / (3 * RUN), SAMPLE_RUNS);
        const bool vec = (reinterpret_cast<uintptr_t>(row) & 15) == 0;
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < SAMPLE_RUNS / (T / 8); ++i) {
            const int run = i * (T / 8) + (tid >> 3);
            if (run < runs) {
                const int at = (lo + (int)((long)run * (n_slice - RUN) / runs)) / 4 * 4 + 4 * (tid & 7);
                const int from = max(at, lo);
                if (vec && from == at) {
                    const float4 x = *reinterpret_cast<const float4*>(row + at);
                    m = fmaxf(fmaxf(m, fmaxf(x.x, x.y)), fmaxf(x.z, x.w));
                } else {
                    for (int j = from; j < at + 4; ++j) m = fmaxf(m, row[j]);
                }
            }
        }
        // the cut: the start of the maxima's bin that holds the k-th largest
        const uint32_t top = key_of(m);
        const uint32_t least = __reduce_min_sync(0xffffffffu, top), most = __reduce_max_sync(0xffffffffu, top);
        if ((tid & 31) == 0) {
            atomicMin(&s.low, least);
            atomicMax(&s.high, most);
        }
        __syncthreads();
        const uint32_t c = narrow(s, T, [&](int, uint32_t& v) { v = top; return true; }, s.low, s.high, k, 14).low;
        if (c <= key_of(-INFINITY)) exact = true;              // fewer than k finite maxima
        else cut = value_of(c);
        if (tid == 0) s.high = 0;
        __syncthreads();
    }
    if (!exact) {
        auto keep = [&](float v, int at) {
            const int j = atomicAdd(&s.count, 1);
            if (j < LIST<T>) {
                s.key[j] = key_of(v);
                s.idx[j] = (uint32_t)at;
            }
        };
        if (n_slice <= LIST<T>) {
            for_values<T>(row, lo, hi, keep);
        } else {
            for_values<T>(row, lo, hi, [&](const float4& x, int at) {
                if (fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)) >= cut) {
                    if (x.x >= cut) keep(x.x, at);
                    if (x.y >= cut) keep(x.y, at + 1);
                    if (x.z >= cut) keep(x.z, at + 2);
                    if (x.w >= cut) keep(x.w, at + 3);
                }
            }, [&](float v, int at) {
                if (v >= cut) keep(v, at);
            });
        }
        __syncthreads();
        if (s.count > LIST<T> || s.count < k) exact = true;
    }
    const uint32_t floor_key = n_slice > LIST<T> && !exact ? key_of(cut) : 0u;
    const bool sends = cluster > 1;
    int have = k;
    const uint32_t *from_key = s.key, *from_idx = s.idx;       // what the blocks of a cluster send, what one block selects among
    int n = s.count;
    if (exact) {
        select_exact(s, row, lo, hi, k);
        from_key = s.best_key;
        from_idx = s.best_idx;
        n = k;
    } else if (!sends || n > SENT<T>) {
        uint32_t high = 0;
        for (int j = tid; j < n; j += T) high = max(high, s.key[j]);
        high = __reduce_max_sync(0xffffffffu, high);
        if ((tid & 31) == 0) atomicMax(&s.high, high);
        __syncthreads();
        n = select(s, s.key, s.idx, n, k, floor_key, s.high);
        from_key = s.best_key;
        from_idx = s.best_idx;
    }
    if (sends) {
        sm100::cluster_wait();
        const uint32_t to_key = sm100::map_to_cta(smem_u32(sent_key), 0), to_idx = sm100::map_to_cta(smem_u32(sent_idx), 0);
        for (int i = tid; i < n; i += T) {
            sm100::st_cluster_u32(to_key + (uint32_t)(rank * SENT<T> + i) * 4u, from_key[i]);
            sm100::st_cluster_u32(to_idx + (uint32_t)(rank * SENT<T> + i) * 4u, from_idx[i]);
        }
        if (tid == 0) sm100::st_cluster_u32(sm100::map_to_cta(smem_u32(&s.sent[rank]), 0), (uint32_t)n);
        sm100::cluster_sync();
        if (rank > 0) return;
        if (tid == 0) {
            s.low = ~0u;
            s.high = 0;
        }
        __syncthreads();
        uint32_t low = ~0u, high = 0;
        int at = 0;
        for (int c = 0; c < cluster; ++c) {
            const int m = s.sent[c];
            for (int i = tid; i < m; i += T) {
                const uint32_t key = sent_key[c * SENT<T> + i];
                s.key[at + i] = key;
                s.idx[at + i] = sent_idx[c * SENT<T> + i];
                low = min(low, key);
                high = max(high, key);
            }
            at += m;
        }
        low = __reduce_min_sync(0xffffffffu, low);
        high = __reduce_max_sync(0xffffffffu, high);
        if ((tid & 31) == 0) {
            atomicMin(&s.low, low);
            atomicMax(&s.high, high);
        }
        __syncthreads();
        have = select(s, s.key, s.idx, at, K, s.low, s.high);
    }
    // in order: an entry's place is the number of better ones; FAN threads count for an entry
    const int e = tid / FAN;
    int place = 0;
    uint32_t key = 0, idx = 0;
    if (e < have) {
        key = s.best_key[e];
        idx = s.best_idx[e];
        for (int o = tid % FAN; o < have; o += FAN) place += s.best_key[o] > key || (s.best_key[o] == key && s.best_idx[o] < idx);
    }
#pragma unroll
    for (int o = 1; o < FAN; o <<= 1) place += __shfl_xor_sync(0xffffffffu, place, o);
    if (tid % FAN == 0 && e < K) {
        const size_t to = r * K + (e < have ? place : e);
        ids[to] = e < have ? (int32_t)idx : -1;
        // (a key does not tell -0 from 0, nor one NaN from another)
        values[to] = e >= have ? -INFINITY : key == 0 || key == 0x80000000u ? row[idx] : value_of(key);
    }
}

// BLOCKS of T threads to an SM.
template <int T, int BLOCKS>
static int launch(int M, int V, const float* logits, int K, int cluster, int32_t* ids, float* values, cudaStream_t st) {
    constexpr size_t SENT_BYTES = 2 * LIST<T> * sizeof(uint32_t);
    DEER_CUDA(cudaFuncSetAttribute(top_logits_kernel<T, BLOCKS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Shared<T>) + SENT_BYTES)));
    DEER_CUDA(launch_pdl_cluster(cluster, top_logits_kernel<T, BLOCKS>, dim3((unsigned)(M * cluster)), dim3(T), sizeof(Shared<T>) + (cluster > 1 ? SENT_BYTES : 0), st,
                                 V, logits, K, cluster, ids, values));
    return DEER_OK;
}

}  // namespace toplogits

extern "C" int deer_top_logits(int M, int V, const float* logits, int K, int32_t* ids, float* values, void* stream) {
    using namespace toplogits;
    DEER_CHECK_ARG(M >= 0 && V >= 1, DEER_ERR_INVALID_ARG, "deer_top_logits: M must not be negative, V at least 1");
    DEER_CHECK_ARG(M <= (1 << 24) && V <= (1 << 30), DEER_ERR_UNSUPPORTED, "deer_top_logits: more than 2^24 rows or 2^30 tokens");
    DEER_CHECK_ARG(K >= 1 && K <= MAX_TOP, DEER_ERR_UNSUPPORTED, "deer_top_logits: K must be 1 to %d", MAX_TOP);
    if (M == 0) return DEER_OK;
    DEER_CHECK_ARG(logits && ids && values, DEER_ERR_INVALID_ARG, "deer_top_logits: null pointer");
    DEER_CHECK_ARG(deer_aligned16(logits) && deer_aligned4(ids) && deer_aligned4(values), DEER_ERR_INVALID_ARG,
                   "deer_top_logits: logits must be 16-byte aligned, ids and values 4-byte");
    // Eight or four blocks to a row where there is room for all of them at once (three to an SM), on slices of LIST values at
    // least.  Rows of 151936, the 64 best: 32 rows 17 us by eight blocks, 19 by two, 25 by one; 100 rows 25 by four, 33 by one;
    // 200 rows 36 by one, 39 by two, and in several rounds clusters lose (512 rows: 59 by one, 103 by two).  Where clusters fill
    // the room to the last place not all of them fit side by side, and the rule loses: 55 rows 27.5 by eight, 23 by two; 110 rows
    // 37.5 by four, 28 by two, 33 by one.
    const long slots = 3L * deer_sm_count();
    int cluster = MAX_CLUSTER;
    while (cluster > 1 && ((long)M * cluster > slots || V / cluster < LIST<512>)) cluster /= 2;
    if (cluster == 2) cluster = 1;
    // Many shorter rows by half the threads: what a row costs beside its reading is a chain of steps, and more rows go side by
    // side (2048 rows of 5000: 35 us by 512 threads, 24 by 256; 1492 of 14725: 41 and 33; 2048 of 32768: 75 and 69).  Longer rows
    // go either way (2048 of 40000: 82 and 78; 1332 of 50257: 94 and 102) until the reading counts (512 of 151936: 60 and 72,
    // 2048: 222 and 228).
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (M <= slots) return launch<512, 3>(M, V, logits, K, cluster, ids, values, st);
    // A third more rows to an SM, at 32 registers a thread, where that saves a round of them (512 rows of 151936: 78 us in two
    // rounds, 59 in one; 1184: 131 and 126; 4096: 420 and 405; 2048 of 32768 by 256 threads: 79 and 69); where it saves none, a
    // round only takes longer (700 rows: 85 and 98; 1332: 140 and 157; 1492 of 14725: 33 and 36).
    const bool short_rows = V <= 32768;
    const long wave = short_rows ? 2 * slots : slots, wider = wave / 3 * 4;
    if ((M + wider - 1) / wider < (M + wave - 1) / wave)
        return short_rows ? launch<256, 8>(M, V, logits, K, 1, ids, values, st) : launch<512, 4>(M, V, logits, K, 1, ids, values, st);
    return short_rows ? launch<256, 6>(M, V, logits, K, 1, ids, values, st) : launch<512, 3>(M, V, logits, K, 1, ids, values, st);
}
