// The K largest logits of each row, ids and values, falling, the lowest index first among equals.
//
// A row is read once.  A sample of it (16384 values in 128-byte runs spread over the row, which L2 gives again to the pass
// behind) yields a cut: each of the 512 threads keeps its share's maximum, and the K-th largest of those maxima has K values
// of the row at or above it, whatever the row looks like.  The pass keeps what is not below the cut -- some 10 K of 151936
// values -- in shared memory, one compare per value; the K best of those are found by a search over the bits of their keys
// and put in order by counting.  A row that overfills the list (long ties, a sample that says nothing about the row) is
// selected exactly instead, by four histogram passes over the digits of the key and one that collects in order of index.
// The key is the value's bits in an order of whole numbers: NaN below everything, -0 equal to 0.
//
// With few rows a cluster of up to eight blocks shares one, each a slice, and the first block selects among their best.
#include <math.h>

#include "sm100.cuh"

namespace toplogits {

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int LIST = 4096;                 // candidates a block holds; PER of them a thread
constexpr int PER = LIST / THREADS;
constexpr int MAX_TOP = 128;
constexpr int MAX_CLUSTER = 8;
constexpr int RUN = 32, SAMPLE_RUNS = 512; // values of a sampled run, runs of a sample

__device__ __forceinline__ uint32_t key_of(float v) {
    uint32_t b = __float_as_uint(v);
    if (b == 0x80000000u) b = 0;
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

struct Shared {
    uint32_t key[LIST], idx[LIST];
    uint32_t best_key[MAX_CLUSTER * MAX_TOP], best_idx[MAX_CLUSTER * MAX_TOP];   // a block's best; the first block's: all blocks'
    int hist[256];
    int part[2][WARPS];
    int count, found, flip;
};

// Sum over the block, for every thread.  One barrier: consecutive sums use the two rows of `part` in turn.
__device__ __forceinline__ int block_sum(Shared& s, int v, int& turn) {
    v = __reduce_add_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) s.part[turn][threadIdx.x >> 5] = v;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) t += s.part[turn][i];
    turn ^= 1;
    return t;
}

// The largest c such that at least k of the block's values are >= c (k of them at most n).  `exact`: exactly k are.
__device__ __forceinline__ uint32_t kth_largest(Shared& s, const uint32_t (&v)[PER], int have, int k, bool& exact, int& turn) {
    uint32_t c = 0;
    exact = false;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t cand = c | (1u << bit);
        int n = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) n += i < have && v[i] >= cand;
        n = block_sum(s, n, turn);
        if (n >= k) c = cand;
        if (n == k) {
            exact = true;
            break;
        }
    }
    return c;
}

// The k best of the n <= LIST entries (key, idx): to best_key / best_idx in any order.  Returns how many (min(n, k)).
__device__ int select(Shared& s, const uint32_t* keys, const uint32_t* idxs, int n, int k, uint32_t* out_key, uint32_t* out_idx, int& turn) {
    const int tid = threadIdx.x;
    uint32_t key[PER], inv[PER];               // inv: falling in the index, so that the lowest index is the largest
    int have = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int j = tid + i * THREADS;
        key[i] = inv[i] = 0;
        if (j < n) {
            key[i] = keys[j];
            inv[i] = ~idxs[j];
            have = i + 1;
        }
    }
    if (tid == 0) s.found = 0;
    __syncthreads();                           // (and every entry is in registers: out_key may be keys)
    uint32_t cut = 0, cut_inv = 0;             // taken: key > cut, or key == cut and inv >= cut_inv
    if (n > k) {
        bool exact;
        cut = kth_largest(s, key, have, k, exact, turn);
        if (!exact) {                          // more than k values >= cut: the ones equal to it by index
            int above = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) above += i < have && key[i] > cut;
            above = block_sum(s, above, turn);
            uint32_t tie[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) tie[i] = i < have && key[i] == cut ? inv[i] : 0;      // (inv is never 0)
            cut_inv = kth_largest(s, tie, have, k - above, exact, turn);
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (i < have && (key[i] > cut || (key[i] == cut && inv[i] >= cut_inv))) {
            const int at = atomicAdd(&s.found, 1);
            out_key[at] = key[i];
            out_idx[at] = ~inv[i];
        }
    __syncthreads();
    return min(n, k);
}

// Calls f(value, index) for the values [lo, hi) of the row, 16 bytes at a time where the alignment allows it.
template <typename F>
__device__ __forceinline__ void for_values(const float* row, int lo, int hi, F f) {
    const int tid = threadIdx.x;
    const int skew = (int)((4 - ((reinterpret_cast<uintptr_t>(row + lo) >> 2) & 3)) & 3);
    const int v0 = min(lo + skew, hi), nv = (hi - v0) / 4;
    if (tid < v0 - lo) f(row[lo + tid], lo + tid);
    const float4* vec = reinterpret_cast<const float4*>(row + v0);
    int i = tid;
    for (; i + 3 * THREADS < nv; i += 4 * THREADS) {
        float4 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __ldg(vec + i + j * THREADS);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int at = v0 + 4 * (i + j * THREADS);
            f(x[j].x, at);
            f(x[j].y, at + 1);
            f(x[j].z, at + 2);
            f(x[j].w, at + 3);
        }
    }
    for (; i < nv; i += THREADS) {
        const float4 x = __ldg(vec + i);
        const int at = v0 + 4 * i;
        f(x.x, at);
        f(x.y, at + 1);
        f(x.z, at + 2);
        f(x.w, at + 3);
    }
    const int rest = v0 + 4 * nv + tid;
    if (rest < hi) f(row[rest], rest);
}

// Exact selection of the k best of [lo, hi), k <= hi - lo, whatever the values: the k-th largest key digit by digit, then
// what is above it and, in order of index, as many of its equals as are missing.
__device__ void select_exact(Shared& s, const float* row, int lo, int hi, int k, int& turn) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    int need = k;                              // still to come from values that share the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += THREADS) s.hist[i] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        uint32_t last = 0;                     // a thread adds a run of one digit at once: rows of equal values meet in one bin
        int run = 0;
        for_values(row, lo, hi, [&](float v, int) {
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
        if (tid == 0) {
            int d = 255, sum = 0;
            while (d > 0 && sum + s.hist[d] < need) sum += s.hist[d--];
            s.flip = d;
            s.count = need - sum;
        }
        __syncthreads();
        prefix |= (uint32_t)s.flip << shift;
        need = s.count;
        __syncthreads();
    }
    if (tid == 0) s.found = 0;
    __syncthreads();
    for_values(row, lo, hi, [&](float v, int at) {
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
    for (int base = lo; base < hi && done < need; base += THREADS) {
        const int at = base + tid;
        const bool eq = at < hi && key_of(row[at]) == prefix;
        const unsigned mask = __ballot_sync(0xffffffffu, eq);
        const int warp = tid >> 5, lane = tid & 31;
        if (lane == 0) s.part[turn][warp] = __popc(mask);
        __syncthreads();
        int before = done, all = 0;
        for (int i = 0; i < WARPS; ++i) {
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

__global__ void __launch_bounds__(THREADS) top_logits_kernel(int V, const float* logits, int K, int cluster, int32_t* ids, float* values) {
    extern __shared__ __align__(16) unsigned char raw[];
    Shared& s = *reinterpret_cast<Shared*>(raw);
    const int tid = threadIdx.x, rank = (int)blockIdx.x % cluster;
    const size_t r = blockIdx.x / cluster;
    const float* row = logits + r * V;
    const int lo = (int)((long)rank * V / cluster), hi = (int)((long)(rank + 1) * V / cluster), n_slice = hi - lo;
    const int k = min(K, n_slice);
    int turn = 0;
    pdl_trigger();
    if (cluster > 1) sm100::cluster_arrive();                  // met before the first store to another block
    pdl_wait();
    if (tid == 0) s.count = 0;
    float cut = -INFINITY;
    bool exact = false;
    if (n_slice > LIST) {
        // runs of 32 values, eight lanes (16 bytes each) to a run; apart by more than a run, whatever their starts' rounding:
        // no value may be counted twice
        const int runs = min((n_slice - RUN) / (RUN + 4), SAMPLE_RUNS);
        const bool vec = (reinterpret_cast<uintptr_t>(row) & 15) == 0;
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < SAMPLE_RUNS / (THREADS / 8); ++i) {
            const int run = i * (THREADS / 8) + (tid >> 3);
            if (run < runs) {
                const int at = (lo + (int)((long)run * (n_slice - RUN) / runs)) / 4 * 4 + 4 * (tid & 7);
                const int from = max(at, lo);
                if (vec && from == at) {
                    const float4 x = __ldg(reinterpret_cast<const float4*>(row + at));
                    m = fmaxf(fmaxf(m, fmaxf(x.x, x.y)), fmaxf(x.z, x.w));
                } else {
                    for (int j = from; j < at + 4; ++j) m = fmaxf(m, row[j]);
                }
            }
        }
        const uint32_t top = key_of(m);
        // its upper half is enough: a cut that is a little lower keeps a few values more
        uint32_t c = 0;
        for (int bit = 31; bit >= 16; --bit)
            if (__syncthreads_count(top >= (c | (1u << bit))) >= k) c |= 1u << bit;
        if (c <= key_of(-INFINITY)) exact = true;             // fewer than k finite maxima
        else cut = value_of(c);
    } else {
        __syncthreads();
    }
    if (!exact) {
        const bool all = n_slice <= LIST;
        for_values(row, lo, hi, [&](float v, int at) {
            if (all || v >= cut) {
                const int j = atomicAdd(&s.count, 1);
                if (j < LIST) {
                    s.key[j] = key_of(v);
                    s.idx[j] = (uint32_t)at;
                }
            }
        });
        __syncthreads();
        if (s.count > LIST || s.count < k) exact = true;
        else select(s, s.key, s.idx, s.count, k, s.best_key, s.best_idx, turn);
    }
    if (exact) select_exact(s, row, lo, hi, k, turn);

    int have = k;
    if (cluster > 1) {
        // the blocks' best to the first block
        sm100::cluster_wait();
        if (rank > 0 && tid < k) {
            const uint32_t at = (uint32_t)(rank * MAX_TOP + tid) * 4u;
            sm100::st_cluster_u32(sm100::map_to_cta(smem_u32(s.best_key), 0) + at, s.best_key[tid]);
            sm100::st_cluster_u32(sm100::map_to_cta(smem_u32(s.best_idx), 0) + at, s.best_idx[tid]);
        }
        sm100::cluster_sync();
        if (rank > 0) return;
        // (every slice is longer than K: each has sent K)
        for (int i = tid; i < cluster * K; i += THREADS) {
            s.key[i] = s.best_key[i / K * MAX_TOP + i % K];
            s.idx[i] = s.best_idx[i / K * MAX_TOP + i % K];
        }
        __syncthreads();
        have = select(s, s.key, s.idx, cluster * K, K, s.best_key, s.best_idx, turn);
    }
    // in order: an entry's place is the number of better ones; four threads count for an entry
    const int e = tid >> 2;
    int place = 0;
    uint32_t key = 0, idx = 0;
    if (e < have) {
        key = s.best_key[e];
        idx = s.best_idx[e];
        for (int o = tid & 3; o < have; o += 4) place += s.best_key[o] > key || (s.best_key[o] == key && s.best_idx[o] < idx);
    }
    place += __shfl_xor_sync(0xffffffffu, place, 1);
    place += __shfl_xor_sync(0xffffffffu, place, 2);
    if ((tid & 3) == 0 && e < K) {
        const size_t at = r * K + (e < have ? place : e);
        ids[at] = e < have ? (int32_t)idx : -1;
        values[at] = e < have ? row[idx] : -INFINITY;
    }
}

}  // namespace toplogits

extern "C" int deer_top_logits(int M, int V, const float* logits, int K, int32_t* ids, float* values, void* stream) {
    using namespace toplogits;
    DEER_CHECK_ARG(M >= 0 && V >= 1, DEER_ERR_INVALID_ARG, "deer_top_logits: M must not be negative, V at least 1");
    DEER_CHECK_ARG(M <= (1 << 24) && V <= (1 << 30), DEER_ERR_UNSUPPORTED, "deer_top_logits: more than 2^24 rows or 2^30 tokens");
    DEER_CHECK_ARG(K >= 1 && K <= MAX_TOP, DEER_ERR_UNSUPPORTED, "deer_top_logits: K must be 1 to %d", MAX_TOP);
    DEER_CHECK_ARG(logits && ids && values, DEER_ERR_INVALID_ARG, "deer_top_logits: null pointer");
    DEER_CHECK_ARG(deer_aligned16(logits) && deer_aligned4(ids) && deer_aligned4(values), DEER_ERR_INVALID_ARG,
                   "deer_top_logits: logits must be 16-byte aligned, ids and values 4-byte");
    if (M == 0) return DEER_OK;
    // as many blocks to a row as fill two blocks an SM, each with a slice worth a pass of its own
    int cluster = 1;
    while (cluster < MAX_CLUSTER && (long)M * cluster * 2 <= 2L * deer_sm_count() && V / (cluster * 2) >= LIST) cluster *= 2;
    DEER_CUDA(cudaFuncSetAttribute(top_logits_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)));
    DEER_CUDA(launch_pdl_cluster(cluster, top_logits_kernel, dim3((unsigned)(M * cluster)), dim3(THREADS), sizeof(Shared),
                                 static_cast<cudaStream_t>(stream), V, logits, K, cluster, ids, values));
    return DEER_OK;
}
