// deer_linear_quant: y = x w^T of e4m3 codes with a scale per 128 columns of a row of x and per 128 x 128 block of w.
//
// y[m][n] = sum over column groups g of  x_scale[m][g] * w_scale[n / 128][g] * (sum_{c in g} x[m][c] w[n][c]).
//
// The inner sums are tcgen05 e4m3 MMAs.  The weight rows sit on the 128 TMEM lanes -- so a tile of 128 output columns
// has ONE weight scale per column group -- and NT rows of x on the accumulator columns, NT chosen by M: few rows cost
// few MMA columns and few shared-memory bytes, and all four lane quarters of the epilogue have work whatever M is.
// Each column group goes into an accumulator of its own (a ring of them in TMEM); the epilogue warps read it, scale it
// by x_scale * w_scale and add it to fp32 sums that stay in registers.  What bounds it: the weight bytes for M up to a
// few hundred, above that the MMAs together with those scaled sums.
//
// Few output columns do not fill the SMs, so a cluster of `split` blocks shares an output tile, each with a range of
// the column groups; the partial sums meet in shared memory (every block of the cluster adds up, in rank order, its
// part of the tile's rows of x), so there is no workspace, no second kernel, and the order of the sums is fixed.
//
// Warp roles: warp 0 = TMA producer, warp 1 = MMA issuer (+ TMEM owner), the others = epilogue.  All waits are bounded;
// a block whose wait runs out leaves its output unwritten (and so does its cluster).

#include "quant.cuh"
#include "sm100.cuh"

namespace linq {

using namespace sm100;
using quant::GROUP;

constexpr int BN = 128;                        // weight rows (output columns) of a tile
constexpr int W_BYTES = BN * GROUP;            // 16 KB per stage

// NT rows of x per tile; stages such that two blocks fit an SM (one for NT = 256).
template <int NT>
struct Cfg {
    static constexpr int STAGE = W_BYTES + NT * GROUP;
    static constexpr int STAGES = NT == 16 ? 6 : NT == 32 ? 5 : NT == 64 ? 4 : NT == 128 ? 3 : 4;
    static constexpr int NBUF = NT <= 64 ? 4 : 2;                 // accumulators in TMEM
    static constexpr int TMEM_COLS = NT * NBUF < 64 ? 64 : NT * NBUF;
    static constexpr int EPI_WARPS = NT == 256 ? 8 : 4;
    static constexpr int THREADS = 64 + EPI_WARPS * 32;
    static constexpr int COLS = NT == 256 ? 128 : NT;             // accumulator columns of one epilogue thread
    static constexpr int SMEM = STAGES * STAGE + 1024 /*alignment slack*/ + 2 * NT * 4 /*scales*/ + (2 * STAGES + 2 * NBUF) * 8 + 16;
};

struct Args {
    const float* x_scale;
    const float* w_scale;
    const __nv_bfloat16* residual;
    __nv_bfloat16* y;
    int M, K, N, groups, m_tiles, split;
};

__device__ __forceinline__ float ld_cluster_f32(uint32_t cluster_addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t cluster_addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
    return v;
}

template <int NT>
__global__ void __launch_bounds__(Cfg<NT>::THREADS, NT == 256 ? 1 : 2)
linear_quant_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Args a) {
    using C = Cfg<NT>;
    constexpr int EPI_THREADS = C::EPI_WARPS * 32;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* sc = reinterpret_cast<float*>(ring + C::STAGES * C::STAGE);           // [2][NT] x_scale * w_scale of a column group
    uint64_t* bars = reinterpret_cast<uint64_t*>(sc + 2 * NT);                   // full, empty [STAGES]; tfull, tempty [NBUF]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::STAGES + 2 * C::NBUF);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)blockIdx.x % a.split;
    const int tile = (int)blockIdx.x / a.split;
    const int m0 = (tile % a.m_tiles) * NT, n0 = (tile / a.m_tiles) * BN;
    const int g0 = (int)((long)rank * a.groups / a.split), ng = (int)((long)(rank + 1) * a.groups / a.split) - g0;

    const uint32_t ring_addr = smem_u32(ring), bar_base = smem_u32(bars);
    auto full = [&](int s) { return bar_base + 8u * s; };
    auto empty = [&](int s) { return bar_base + 8u * (C::STAGES + s); };
    auto tfull = [&](int b) { return bar_base + 8u * (2 * C::STAGES + b); };
    auto tempty = [&](int b) { return bar_base + 8u * (2 * C::STAGES + C::NBUF + b); };
    if (tid == 0) {
        for (int s = 0; s < C::STAGES; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
        }
        for (int b = 0; b < C::NBUF; ++b) {
            mbar_init(tfull(b), 1);
            mbar_init(tempty(b), C::EPI_WARPS);
        }
        *abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tensormap(&tm_w);
        prefetch_tensormap(&tm_x);
        // the first weight tiles travel to L2 while the kernel before is still running
        for (int i = 0; i < ng && i < C::STAGES; ++i) tma_prefetch_2d(&tm_w, (g0 + i) * GROUP, n0);
    }
    if (warp == 1) tmem_alloc(smem_u32(tmem_slot), C::TMEM_COLS);
    pdl_trigger();
    pdl_wait();
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    float acc[C::COLS];
    if (warp == 0) {
        if (lane == 0) {
            for (int i = 0; i < ng; ++i) {
                const int s = i % C::STAGES;
                if (!mbar_wait(empty(s), ((uint32_t)(i / C::STAGES) & 1u) ^ 1u, abort_flag)) break;
                mbar_expect_tx(full(s), C::STAGE);
                tma_load_2d(ring_addr + s * C::STAGE, &tm_w, (g0 + i) * GROUP, n0, full(s));
                tma_load_2d(ring_addr + s * C::STAGE + W_BYTES, &tm_x, (g0 + i) * GROUP, m0, full(s));
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = make_idesc_e4m3(NT);
            for (int i = 0; i < ng; ++i) {
                const int s = i % C::STAGES, b = i % C::NBUF;
                if (!mbar_wait(tempty(b), ((uint32_t)(i / C::NBUF) & 1u) ^ 1u, abort_flag)) break;
                if (!mbar_wait(full(s), (uint32_t)(i / C::STAGES) & 1u, abort_flag)) break;
                tcgen05_fence_after();
                const uint64_t wd = smem_desc_sw128_kmajor(ring_addr + s * C::STAGE);
                const uint64_t xd = smem_desc_sw128_kmajor(ring_addr + s * C::STAGE + W_BYTES);
#pragma unroll
                for (int kk = 0; kk < GROUP / 32; ++kk)
                    umma_f8_ss(tmem_base + (uint32_t)(b * NT), wd + (uint64_t)(kk * 2), xd + (uint64_t)(kk * 2), idesc, kk != 0 ? 1u : 0u);
                umma_commit(empty(s));
                umma_commit(tfull(b));
            }
        }
    } else {
        const int et = tid - 64;                                   // 0 .. EPI_THREADS - 1
        const int half = NT == 256 ? (et >> 7) : 0;                // which 128 accumulator columns
        const uint32_t t_lane = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(half * 128);
#pragma unroll
        for (int j = 0; j < C::COLS; ++j) acc[j] = 0.f;
        // thread et brings the scale of row m0 + et, four column groups ahead
        const bool brings = et < NT;
        const float* xs = (brings && m0 + et < a.M) ? a.x_scale + (size_t)(m0 + et) * a.groups + g0 : nullptr;
        const float* ws = a.w_scale + (size_t)(n0 / GROUP) * a.groups + g0;
        float nx[4], nw[4];
        auto fetch = [&](int i0) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                nx[u] = (xs && i0 + u < ng) ? xs[i0 + u] : 0.f;
                nw[u] = (xs && i0 + u < ng) ? ws[i0 + u] : 0.f;
            }
        };
        fetch(0);
        bool alive = true;
        for (int i0 = 0; i0 < ng; i0 += 4) {
            float s4[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) s4[u] = nx[u] * nw[u];
            fetch(i0 + 4);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u;
                if (i >= ng) break;
                const int b = i % C::NBUF;
                float* slot = sc + (i & 1) * NT;
                if (brings) slot[et] = s4[u];
                asm volatile("bar.sync 1, %0;" ::"n"(EPI_THREADS) : "memory");
                // a warp whose wait ran out keeps meeting the others at the barrier
                const bool got = alive && mbar_wait(tfull(b), (uint32_t)(i / C::NBUF) & 1u, abort_flag);
                if (!__all_sync(0xffffffffu, got)) {
                    alive = false;
                    continue;
                }
                tcgen05_fence_after();
                const float4* s_row = reinterpret_cast<const float4*>(slot + half * 128);
#pragma unroll
                for (int c = 0; c < C::COLS; c += 16) {
                    uint32_t r[16];
                    TMEM_LD_X16(t_lane + (uint32_t)(b * NT + c), r);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const float4 s = s_row[(c + j) / 4];
                        acc[c + j] = fmaf(__uint_as_float(r[j]), s.x, acc[c + j]);
                        acc[c + j + 1] = fmaf(__uint_as_float(r[j + 1]), s.y, acc[c + j + 1]);
                        acc[c + j + 2] = fmaf(__uint_as_float(r[j + 2]), s.z, acc[c + j + 2]);
                        acc[c + j + 3] = fmaf(__uint_as_float(r[j + 3]), s.w, acc[c + j + 3]);
                    }
                }
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(tempty(b));
            }
        }
    }

    // ---- the tile's rows of x: this block writes all of them, or adds up its part of the cluster's partial sums ----
    const int et = tid - 64, half = NT == 256 ? (et >> 7) : 0;
    const int lane_row = (warp & 3) * 32 + lane;                   // TMEM lane = output column within the tile
    const int n = n0 + lane_row;
    auto put = [&](int j, float v) {                               // row m0 + j of the output
        const int m = m0 + j;
        if (m >= a.M || n >= a.N) return;
        const size_t at = (size_t)m * a.N + n;
        if (a.residual) v += __bfloat162float(a.residual[at]);
        a.y[at] = __float2bfloat16(v);
    };
    if (a.split == 1) {
        if (warp >= 2 && !*abort_flag) {
#pragma unroll
            for (int j = 0; j < C::COLS; ++j) put(half * 128 + j, acc[j]);
        }
    } else {
        // every operand that was requested has been consumed (or the block is aborting and writes nothing): the ring is free
        float* buf = reinterpret_cast<float*>(ring);               // [NT][128]
        if (warp >= 2 && !*abort_flag) {
#pragma unroll
            for (int j = 0; j < C::COLS; ++j) buf[(half * 128 + j) * BN + lane_row] = acc[j];
        }
        __syncwarp();
        cluster_sync();
        bool good = true;
        const uint32_t flag_addr = smem_u32(const_cast<int*>(abort_flag));
        for (int r = 0; r < a.split; ++r) good = good && ld_cluster_u32(map_to_cta(flag_addr, (uint32_t)r)) == 0;
        if (warp >= 2 && good) {
            const int lo = NT * rank / a.split, hi = NT * (rank + 1) / a.split;
            for (int j = lo + half; j < hi; j += C::EPI_WARPS / 4) {
                if (m0 + j >= a.M) break;
                float v = 0.f;
                for (int r = 0; r < a.split; ++r) v += ld_cluster_f32(map_to_cta(ring_addr + (uint32_t)((j * BN + lane_row) * 4), (uint32_t)r));
                put(j, v);
            }
        }
        __syncwarp();
        cluster_sync();                                            // nobody's shared memory goes away while it is being read
    }

    tcgen05_fence_before();
    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(10000);           // copies still in flight land before the memory goes away
        __syncthreads();
    }
    if (warp == 1) {
        __syncwarp();
        tcgen05_fence_after();
        tmem_dealloc(tmem_base, C::TMEM_COLS);
    }
}

template <int NT>
int launch(Args a, const void* x, const void* w, cudaStream_t st) {
    using C = Cfg<NT>;
    CUtensorMap tm_w, tm_x;
    const uint64_t str[1] = {(uint64_t)a.K};
    {
        const uint64_t dims[2] = {(uint64_t)a.K, (uint64_t)a.N};
        const uint32_t box[2] = {GROUP, BN};
        const int rc = make_map_u8(&tm_w, w, 2, dims, str, box);
        if (rc != DEER_OK) return rc;
    }
    {
        const uint64_t dims[2] = {(uint64_t)a.K, (uint64_t)a.M};
        const uint32_t box[2] = {GROUP, NT};
        const int rc = make_map_u8(&tm_x, x, 2, dims, str, box);
        if (rc != DEER_OK) return rc;
    }
    a.m_tiles = (a.M + NT - 1) / NT;
    const long long tiles = (long long)((a.N + BN - 1) / BN) * a.m_tiles;
    // As many blocks of a cluster as still fit beside each other (two per SM, one for NT = 256) with at least four
    // column groups each.
    const long long room = (long long)deer_sm_count() * (NT == 256 ? 1 : 2);
    a.split = 1;
    while (a.split < 8 && tiles * a.split * 2 <= room && a.groups >= a.split * 2 * 4) a.split *= 2;
    DEER_CHECK_ARG(tiles * a.split <= 0x7fffffffLL, DEER_ERR_UNSUPPORTED, "deer_linear_quant: too many tiles");
    DEER_CUDA(cudaFuncSetAttribute(linear_quant_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * a.split));
    cfg.blockDim = dim3(C::THREADS);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    DEER_CUDA(cudaLaunchKernelEx(&cfg, linear_quant_kernel<NT>, tm_w, tm_x, a));
    return DEER_OK;
}

}  // namespace linq

using namespace linq;

extern "C" int deer_linear_quant(const void* x, const float* x_scale, const void* w, const float* w_scale, const void* residual, void* y,
                                 int M, int K, int N, void* stream) {
    DEER_CHECK_ARG(x && x_scale && w && w_scale && y, DEER_ERR_INVALID_ARG, "deer_linear_quant: null argument");
    DEER_CHECK_ARG(deer_aligned16(x) && deer_aligned16(w) && deer_aligned16(residual) && deer_aligned16(y) && deer_aligned4(x_scale) &&
                       deer_aligned4(w_scale),
                   DEER_ERR_INVALID_ARG, "deer_linear_quant: pointers must be 16-byte aligned (scales: 4)");
    DEER_CHECK_ARG(M >= 0, DEER_ERR_INVALID_ARG, "deer_linear_quant: M must be >= 0");
    DEER_CHECK_ARG(K >= 16 && K % 16 == 0 && N >= 16 && N % 16 == 0, DEER_ERR_UNSUPPORTED,
                   "deer_linear_quant: K and N must be multiples of 16, at least 16");
    if (M == 0) return DEER_OK;
    Args a = {};
    a.x_scale = x_scale;
    a.w_scale = w_scale;
    a.residual = static_cast<const __nv_bfloat16*>(residual);
    a.y = static_cast<__nv_bfloat16*>(y);
    a.M = M;
    a.K = K;
    a.N = N;
    a.groups = (K + GROUP - 1) / GROUP;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (M <= 16) return launch<16>(a, x, w, st);
    if (M <= 32) return launch<32>(a, x, w, st);
    if (M <= 64) return launch<64>(a, x, w, st);
    if (M <= 128) return launch<128>(a, x, w, st);
    return launch<256>(a, x, w, st);
}
