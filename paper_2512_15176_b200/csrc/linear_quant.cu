// deer_linear_quant: y = x w^T of e4m3 codes with a scale per 128 columns of a row of x and per 128 x 128 block of w.
//
// y[m][n] = sum over column groups g of  x_scale[m][g] * w_scale[n / 128][g] * (sum_{c in g} x[m][c] w[n][c]).
//
// The inner sums are tcgen05 e4m3 MMAs.  The weight rows sit on the 128 TMEM lanes -- so a tile of 128 output columns
// has ONE weight scale per column group -- and NT rows of x on the accumulator columns, NT chosen by M: few rows cost
// few MMA columns and few shared-memory bytes, and all four lane quarters of the epilogue have work whatever M is.
// Each column group goes into an accumulator of its own (a ring of them in TMEM); the epilogue warps read it, scale it
// by x_scale * w_scale and add it to fp32 sums that stay in registers.
//
// What bounds it.  Few rows: the weight bytes (one row, 4096 x 4096, 6.8 us, 2.6 of them HBM's; 32 rows, 12288 x 4096,
// 13.3 us = 3.9 TB/s, 7.8 HBM's): the loads run at HBM's rate, the rest is the first tile's latency (1.5 us), the cluster's
// meeting (2 us) and a launch.  Many rows (512 x 4096 x 24576, 56 us = 1.85 PFLOP/s in a graph of twenty calls, 64 to 66 us
// in a long row of calls, where power caps the clock; twice the bf16 rate would take 31): the epilogue.  A column group takes
// it about 1100 cycles with 256 weight rows and 0.57 of that with 128, so about 120 for 16 columns and 150 for a hand-over: the
// tensor-memory load of the next 16 columns is under way while eight multiply-adds scale the present ones, which does not cover
// its latency, and the registers (168, of which 128 are sums; the form for 256 weight rows spills two) hold no more loads.
//
// Few output columns do not fill the SMs, so a cluster of `split` blocks shares an output tile, each with a range of
// the column groups.  Every block of the cluster owns a part of the tile's rows of x: the others send it their partial sums
// for those, into its shared memory, and it adds them up in rank order, so there is no workspace, no second kernel, and the
// order of the sums is fixed.  (Sent, not fetched: a remote load takes about 700 cycles, and a block whose memory nobody
// reads needs no barrier at its end.  32 rows, 12288 x 4096: fetched 15.4, sent 13.9 us.)
//
// Many rows: the second kernel, pairs of blocks, the rows of x on the lanes (see there).
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
constexpr int MAX_SPLIT = 8;                   // blocks of a cluster: the portable limit

// NT rows of x per tile; stages such that two blocks fit an SM, whose tensor memory then suffices for both (a block
// allocates it before it lets the next kernel in, so blocks that share an SM never wait for one another's columns).
template <int NT>
struct Cfg {
    static constexpr int STAGE = W_BYTES + NT * GROUP;
    static constexpr int STAGES = NT == 16 ? 5 : 4;
    // Column groups that change hands together (each with NT accumulator columns of its own): a hand-over costs the issuer and
    // the epilogue several hundred cycles of waits and arrivals, as much as four MMAs.  Two hand-overs' worth of accumulators.
    static constexpr int H = NT <= 32 ? 4 : 2;
    static constexpr int NBUF = 2;
    static constexpr int TMEM_COLS = NT * H * NBUF;
    static constexpr int CH = NT < 32 ? 16 : 32;                  // columns of one tensor-memory load
    static constexpr int EPI_WARPS = 4;
    static constexpr int THREADS = 64 + EPI_WARPS * 32;
    // The cluster's partial sums have a place of their own where it is small; in the ring they have to wait for the slowest block.
    static constexpr bool OWN_PLACE = NT <= 32;
    static constexpr int PLACE = NT * BN * 4;
    static constexpr int SMEM = (OWN_PLACE ? PLACE : 0) + STAGES * STAGE + 1024 /*alignment slack*/ + 2 * H * NT * 4 /*scales*/ + (2 * STAGES + 2 * NBUF) * 8 + 16 + MAX_SPLIT * EPI_WARPS * 4;
};

struct Args {
    const float* x_scale;
    const float* w_scale;
    const __nv_bfloat16* residual;
    __nv_bfloat16* y;
    int M, K, N, groups, m_tiles, split;
};

template <int NT>
__global__ void __launch_bounds__(Cfg<NT>::THREADS, 2)
linear_quant_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Args a) {
    using C = Cfg<NT>;
    constexpr int EPI_THREADS = C::EPI_WARPS * 32;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char* place = ring + (C::OWN_PLACE ? C::STAGES * C::STAGE : 0);     // [rank][4 rows][128 columns][4] partial sums
    float* sc = reinterpret_cast<float*>(ring + C::STAGES * C::STAGE + (C::OWN_PLACE ? C::PLACE : 0));   // [2][H][NT] x_scale * w_scale of a hand-over's column groups
    uint64_t* bars = reinterpret_cast<uint64_t*>(sc + 2 * C::H * NT);            // full, empty [STAGES]; tfull, tempty [NBUF]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::STAGES + 2 * C::NBUF);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    uint32_t* whole = tmem_slot + 4;                                             // [rank][epilogue warp]: its sums are complete

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;   // (uniform, and known to be)
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
    if (C::OWN_PLACE && a.split > 1) cluster_arrive();             // (waited for before anything is sent)

    uint64_t acc[NT / 2];                          // two rows of x each
    bool alive = true;
    const int lane_row = (warp & 3) * 32 + lane;                   // TMEM lane = output column within the tile
    const int n = n0 + lane_row;
    // the rows that this block writes, and the residual of the first of them, which may have to come from far
    const int own_rows = NT / a.split, own0 = m0 + rank * own_rows;
    float res[4] = {0.f, 0.f, 0.f, 0.f};
    auto fetch_residual = [&](int m) {
#pragma unroll
        for (int q = 0; q < 4; ++q) res[q] = a.residual && q < own_rows && m + q < a.M && n < a.N ? __bfloat162float(a.residual[(size_t)(m + q) * a.N + n]) : 0.f;
    };
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
        const uint32_t idesc = make_idesc_e4m3(NT);
        const bool leader = elect_one();
        bool ok = true;
        for (int i0 = 0, n = 0; i0 < ng && ok; i0 += C::H, ++n) {
            const int b = n % C::NBUF;
            ok = __all_sync(0xffffffffu, mbar_wait(tempty(b), ((uint32_t)(n / C::NBUF) & 1u) ^ 1u, abort_flag));
            for (int u = 0; u < C::H && i0 + u < ng && ok; ++u) {
                const int i = i0 + u, s = i % C::STAGES;
                ok = __all_sync(0xffffffffu, mbar_wait(full(s), (uint32_t)(i / C::STAGES) & 1u, abort_flag));
                if (!ok) break;
                tcgen05_fence_after();
                const uint64_t wd = smem_desc_sw128_kmajor(ring_addr + s * C::STAGE);
                const uint64_t xd = smem_desc_sw128_kmajor(ring_addr + s * C::STAGE + W_BYTES);
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < GROUP / 32; ++kk)
                        umma_f8_ss(tmem_base + (uint32_t)((b * C::H + u) * NT), wd + (uint64_t)(kk * 2), xd + (uint64_t)(kk * 2), idesc, kk != 0 ? 1u : 0u);
                    umma_commit(empty(s));
                }
                __syncwarp();
            }
            if (ok && leader) umma_commit(tfull(b));
            __syncwarp();
        }
    } else {
        const int et = tid - 64;                                   // 0 .. EPI_THREADS - 1
        const uint32_t t_lane = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
#pragma unroll
        for (int j = 0; j < NT / 2; ++j) acc[j] = 0;
        // thread et brings the scale of row et / H and column group et % H of a hand-over, one hand-over ahead
        const int my_row = et / C::H, my_u = et % C::H;
        const bool brings = my_row < NT;
        const float* xs = (brings && m0 + my_row < a.M) ? a.x_scale + (size_t)(m0 + my_row) * a.groups + g0 + my_u : nullptr;
        const float* ws = a.w_scale + (size_t)(n0 / GROUP) * a.groups + g0 + my_u;
        float nx = xs && my_u < ng ? xs[0] : 0.f, nw = xs && my_u < ng ? ws[0] : 0.f;
        fetch_residual(own0);
        for (int i0 = 0, n = 0; i0 < ng; i0 += C::H, ++n) {
            const int b = n % C::NBUF, cnt = min(C::H, ng - i0);
            float* slot = sc + (n & 1) * C::H * NT;
            if (brings) slot[my_u * NT + my_row] = nx * nw;
            if (xs && i0 + C::H + my_u < ng) {
                nx = xs[i0 + C::H];
                nw = ws[i0 + C::H];
            }
            asm volatile("bar.sync 1, %0;" ::"n"(EPI_THREADS) : "memory");
            // a warp whose wait ran out keeps meeting the others at the barrier
            const bool got = alive && mbar_wait(tfull(b), (uint32_t)(n / C::NBUF) & 1u, abort_flag);
            if (!__all_sync(0xffffffffu, got)) {
                alive = false;
                continue;
            }
            tcgen05_fence_after();
            const ulonglong2* s_row = reinterpret_cast<const ulonglong2*>(slot);
            const uint32_t taddr = t_lane + (uint32_t)(b * C::H * NT);
#pragma unroll
            for (int c0 = 0; c0 < C::H * NT; c0 += C::CH) {        // columns c0 .. of column group c0 / NT
                if (c0 / NT >= cnt) break;
                uint32_t v[C::CH];
                if constexpr (C::CH == 16) TMEM_LD_X16(taddr + c0, v);
                else TMEM_LD_X32(taddr + c0, v);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < C::CH; j += 4) {
                    const ulonglong2 s = s_row[(c0 + j) / 4];
                    fma_f32x2(acc[((c0 + j) % NT) / 2], v[j], v[j + 1], s.x);
                    fma_f32x2(acc[((c0 + j) % NT) / 2 + 1], v[j + 2], v[j + 3], s.y);
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(tempty(b));
        }
    }

    // ---- the tile's rows of x: this block writes all of them, or its part of them ----
    auto put = [&](int m, const float (&v)[4], int rows) {         // rows m .. of the output
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < rows && m + q < a.M && n < a.N) a.y[(size_t)(m + q) * a.N + n] = __float2bfloat16(v[q] + res[q]);
    };
    if (a.split == 1) {
        if (warp >= 2 && alive) {
#pragma unroll
            for (int j = 0; j < NT; j += 4) {
                float v[4];
                unpack_f32x2(acc[j / 2], v[0], v[1]);
                unpack_f32x2(acc[j / 2 + 1], v[2], v[3]);
                if (j > 0) fetch_residual(m0 + j);
                put(m0 + j, v, 4);
            }
        }
    } else {
        __syncwarp();
        // every block has begun, or (its ring is the place) every operand that was requested has been consumed
        if (!C::OWN_PLACE) cluster_arrive();
        cluster_wait();
        if (warp >= 2) {
            const uint32_t place_addr = smem_u32(place);
            const int own_log = __ffs(own_rows) - 1;               // (a power of two)
#pragma unroll
            for (int j = 0; j < NT; j += 4) {                      // rows j .. j + 3 belong to one owner, or two each to two
                if (m0 + j >= a.M) break;
                float v[4];
                unpack_f32x2(acc[j / 2], v[0], v[1]);
                unpack_f32x2(acc[j / 2 + 1], v[2], v[3]);
                if (own_rows >= 4) {
                    const uint32_t at = place_addr + (uint32_t)(((rank * own_rows + (j & (own_rows - 1))) * BN + lane_row * 4) * 4);
                    st_cluster_f32x4(map_to_cta(at, (uint32_t)(j >> own_log)), v[0], v[1], v[2], v[3]);
                } else {
                    const uint32_t at = place_addr + (uint32_t)((rank * 2 * BN + lane_row * 2) * 4);
                    st_cluster_f32x2(map_to_cta(at, (uint32_t)(j / 2)), v[0], v[1]);
                    st_cluster_f32x2(map_to_cta(at, (uint32_t)(j / 2 + 1)), v[2], v[3]);
                }
            }
            if (lane < a.split) st_cluster_u32(map_to_cta(smem_u32(whole + rank * C::EPI_WARPS + (warp & 3)), (uint32_t)lane), alive ? 1u : 0u);
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (warp >= 2 && !*abort_flag) {
            bool ok = true;
            for (int r = 0; r < a.split; ++r) ok = ok && whole[r * C::EPI_WARPS + (warp & 3)] != 0u;
#pragma unroll 1                                                   // (code that runs once waits for its fetching: 64 x 2048 x 4096 9.0 us unrolled, 8.8)
            for (int j = 0; j < own_rows && own0 + j < a.M && ok; j += 4) {
                if (j > 0) fetch_residual(own0 + j);
                float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < MAX_SPLIT; ++r) {
                    if (r >= a.split) break;
                    if (own_rows >= 4) {
                        const float4 w = *reinterpret_cast<const float4*>(place + ((r * own_rows + j) * BN + lane_row * 4) * 4);
                        v[0] += w.x; v[1] += w.y; v[2] += w.z; v[3] += w.w;
                    } else {
                        const float2 w = *reinterpret_cast<const float2*>(place + (r * 2 * BN + lane_row * 2) * 4);
                        v[0] += w.x; v[1] += w.y;
                    }
                }
                put(own0 + j, v, own_rows);
            }
        }
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

// ---- many rows of x: pairs of blocks ---------------------------------------------------------------------
// A cluster of two shares tiles of 256 rows of x (128 on each block's TMEM lanes) by BNP rows of w: one cta_group::2 MMA
// reads half of the weight rows from each block's shared memory, so a block stages 128 + BNP / 2 rows per column group
// where a tile of its own would take 128 + BNP.  A row of x per thread makes the scale of a column group ONE number per
// thread and 128 columns -- no shared memory, no barrier between the epilogue's warps -- and eight epilogue warps, half
// of the columns each, keep the sums in registers.  Clusters walk the tiles of the product, the tiles of 256 rows of x
// that share weight rows next to each other in time.  Block 0 of the pair issues the MMAs; its `full` barriers count both
// blocks' bytes, `empty` and `accumulator full` arrive in both blocks, both blocks' epilogue warps free an accumulator.
template <int BNP>
struct PairCfg {
    static constexpr int HALF = BNP / 2;                          // weight rows a block stages; columns of an epilogue warp
    static constexpr int X_BYTES = 128 * GROUP;
    static constexpr int STAGE = X_BYTES + HALF * GROUP;
    static constexpr int STAGES = 192 * 1024 / STAGE;
    static constexpr int OUT_BYTES = 32 * 128;                    // an epilogue warp's 32 rows of 64 output columns
    static constexpr int NBUF = 512 / BNP;                        // accumulators: all of tensor memory
    static constexpr int EPI_WARPS = 8;
    static constexpr int THREADS = 64 + EPI_WARPS * 32;
    static constexpr int SMEM = STAGES * STAGE + EPI_WARPS * OUT_BYTES + 1024 + (2 * STAGES + 2 * NBUF) * 8 + 16;
};

template <int BNP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairCfg<BNP>::THREADS, 1)
linear_quant_pair_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, const Args a) {
    using C = PairCfg<BNP>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char* out = ring + C::STAGES * C::STAGE;
    uint64_t* bars = reinterpret_cast<uint64_t*>(out + C::EPI_WARPS * C::OUT_BYTES);   // full, empty [STAGES]; tfull, tempty [NBUF]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * C::STAGES + 2 * C::NBUF);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;   // (uniform, and known to be)
    const uint32_t rank = cluster_ctarank();
    const int cluster = (int)blockIdx.x >> 1, n_clusters = (int)gridDim.x >> 1;
    const int tiles = a.m_tiles * ((a.N + BNP - 1) / BNP);

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
            mbar_init(tempty(b), 2 * C::EPI_WARPS);                // both blocks' epilogue warps
        }
        *abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == 0 && lane == 0) {
        prefetch_tensormap(&tm_w);
        prefetch_tensormap(&tm_x);
        const int n0 = cluster / a.m_tiles * BNP + (int)rank * C::HALF;
        for (int i = 0; i < a.groups && i < C::STAGES && n0 < a.N; ++i) tma_prefetch_2d(&tm_w, i * GROUP, n0);
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), 512);
    pdl_trigger();
    tcgen05_fence_before();
    __syncthreads();
    cluster_sync();                                                // the peer's barriers exist before anything signals them
    tcgen05_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();

    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int t = cluster; t < tiles && ok; t += n_clusters) {
                const int m0 = t % a.m_tiles * 256 + (int)rank * 128, n0 = t / a.m_tiles * BNP + (int)rank * C::HALF;
                for (int i = 0; i < a.groups; ++i, ++it) {
                    const int s = it % C::STAGES;
                    if (!mbar_wait(empty(s), ((uint32_t)(it / C::STAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                    if (rank == 0) mbar_expect_tx(full(s), 2u * C::STAGE);
                    const uint32_t lead_full = map_to_cta(full(s), 0);
                    tma_load_2d_pair(ring_addr + s * C::STAGE + C::X_BYTES, &tm_w, i * GROUP, n0, lead_full);
                    tma_load_2d_pair(ring_addr + s * C::STAGE, &tm_x, i * GROUP, m0, lead_full);
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc = make_idesc_e4m3_pair(BNP);
            const bool leader = elect_one();
            int it = 0;
            bool ok = true;
            for (int t = cluster; t < tiles && ok; t += n_clusters) {
                for (int i = 0; i < a.groups; ++i, ++it) {
                    const int s = it % C::STAGES, b = it % C::NBUF;
                    ok = mbar_wait(tempty(b), ((uint32_t)(it / C::NBUF) & 1u) ^ 1u, abort_flag) &&
                         mbar_wait(full(s), (uint32_t)(it / C::STAGES) & 1u, abort_flag);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tcgen05_fence_after();
                    const uint64_t xd = smem_desc_sw128_kmajor(ring_addr + s * C::STAGE);
                    const uint64_t wd = smem_desc_sw128_kmajor(ring_addr + s * C::STAGE + C::X_BYTES);
                    if (leader) {
#pragma unroll
                        for (int kk = 0; kk < GROUP / 32; ++kk)
                            umma_f8_ss_pair(tmem_base + (uint32_t)(b * BNP), xd + (uint64_t)(kk * 2), wd + (uint64_t)(kk * 2), idesc, kk != 0 ? 1u : 0u);
                        umma_commit_pair(tfull(b), 3);
                        umma_commit_pair(empty(s), 3);
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        const int quarter = warp & 3, half = (warp - 2) >> 2;      // TMEM lanes; which half of the columns
        const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * C::HALF);
        const uint32_t lead_tempty = map_to_cta(tempty(0), 0);
        int it = 0;
        bool alive = true;
        for (int t = cluster; t < tiles && alive; t += n_clusters) {
            const int m = t % a.m_tiles * 256 + (int)rank * 128 + quarter * 32 + lane;
            const int n0 = t / a.m_tiles * BNP + half * C::HALF;
            const float* xs = a.x_scale + (size_t)(m < a.M ? m : 0) * a.groups;
            const float* ws = a.w_scale + (size_t)(n0 < a.N ? n0 / GROUP : 0) * a.groups;
            uint64_t acc[C::HALF / 2];
#pragma unroll
            for (int j = 0; j < C::HALF / 2; ++j) acc[j] = 0;
            float nx = xs[0], nw = ws[0];
            if (a.residual && m < a.M) {                           // on its way to L2 while the products run
#pragma unroll
                for (int c = 0; c < C::HALF; c += 64)
                    if (n0 + c < a.N) asm volatile("prefetch.global.L2 [%0];" ::"l"(a.residual + (size_t)m * a.N + n0 + c));
            }
            for (int i = 0; i < a.groups; ++i, ++it) {
                const int b = it % C::NBUF;
                const float sc = nx * nw;
                if (i + 1 < a.groups) {                            // the next column group's scales
                    nx = xs[i + 1];
                    nw = ws[i + 1];
                }
                const bool got = mbar_wait(tfull(b), (uint32_t)(it / C::NBUF) & 1u, abort_flag);
                if (!__all_sync(0xffffffffu, got)) { alive = false; break; }
                tcgen05_fence_after();
                const uint64_t s2 = pack_f32x2(sc, sc);
                uint32_t r[2][16];
                TMEM_LD_X16(t_lane + (uint32_t)(b * BNP), r[0]);
#pragma unroll
                for (int c = 0; c < C::HALF; c += 16) {
                    tmem_wait_ld();
                    if (c + 16 < C::HALF) {
                        TMEM_LD_X16(t_lane + (uint32_t)(b * BNP + c + 16), r[(c / 16 + 1) & 1]);
                    } else {                                       // the accumulator has been read
                        tcgen05_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_peer(lead_tempty + 8u * b);
                    }
                    const uint32_t(&v)[16] = r[(c / 16) & 1];
#pragma unroll
                    for (int j = 0; j < 16; j += 2) fma_f32x2(acc[(c + j) / 2], v[j], v[j + 1], s2);
                }
            }
            if (!alive) continue;
            // 64 columns at a time through shared memory: a row per lane there, four rows of 128 bytes per instruction in global
            // memory (a row per lane would touch 32 lines with each; 512 x 4096 x 24576: 61.4 us so, 56.0 like this).  The residual is
            // read by rows all the same: through shared memory its loads would wait for one another (80 against 69 us).
            unsigned char* mine = out + (warp - 2) * C::OUT_BYTES;
            const int piece = lane & 7, m_warp = m - lane;
            auto at = [&](int r, int x) { return reinterpret_cast<uint4*>(mine + r * 128 + ((x ^ (r & 7)) << 4)); };
#pragma unroll
            for (int c0 = 0; c0 < C::HALF; c0 += 64) {
                const int col = n0 + c0 + piece * 8;               // (N is a multiple of 16, a piece 8 columns)
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; j += 2) unpack_f32x2(acc[(c0 + x * 8 + j) / 2], v[j], v[j + 1]);
                    if (a.residual && m < a.M && n0 + c0 + x * 8 < a.N) {
                        float r[8];
                        quant::unpack_bf16x8(*reinterpret_cast<const uint4*>(a.residual + (size_t)m * a.N + n0 + c0 + x * 8), r);
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += r[j];
                    }
                    *at(lane, x) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
                }
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int r = q * 4 + (lane >> 3);
                    if (m_warp + r < a.M && col < a.N) *reinterpret_cast<uint4*>(a.y + (size_t)(m_warp + r) * a.N + col) = *at(r, piece);
                }
                __syncwarp();
            }
        }
    }

    // ---- tear-down: neither block leaves while the other may still signal it or read its shared memory ----
    tcgen05_fence_before();
    __syncthreads();
    if (*abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(10000);
        __syncthreads();
    }
    cluster_sync();
    if (warp == 1) {
        __syncwarp();
        tcgen05_fence_after();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

static int operand_maps(CUtensorMap* tm_w, CUtensorMap* tm_x, const Args& a, const void* w, const void* x, uint32_t w_rows, uint32_t x_rows) {
    const uint64_t str[1] = {(uint64_t)a.K};
    const uint64_t dims_w[2] = {(uint64_t)a.K, (uint64_t)a.N}, dims_x[2] = {(uint64_t)a.K, (uint64_t)a.M};
    const uint32_t box_w[2] = {GROUP, w_rows}, box_x[2] = {GROUP, x_rows};
    const int rc = make_map_u8(tm_w, w, 2, dims_w, str, box_w);
    return rc != DEER_OK ? rc : make_map_u8(tm_x, x, 2, dims_x, str, box_x);
}

template <int BNP>
int launch_pair(Args a, const void* x, const void* w, cudaStream_t st) {
    using C = PairCfg<BNP>;
    static_assert(C::SMEM <= 227 * 1024, "a block's shared memory");
    CUtensorMap tm_w, tm_x;
    const int rc = operand_maps(&tm_w, &tm_x, a, w, x, C::HALF, 128);
    if (rc != DEER_OK) return rc;
    a.m_tiles = (a.M + 255) / 256;
    const long long tiles = (long long)a.m_tiles * ((a.N + BNP - 1) / BNP);
    DEER_CHECK_ARG(tiles <= 0x3fffffffLL, DEER_ERR_UNSUPPORTED, "deer_linear_quant: too many tiles");
    const long long clusters = tiles < deer_sm_count() / 2 ? tiles : deer_sm_count() / 2;
    DEER_CUDA(cudaFuncSetAttribute(linear_quant_pair_kernel<BNP>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM));
    DEER_CUDA(launch_pdl(linear_quant_pair_kernel<BNP>, dim3((unsigned)(2 * clusters)), dim3(C::THREADS), (size_t)C::SMEM, st, tm_w, tm_x, a));
    return DEER_OK;
}

template <int NT>
int launch(Args a, const void* x, const void* w, cudaStream_t st) {
    using C = Cfg<NT>;
    static_assert(2 * (C::SMEM + 1024) <= 228 * 1024, "two blocks (each with a system kilobyte) on an SM");
    CUtensorMap tm_w, tm_x;
    const int rc = operand_maps(&tm_w, &tm_x, a, w, x, BN, NT);
    if (rc != DEER_OK) return rc;
    a.m_tiles = (a.M + NT - 1) / NT;
    const long long tiles = (long long)((a.N + BN - 1) / BN) * a.m_tiles;
    // As many blocks to a cluster as still fit beside each other (two per SM), with at least four column groups each.
    const long long room = 2LL * deer_sm_count();
    a.split = 1;
    while (a.split < MAX_SPLIT && tiles * a.split * 2 <= room && a.groups >= a.split * 2 * 4) a.split *= 2;
    DEER_CHECK_ARG(tiles * a.split <= 0x7fffffffLL, DEER_ERR_UNSUPPORTED, "deer_linear_quant: too many tiles");
    DEER_CUDA(cudaFuncSetAttribute(linear_quant_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM));
    DEER_CUDA(launch_pdl_cluster(a.split, linear_quant_kernel<NT>, dim3((unsigned)(tiles * a.split)), dim3(C::THREADS), C::SMEM, st, tm_w, tm_x, a));
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
    DEER_CHECK_ARG(M <= 1 << 30 && N <= 1 << 30 && K <= 1 << 30, DEER_ERR_UNSUPPORTED, "deer_linear_quant: M, K and N must be at most 2^30");
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
    // Pairs: the tiles of the product are done in rounds of one per pair of SMs; a round of 128 weight rows takes 0.57 of
    // one of 256 (512 rows, 12288 x 4096, one round: 34.0 / 58.4 us; 4096 x 24576, six rounds or three: 80.4 / 75.3).
    const long long pairs = deer_sm_count() / 2, m_tiles = (M + 255) / 256;
    const long long wide = (m_tiles * ((N + 255) / 256) + pairs - 1) / pairs, narrow = (m_tiles * ((N + 127) / 128) + pairs - 1) / pairs;
    // The first kernel above 32 rows: where its tiles leave room for four blocks each at the least, or there are not more rows
    // than one of them has (us, first kernel / pairs: 128 x 4096 x 4096 13.2 / 14.3, 128 x 12288 x 4096 23.9 / 33, 128 x 4096 x 8192
    // 21.7 / 14.5, 256 x 4096 x 4096 20.2 / 14.5, 64 x 4096 x 24576 34.5 / 41.4); but not where the product is so shallow that one round
    // of pairs is over before a cluster has met (64 x 256 x 1024 8.4 / 4.8, 64 x 1536 x 4096 9.8 / 7.5, 64 x 2048 x 256 7.2 / 8.1).
    const bool room = M <= 64 || (long long)((M + 63) / 64) * ((N + BN - 1) / BN) <= pairs;
    const bool shallow = a.groups <= 12 && narrow == 1;
    if (room && !shallow) return launch<64>(a, x, w, st);
    return narrow * 57 < wide * 100 ? launch_pair<128>(a, x, w, st) : launch_pair<256>(a, x, w, st);
}
