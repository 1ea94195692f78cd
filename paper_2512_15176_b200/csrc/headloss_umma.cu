// The products of the LM head's losses on the tensor cores:
//
//   STATS  z = h w^T                 [live][V]      rows of h on the lanes, contraction hid; eight warps per block beside
//                                                   it compute the listed tokens' z once more on the CUDA cores
//   GRAD   G = coef (p - t)          [live][piece]  the same z again, softmax and targets in the epilogue
//   BACK   dh = G w                  [live][hid]    contraction over the piece's vocabulary, in ranges
//          dw = G^T h                [piece][hid]   contraction over the live rows
//
// One kernel body; the two products of BACK share a launch, so that the many short tiles of dw fill what the few long ones
// of dh leave of the last wave.  Pairs of blocks (tcgen05.mma.cta_group::2, 256 x n tiles, n <= 256, fp32 accumulators in two
// tensor-memory buffers) walk a list of tiles: a warp per block brings 64-deep steps of both operands by TMA into a ring
// of as many stages as fit, one warp of the pair issues the MMAs, eight warps per block (BACK: four) take the finished tile
// while the next one is computed.  Up to ONE_BLOCK rows STATS and GRAD take single blocks, whose 128 rows pairs would leave
// half empty.  h and G are stored row-major once; where the contraction runs along their rows (dw, and w in dh) the
// operand is read MN-major: boxes of 64 contraction rows x 64 columns, two of them side by side.
//
// 1024 rows x 32768 x 2048, each launch alone and cold: STATS 95 us (tensor pipe 77 % busy), GRAD 96 (76 %), BACK 186 (81 %):
// the tensor cores bound them.  96 rows x 65536 x 2048: 48, 54 and 112 us for 270, 282 and 534 MB of HBM traffic: memory does,
// and in dw's part the way out of the SMs.
//
// G is rounded to bf16 for the products: as much as dh and dw are themselves, and with many rows the errors of different
// rows are as independent as theirs.  At a listed token p - t is formed in fp32 first, so that a target the model is sure of
// keeps its difference.  coef is taken relative to a scale of the whole call, of which head_factor_kernel tries 32 between
// two powers of two for the one at which rounding takes the least from the listed tokens, so that a few heavy rows do not
// decide the gradient's error.  With few live rows (TWO_TERMS) a single rounding would show in a whole gradient, and there
// G is kept as two bf16 terms: 1 % of the gradients' time at 20 rows x 151936 x 2048 (363 us and 359 with one), 5 % at 64 and
// 128 (385 and 369, 409 and 389).  lse, p and all sums are fp32.
//
// The tensor cores' accumulation rounds towards zero at every step (tile_scale_of).  Where a target stands out the loss is the
// difference of two large numbers, lse and the target's z: hence the listed tokens' z a second time, as plain fp32 sums (4 %
// of the products' bytes at lists of 64, hidden behind them).  The loss takes those, and lse the difference that they make.
#include <math.h>

#include <type_traits>

#include "headloss.cuh"
#include "sm100.cuh"

using namespace sm100;

namespace headloss {

constexpr int BOX = 4096;                  // 32 rows x 128 bytes of a finished tile, as they leave through TMA
constexpr int DOT_WARPS = 8;
// What a variant is made of: P the product, CG the blocks that share a tile.
template <int P, int CG>
struct Shape {
    static constexpr int A = 16384;                        // a block's share of an operand's step: 128 rows (columns) x 64 bf16
    static constexpr int B = 32768 / CG;                   // n columns, or this block's half of them
    static constexpr int EPI = P == BACK ? 4 : 8;          // epilogue warps: with eight, two share a quarter of the lanes
    static constexpr int STAGING = P == STATS ? EPI * BOX : EPI * 2 * BOX;
    static constexpr int STAGES = (232448 - STAGING - 1024 - 256) / (A + B);
    static constexpr int SMEM = STAGES * (A + B) + STAGING + 1024 /*alignment*/ + 256 /*barriers*/;
    static constexpr int THREADS = 64 + 32 * EPI + (P == STATS ? 32 * DOT_WARPS : 0);
    static constexpr int ROWS = 128 * CG;                  // lanes of a tile
};
static_assert(Shape<STATS, 1>::EPI == 4 * STATS_SHARE && Shape<STATS, 2>::EPI == 4 * STATS_SHARE, "partial sums of a tile");
constexpr int ACC = 256;                   // columns of one accumulator

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void tma_reduce_add_2d(const CUtensorMap* tm, uint32_t src, int x, int y) {
    asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tm), "r"(src), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void st_shared_bf16(uint32_t addr, __nv_bfloat16 v) {
    asm volatile("st.shared.b16 [%0], %1;" ::"r"(addr), "h"(__bfloat16_as_ushort(v)) : "memory");
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float ld_shared_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// kind::f16 instruction descriptor: bf16 x bf16 -> fp32, M = 128 of each block, N = n.
template <int CG>
__device__ __forceinline__ uint32_t idesc_of(int n, bool a_mn, bool b_mn) {
    return (CG == 2 ? make_idesc_bf16_pair(n) : make_idesc_bf16(n, 0)) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
}

// A tile: rows and columns of the product, range of the contraction in steps.
struct Tile {
    int r, c, k0, kb;
    int y;                     // dh: row of the slabs
    bool dw;                   // BACK: of dw
};
// The tiles of the launch, and those of one block or pair among them, in its order.
template <int P, int CG>
struct List {
    int live, steps, mt, ct, low, ranges, dw_steps, n, n_dw, group, groups;    // low: place of the second term's rows, 0: none
    int mine, light, ahead;
    __device__ __forceinline__ List(const ProductArgs& a) {
        live = P == STATS && a.as_is ? a.M : a.hdr_in[HDR_LIVE];
        mt = (live + Shape<P, CG>::ROWS - 1) / Shape<P, CG>::ROWS;
        ct = a.col_tiles;
        low = P != STATS && live <= TWO_TERMS ? low_term(live) : 0;
        group = blockIdx.x / CG;
        groups = gridDim.x / CG;
        if (P != BACK) {
            steps = a.hid / STEP;
            n = mt * ct;
            return;
        }
        steps = (a.vn + STEP - 1) / STEP;
        ranges = a.hdr_in[HDR_RANGES];
        dw_steps = dw_contraction(live);
        n = a.want_dh ? mt * ct * ranges : 0;
        n_dw = a.row_tiles * ct;
        // dh's tiles first, in turn; groups that have one of them less take `ahead` of dw's before the others begin
        mine = group < n ? (n - group + groups - 1) / groups : 0;
        light = n % groups ? groups - n % groups : 0;
        ahead = light ? dh_tile_cost(steps, ranges) / dw_tile_cost(dw_steps) : 0;
    }
    // The group's k-th tile; false behind its last.
    __device__ __forceinline__ bool tile(int k, Tile& t) const {
        t.k0 = t.y = 0;
        t.kb = steps;
        t.dw = false;
        int u = group + k * groups;
        if (P != BACK) {                    // row tiles fastest: the groups share a few tiles of w at a time
            if (u >= n) return false;
            t.r = u % mt;
            t.c = u / mt;
            return true;
        }
        if (k < mine) {                     // columns (of hid) fastest: the groups share tiles of G
            const int q = u / ct, s = q / mt;
            t.c = u - q * ct;
            t.y = q * TILE;
            t.r = q - s * mt;
            t.k0 = (int)((long)s * steps / ranges);
            t.kb = (int)((long)(s + 1) * steps / ranges) - t.k0;
            return true;
        }
        k -= mine;
        const int first = group - (groups - light);      // the group's place among the light ones
        u = light && first >= 0 ? (k < ahead ? k * light + first : light * ahead + (k - ahead) * groups + group)
                                : light * ahead + k * groups + group;
        if (u >= n_dw) return false;
        t.dw = true;
        t.r = u / ct;
        t.c = u - t.r * ct;
        t.kb = dw_steps;
        return true;
    }
};

// z of the listed tokens by plain fp32 sums: a warp takes four entries of a row at a time.
__device__ __forceinline__ void listed_logits(const ProductArgs& a, int live, int warp, int warps, int lane) {
    const int groups = (a.K + 3) / 4;
    for (long i = warp; i < (long)live * groups; i += warps) {
        const int slot = (int)(i / groups), e0 = (int)(i % groups) * 4, m = a.as_is ? slot : a.row[slot];
        if (a.as_is && !is_live(a.list, a.weight, a.K, m)) continue;
        const __nv_bfloat16* w[4];
        bool on[4], any = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int id = e0 + j < a.K ? a.list[(size_t)m * a.K + e0 + j] : -1;
            on[j] = id >= 0 && id < a.V;      // (an entry behind a list's end may be summed: what it gives is not read)
            any |= on[j];
            w[j] = a.w + (on[j] ? (size_t)id * a.hid : 0);
        }
        if (!any) continue;
        const __nv_bfloat16* h = a.h + (size_t)slot * a.hid;
        float sum[4][2] = {};
        for (int c0 = lane * 8; c0 < a.hid; c0 += 512) {
            uint4 x[2], y[2][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int c = c0 + u * 256;
                x[u] = c < a.hid ? *reinterpret_cast<const uint4*>(h + c) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[u][j] = on[j] && c < a.hid ? *reinterpret_cast<const uint4*>(w[j] + c) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t ys[4] = {y[u][j].x, y[u][j].y, y[u][j].z, y[u][j].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        sum[j][0] = fmaf(__uint_as_float(xs[k] << 16), __uint_as_float(ys[k] << 16), sum[j][0]);
                        sum[j][1] = fmaf(__uint_as_float(xs[k] & 0xffff0000u), __uint_as_float(ys[k] & 0xffff0000u), sum[j][1]);
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float s = sum[j][0] + sum[j][1];
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == 0 && on[j]) a.target_logit[(size_t)m * a.K + e0 + j] = s;
        }
    }
}

// The listed tokens of one row in rising order, from the tile's first column on: `id` is the next, INT_MAX behind the last.
// What belongs to an entry comes one entry ahead.
struct Listed {
    int id = 0x7fffffff, e = 0, next = 0x7fffffff;
    float val = 0.f, next_val = 0.f;           // GRAD: G at the token
    __device__ __forceinline__ int id_at(const ProductArgs& a, int slot, int i) const { return i < a.K ? a.ids[(size_t)slot * a.K + i] : 0x7fffffff; }
    // lists by rising id, from entry `at` on
    template <bool VALUES>
    __device__ __forceinline__ void start(const ProductArgs& a, int slot, int at) {
        e = at;
        id = id_at(a, slot, e);
        next = id_at(a, slot, e + 1);
        if (VALUES) {
            val = e < a.K ? a.gval[(size_t)slot * a.K + e] : 0.f;
            next_val = e + 1 < a.K ? a.gval[(size_t)slot * a.K + e + 1] : 0.f;
        }
    }
    template <bool VALUES>
    __device__ __forceinline__ void advance(const ProductArgs& a, int slot) {
        ++e;
        id = next;
        val = next_val;
        next = id_at(a, slot, e + 1);
        if (VALUES) next_val = e + 1 < a.K ? a.gval[(size_t)slot * a.K + e + 1] : 0.f;
    }
    // a short list as it is; with `store`, z goes to the first entry that names from - 1
    __device__ __forceinline__ void search(const ProductArgs& a, int m, int from, bool store, float z) {
        id = 0x7fffffff;
        bool open = true;
        for (int j0 = 0; j0 < a.K; j0 += 4) {
            int at[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) at[i] = j0 + i < a.K ? a.list[(size_t)m * a.K + j0 + i] : -1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                open &= at[i] >= 0;
                if (open && at[i] >= from) id = min(id, at[i]);
                if (open && store && at[i] == from - 1) {
                    a.z[(size_t)m * a.K + j0 + i] = z;
                    store = false;
                }
            }
            if (!open) break;
        }
    }
};

template <int P, int CG>
__device__ __forceinline__ void epilogue(const ProductArgs& a, const CUtensorMap* tm_out, const CUtensorMap* tm_out_dw, const List<P, CG>& list, int warp, int lane, int rank,
                                         uint32_t tmem_base, uint32_t tfull0, uint32_t tempty0, uint32_t staging, volatile int* abort_flag) {
    constexpr int SHARE = Shape<P, CG>::EPI / 4;                           // warps to a quarter of the lanes: they take its columns in turn
    const int quarter = warp & 3, turn = (warp - 2) >> 2;
    const uint32_t stg = staging + (uint32_t)(warp - 2) * (2u * BOX), stg_row = (uint32_t)lane * 128u, sw = (uint32_t)(lane & 7);
    const int lane_row = rank * 128 + quarter * 32 + lane;                 // the thread's row within a tile
    const float factor = P == GRAD ? __int_as_float(a.hdr_in[HDR_FACTOR]) : 1.f;
    uint32_t stg_i = 0;
    int it = 0;
    // what a tile needs of its rows comes one tile ahead: where a row's list stands at the tile's first column, G's scale
    constexpr bool BY_ROWS = P == STATS || P == GRAD;
    struct Row {
        float coef = 0.f, nlse = 0.f;
        int e = 0;
    } row, row_ahead;
    auto place_of = [&](const Tile& t) { return t.r * Shape<P, CG>::ROWS + lane_row; };
    auto load_row = [&](const Tile& t, Row& r) {
        const int slot = place_of(t);
        if (slot >= list.live) return;
        if (P == GRAD) {
            r.coef = a.coef[slot];
            r.nlse = -a.lse2[slot];
        }
        if (P == GRAD || !a.as_is) r.e = a.first[(size_t)slot * a.first_pitch + a.first_tile + t.c];
    };
    Tile t, t_ahead;
    bool more = list.tile(0, t), more_ahead;
    if (BY_ROWS && more) load_row(t, row);
    for (int k = 0; more; ++k, t = t_ahead, more = more_ahead, row = row_ahead) {
        more_ahead = list.tile(k + 1, t_ahead);
        if (t.kb == 0 && !t.dw) continue;                                 // dh: nothing to add; dw without a live row: zeros
        const int buf = it & 1;
        const bool computed = t.kb > 0;
        const int slot = place_of(t);                                     // STATS, GRAD: place among the live rows
        const bool row_ok = BY_ROWS && slot < list.live && (P != STATS || !a.as_is || is_live(a.list, a.weight, a.K, slot));
        const int col0 = t.c * a.n;
        const float coef = row.coef * factor, nlse = row.nlse;
        Listed listed;
        if (BY_ROWS) {
            if (row_ok) {
                if (P == STATS && a.as_is) listed.search(a, slot, col0, false, 0.f);
                else listed.start<P == GRAD>(a, slot, row.e);
            }
            if (more_ahead) load_row(t_ahead, row_ahead);
        }
        if (computed) {
            const bool got = mbar_wait(tfull0 + 8u * buf, (uint32_t)(it >> 1) & 1u, abort_flag);
            if (!__all_sync(0xffffffffu, got)) break;                     // warp-uniform, so the aligned TMEM loads stay converged
            tcgen05_fence_after();
            ++it;
        }
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * ACC);

        if (P == STATS) {
            const int width = min(a.n, a.vn - col0);                      // columns that exist
            const bool idle = !__any_sync(0xffffffffu, row_ok);           // (lanes behind the last row)
            float run_m = -INFINITY, run_s = 0.f;
            for (int c = 32 * turn; c < width && !idle; c += 32 * SHARE) {
                uint32_t v[32];
                __syncwarp();                                             // the rows' lists part the lanes; TMEM loads want all of them together
                TMEM_LD_X32(taddr + c, v);
                tmem_wait_ld();
                const int have = width - c;
                if (have < 32) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j >= have) v[j] = 0xff800000u;
                }
                float m4[4] = {__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3])};
#pragma unroll
                for (int j = 4; j < 32; ++j) m4[j & 3] = fmaxf(m4[j & 3], __uint_as_float(v[j]));
                float m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                // relative to a whole row's reference in powers of two: rounded where it is small, not where z is
                m = fmaxf(m * a.c2, run_m);
                const float shift = m == -INFINITY ? 0.f : m;              // a row of -inf so far: its exponentials are 0
                run_s *= ex2(run_m - shift);
                run_m = m;
                float s4[4] = {};
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float x = __uint_as_float(v[j]);
                    s4[j & 3] += ex2(fmaf(x, a.c2_low, fmaf(x, a.c2, -shift)));
                }
                run_s += (s4[0] + s4[1]) + (s4[2] + s4[3]);
                // the z of the row's listed tokens among these columns, by way of shared memory: registers have no index
                const int begin = col0 + c, end = col0 + min(c + 32, width);
                if (listed.id < end) {
                    const uint32_t line = staging + (uint32_t)(warp - 2) * BOX + stg_row;
#pragma unroll
                    for (uint32_t j = 0; j < 8; ++j) st_shared_v4(line + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                    do {
                        const bool here = listed.id >= begin;              // (the other warp's columns lie between this one's)
                        const uint32_t k = here ? (uint32_t)(listed.id - begin) : 0;
                        const float z = ld_shared_f32(line + (((k >> 2) ^ sw) << 4) + (k & 3) * 4);
                        if (a.as_is) {
                            listed.search(a, slot, listed.id + 1, here, z);
                        } else {
                            if (here) a.z[(size_t)slot * a.K + listed.e] = z;
                            listed.advance<false>(a, slot);
                        }
                    } while (listed.id < end);
                }
            }
            if (row_ok) a.part[(size_t)slot * a.tiles + t.c * SHARE + turn] = make_float2(run_m, run_s);
        } else if (P == GRAD || t.dw) {
            const int limit = P == GRAD ? a.vn : a.hid;
            const float scale = P == BACK ? __int_as_float(a.hdr_in[HDR_SCALE]) : 1.f;
            const bool two = P == GRAD && list.low > 0;
            const bool idle = two && (rank > 0 || quarter * 32 >= list.low);        // no rows of the first term
            for (int c = 64 * turn; c < a.n && col0 + c < limit && !idle; c += 64 * SHARE) {
                const int wide = min(64, a.n - c);                        // (the last chunk may be narrower than a box)
                // the store from this box two chunks ago has read it (two terms: both boxes are used at once)
                if (lane == 0) {
                    if (two) bulk_wait_read<0>();
                    else bulk_wait_read<1>();
                }
                __syncwarp();
                const uint32_t box = stg + stg_i * BOX, b = box + stg_row, other = BOX - 2u * BOX * stg_i;
                if (!two) stg_i ^= 1;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t v[32];
                    if (computed) {
                        TMEM_LD_X32(taddr + c + 32 * half, v);
                        tmem_wait_ld();
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = 0;
                    }
                    uint32_t o[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float x = __uint_as_float(v[2 * j]), y = __uint_as_float(v[2 * j + 1]);
                        if (P == GRAD) {
                            x = coef * ex2(fmaf(x, a.c2, nlse));
                            y = coef * ex2(fmaf(y, a.c2, nlse));
                            if (!row_ok) x = y = 0.f;                     // places behind the live rows: dw's contraction meets them
                        } else {
                            x *= scale;
                            y *= scale;
                        }
                        o[j] = pack_bf16(x, y);
                        if (P == GRAD && two) v[j] = pack_bf16(x - __uint_as_float(o[j] << 16), y - __uint_as_float(o[j] & 0xffff0000u));
                    }
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j)
                        st_shared_v4(b + (((4 * half + j) ^ sw) << 4), o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                    if (P == GRAD && two)
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j)
                            st_shared_v4(b + other + (((4 * half + j) ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                }
                if (P == GRAD) {
                    const int first = a.v0 + col0 + c;
                    while (listed.id < first + wide) {                    // listed tokens: p - t, formed in fp32 beforehand
                        if (listed.id >= first) {                         // (the other warp's chunks lie between this one's)
                            const uint32_t k = (uint32_t)(listed.id - first);
                            const float val = listed.val * factor;
                            const __nv_bfloat16 hi = __float2bfloat16(val), lo = __float2bfloat16(val - __bfloat162float(hi));
                            const uint32_t at = b + (((k >> 3) ^ sw) << 4) + (k & 7) * 2;
                            st_shared_bf16(at, hi);
                            if (two) st_shared_bf16(at + other, lo);
                        }
                        listed.advance<true>(a, slot);
                    }
                }
                const int y = (P == BACK ? a.v0 : 0) + t.r * Shape<P, CG>::ROWS + rank * 128 + quarter * 32;
                if (wide < 64) {                                          // by plain stores, 16 bytes of a row at a time
                    const int pitch = P == GRAD ? a.g_pitch : a.hid;
                    __nv_bfloat16* row = (P == GRAD ? a.g : a.dw) + (size_t)(y + lane) * pitch + col0 + c;
                    const int stop = P == GRAD || y + lane < a.V ? min(wide, pitch - col0 - c) : 0;
                    for (int k = 0; k < stop; k += 8) {
                        *reinterpret_cast<uint4*>(row + k) = ld_shared_v4(b + (((uint32_t)(k >> 3) ^ sw) << 4));
                        if (two) *reinterpret_cast<uint4*>(row + (size_t)list.low * pitch + k) = ld_shared_v4(b + other + (((uint32_t)(k >> 3) ^ sw) << 4));
                    }
                    if (!two) stg_i ^= 1;                                 // no store by TMA has taken this box: it is next again
                    continue;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0 && (P == GRAD || y < a.V)) {                // rows and columns beyond the tensor are clipped
                    tma_store_2d(P == BACK ? tm_out_dw : tm_out, box, col0 + c, y);
                    if (two) tma_store_2d(tm_out, box + other, col0 + c, list.low + quarter * 32);
                    bulk_commit();
                }
            }
        } else {                                                          // dh: fp32, 32 columns to a box
            for (int c = 32 * turn; c < a.n && col0 + c < a.hid; c += 32 * SHARE) {
                if (lane == 0) bulk_wait_read<1>();
                __syncwarp();
                const uint32_t box = stg + stg_i * BOX, b = box + stg_row;
                stg_i ^= 1;
                uint32_t v[32];
                TMEM_LD_X32(taddr + c, v);
                tmem_wait_ld();
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j) st_shared_v4(b + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    const int y = t.y + rank * 128 + quarter * 32;
                    if (a.add) tma_reduce_add_2d(tm_out, box, col0 + c, y);
                    else tma_store_2d(tm_out, box, col0 + c, y);
                    bulk_commit();
                }
            }
        }
        if (computed) {
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) mbar_arrive_peer(map_to_cta(tempty0 + 8u * buf, 0));
                else mbar_arrive(tempty0 + 8u * buf);
            }
        }
    }
    if (lane == 0) bulk_wait_read<0>();          // the staging area outlives every store that reads it
}

// BACK: the operands and the result of dw's product.
struct DwMaps {
    CUtensorMap a, b, out;
};

template <int CG>
__device__ __forceinline__ void load_2d(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
    if (CG == 2) tma_load_2d_pair(dst, tm, x, y, bar);
    else tma_load_2d(dst, tm, x, y, bar);
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t accumulate) {
    if (CG == 2) umma_bf16_ss_pair(d, ad, bd, idesc, accumulate);
    else umma_bf16_ss(d, ad, bd, idesc, accumulate);
}
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
    if (CG == 2) umma_commit_pair(bar, 3);
    else umma_commit(bar);
}

template <int P, int CG>
__global__ void __launch_bounds__(Shape<P, CG>::THREADS, 1)
product_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_out,
               const __grid_constant__ DwMaps dw, const ProductArgs a) {
    using S = Shape<P, CG>;
    constexpr int STAGES = S::STAGES, STAGE_BYTES = S::A + S::B;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + STAGES * STAGE_BYTES + S::STAGING);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    constexpr bool B_MN = P == BACK;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_ctarank() : 0;
    const bool leader = rank == 0;
    const uint32_t smem_base = smem_u32(smem), bar_base = smem_u32(bars);
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
    const uint32_t tfull0 = bar_base + 8u * (2 * STAGES), tempty0 = tfull0 + 16u;

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(tfull0 + 8u * b, 1);
            mbar_init(tempty0 + 8u * b, CG * S::EPI);      // the epilogue warps of all blocks
        }
        *abort_flag = 0;
        mbar_init_fence();
        prefetch_tensormap(&tm_a);
        prefetch_tensormap(&tm_b);
    }
    if (warp == 1) {
        if (CG == 2) tmem_alloc_pair(smem_u32(tmem_slot), 512);
        else tmem_alloc(smem_u32(tmem_slot), 512);
    }
    pdl_trigger();
    tcgen05_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();                 // the peer's barriers exist before anything signals them
    tcgen05_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_wait();                                  // (the weights too: in training an optimiser step may be what ran before)
    const List<P, CG> list(a);

    if (warp == 0) {
        // ---------------- TMA producer (each block: its rows of one operand, its half of the columns of the other) --------
        if (lane == 0) {
            const int half = a.n / CG;                                     // columns of the tile that this block brings
            // the second block's rows: those behind the first 128, or (dh) the second term
            const bool second_a = CG == 2 && (list.live > 128 || (P == BACK && list.low > 0)), has_a = leader || second_a;
            const int a_step = P == BACK && list.low > 0 ? list.low : 128;
            const int b_boxes = B_MN ? (half + 63) / 64 : 1;
            const uint32_t a_bytes = (uint32_t)a.a_rows * 128u, b_bytes = B_MN ? (uint32_t)b_boxes * 8192u : (uint32_t)half * 128u;
            const uint32_t stage_tx = a_bytes * (second_a ? 2u : 1u) + (uint32_t)CG * b_bytes, dw_tx = CG * (S::A + b_bytes);
            int it = 0;
            bool ok = true;
            Tile t;
            for (int i = 0; ok && list.tile(i, t); ++i) {
                const int ra = t.r * S::ROWS + (int)rank * (t.dw ? 128 : a_step), cb = t.c * a.n + (int)rank * half;
                // one loop for each kind of tile
                auto steps = [&](auto of_dw) {
                    constexpr bool DW = decltype(of_dw)::value;
                    for (int kb = 0; kb < t.kb; ++kb, ++it) {
                        const int s = it % STAGES, k = (t.k0 + kb) * STEP;
                        if (!mbar_wait(empty_bar(s), ((uint32_t)(it / STAGES) & 1u) ^ 1u, abort_flag)) return false;
                        if (leader) mbar_expect_tx(full_bar(s), DW ? dw_tx : stage_tx);
                        const uint32_t full = CG == 2 ? map_to_cta(full_bar(s), 0) : full_bar(s), sa = smem_base + s * STAGE_BYTES, sb = sa + S::A;
                        if (DW) {
                            load_2d<CG>(sa, &dw.a, ra, k, full);
                            load_2d<CG>(sa + 8192, &dw.a, ra + 64, k, full);
                        } else if (has_a) {
                            load_2d<CG>(sa, &tm_a, k, ra, full);
                        }
                        if (B_MN) {
                            const CUtensorMap* tm = DW ? &dw.b : &tm_b;
                            const int y = DW ? k : a.v0 + k;
                            load_2d<CG>(sb, tm, cb, y, full);
                            if (b_boxes > 1) load_2d<CG>(sb + 8192, tm, cb + 64, y, full);
                        } else {
                            load_2d<CG>(sb, &tm_b, k, a.v0 + cb, full);
                        }
                    }
                    return true;
                };
                ok = P == BACK && t.dw ? steps(std::true_type{}) : steps(std::false_type{});
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (first block of the pair) ----------------
        if (leader && lane == 0) {
            int it = 0, done = 0;
            bool ok = true;
            Tile t;
            for (int i = 0; ok && list.tile(i, t); ++i) {
                if (t.kb == 0) continue;
                const int buf = done & 1;
                if (!mbar_wait(tempty0 + 8u * buf, ((uint32_t)(done >> 1) & 1u) ^ 1u, abort_flag)) break;
                ++done;
                tcgen05_fence_after();
                const uint32_t d_tmem = tmem_base + (uint32_t)(buf * ACC);
                auto steps = [&](auto of_dw) {
                    constexpr bool A_MN = decltype(of_dw)::value;
                    const uint32_t idesc = idesc_of<CG>(a.n, A_MN, B_MN);
                    for (int kb = 0; kb < t.kb; ++kb, ++it) {
                        const int s = it % STAGES;
                        if (!mbar_wait(full_bar(s), (uint32_t)(it / STAGES) & 1u, abort_flag)) return false;
                        tcgen05_fence_after();
                        const uint32_t sa = smem_base + s * STAGE_BYTES, sb = sa + S::A;
                        // K-major: 16 contraction columns are 32 bytes; MN-major: 16 contraction rows are 2048 bytes
                        const uint64_t ad = A_MN ? smem_desc_sw128(sa, 8192, 1024) : smem_desc_sw128_kmajor(sa);
                        const uint64_t bd = B_MN ? smem_desc_sw128(sb, 8192, 1024) : smem_desc_sw128_kmajor(sb);
#pragma unroll
                        for (int k = 0; k < STEP / 16; ++k)
                            mma<CG>(d_tmem, ad + (A_MN ? 128 : 2) * k, bd + (B_MN ? 128 : 2) * k, idesc, (kb | k) != 0 ? 1u : 0u);
                        commit<CG>(empty_bar(s));
                    }
                    return true;
                };
                ok = P == BACK && t.dw ? steps(std::true_type{}) : steps(std::false_type{});
                if (ok) commit<CG>(tfull0 + 8u * buf);
            }
        }
    } else if (warp >= 2 + S::EPI) {
        if (P == STATS) listed_logits(a, list.live, (int)blockIdx.x * DOT_WARPS + warp - 2 - S::EPI, (int)gridDim.x * DOT_WARPS, lane);
    } else {
        epilogue<P, CG>(a, &tm_out, &dw.out, list, warp, lane, (int)rank, tmem_base, tfull0, tempty0, smem_base + STAGES * STAGE_BYTES, abort_flag);
    }

    // ---- tear-down: neither block leaves while the other may still signal it or read its shared memory ----
    tcgen05_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // the last kernel of the call turns this into NaN
        if (P != STATS && tid == 0) a.hdr[HDR_GAVE_UP] = 1;
        if (P == STATS) {
            Tile t;
            for (int k = 0; list.tile(k, t); ++k)
                for (int i = tid; i < S::ROWS; i += S::THREADS)
                    if (t.r * S::ROWS + i < list.live) a.part[(size_t)(t.r * S::ROWS + i) * a.tiles + t.c * STATS_SHARE] = make_float2(NAN, NAN);
        }
        for (int i = 0; i < 64; ++i) __nanosleep(10000);
        __syncthreads();
    }
    if (CG == 2) cluster_sync();
    if (warp == 1) {
        __syncwarp();
        tcgen05_fence_after();
        if (CG == 2) tmem_dealloc_pair(tmem_base, 512);
        else tmem_dealloc(tmem_base, 512);
    }
}

// 2-D bf16 tensor [rows][cols] of `pitch` columns, box = box_rows x 64 columns.
static int map_bf16(CUtensorMap* tm, const void* base, long rows, long cols, long pitch, int box_rows) {
    const uint64_t dims[2] = {(uint64_t)cols, (uint64_t)rows};
    const uint64_t strides[1] = {(uint64_t)pitch * 2};
    const uint32_t box[2] = {64, (uint32_t)box_rows};
    return make_map_bf16(tm, base, 2, dims, strides, box);
}

template <int P, int CG>
static int launch(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& to, const DwMaps& dw, const ProductArgs& a, long most_tiles,
                  cudaStream_t st) {
    using S = Shape<P, CG>;
    long groups = deer_sm_count() / CG;
    if (groups > most_tiles) groups = most_tiles;
    static bool sized[64] = {};                  // (set again by a thread that has not seen it: harmless)
    int dev = 0;
    DEER_CUDA(cudaGetDevice(&dev));
    if (dev >= 64 || !sized[dev]) {
        DEER_CUDA(cudaFuncSetAttribute(product_kernel<P, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::SMEM));
        if (dev < 64) sized[dev] = true;
    }
    DEER_CUDA(launch_pdl_cluster(CG, product_kernel<P, CG>, dim3((unsigned)(CG * groups)), dim3(S::THREADS), (size_t)S::SMEM, st, ta, tb, to, dw, a));
    return DEER_OK;
}

int launch_product(Product what, const Space& s, const void* h, const void* w, const int* list, const float* weight, int M, int hid, int V, int K,
                   int piece, float tau, float* target_logit, bool want_dh, void* dw, cudaStream_t st) {
    ProductArgs a = {};
    a.M = M;
    a.list = list;
    a.weight = weight;
    a.hdr_in = a.hdr = s.hdr;
    a.hid = hid;
    a.V = V;
    a.K = K;
    tile_scale_of(tau, hid, a.c2, a.c2_low);
    a.ids = s.ids;
    a.row = s.row;
    a.as_is = what == STATS && takes_rows_as_they_are(M, K);
    a.h = a.as_is ? static_cast<const __nv_bfloat16*>(h) : s.h;
    a.w = static_cast<const __nv_bfloat16*>(w);
    a.target_logit = target_logit;
    a.z = s.z;
    a.part = s.part;
    a.coef = s.coef;
    a.lse2 = s.lse2;
    a.gval = s.gval;
    a.first = s.first;
    a.first_pitch = s.first_pitch;
    a.first_tile = what == GRAD ? piece * s.piece_tiles : 0;
    a.g = s.g;
    a.g_pitch = s.piece;
    a.v0 = what == STATS ? 0 : piece * s.piece;
    a.vn = what == STATS ? V : (V - a.v0 < s.piece ? V - a.v0 : s.piece);
    // Fewer rows than a block's 128 are loaded where there are fewer: the MMA reads whatever the stage holds behind
    // them, into lanes that nothing reads back.
    a.a_rows = M < 128 ? (M + 7) / 8 * 8 : 128;
    const int mt = s.Mp / TILE;
    CUtensorMap ta, tb, to;
    DwMaps td;
    int rc;
#define MAP(call)                     \
    do {                              \
        rc = (call);                  \
        if (rc != DEER_OK) return rc; \
    } while (0)
    if (what == STATS || what == GRAD) {
        a.n = what == STATS ? s.stats_n : s.grad_n;
        a.col_tiles = (a.vn + a.n - 1) / a.n;
        a.tiles = a.col_tiles * STATS_SHARE;
        const int cg = M > ONE_BLOCK ? 2 : 1;
        MAP(map_bf16(&ta, a.h, a.as_is ? M : s.Mp, hid, hid, a.a_rows));
        MAP(map_bf16(&tb, w, V, hid, hid, a.n / cg));
        to = td.a = td.b = td.out = ta;
        const long tiles = (long)mt * a.col_tiles;
        if (what == STATS) return cg == 2 ? launch<STATS, 2>(ta, tb, to, td, a, tiles, st) : launch<STATS, 1>(ta, tb, to, td, a, tiles, st);
        MAP(map_bf16(&to, s.g, s.Mp, a.vn, s.piece, 32));
        return cg == 2 ? launch<GRAD, 2>(ta, tb, to, td, a, tiles, st) : launch<GRAD, 1>(ta, tb, to, td, a, tiles, st);
    }
    a.n = s.hid_n;
    a.col_tiles = (hid + a.n - 1) / a.n;
    a.dw = static_cast<__nv_bfloat16*>(dw);
    a.add = piece > 0;
    a.want_dh = want_dh;
    a.row_tiles = dw ? (a.vn + TILE - 1) / TILE : 0;
    // beyond the piece's columns, and its contraction's last step, G reads as zeros
    MAP(map_bf16(&ta, s.g, s.Mp, a.vn, s.piece, a.a_rows));
    MAP(map_bf16(&tb, w, V, hid, hid, 64));
    const uint64_t dims[2] = {(uint64_t)hid, (uint64_t)s.slab_tiles * TILE};
    const uint64_t strides[1] = {(uint64_t)hid * 4};
    const uint32_t box[2] = {32, 32};
    MAP(make_map_f32(&to, s.slab, 2, dims, strides, box));
    MAP(map_bf16(&td.a, s.g, s.Mp, a.vn, s.piece, 64));
    MAP(map_bf16(&td.b, s.h, s.Mp, hid, hid, 64));
    MAP(map_bf16(&td.out, dw ? dw : s.h, dw ? V : s.Mp, hid, hid, 32));
#undef MAP
    return launch<BACK, 2>(ta, tb, to, td, a, ((want_dh ? (long)s.slab_tiles : 0) + a.row_tiles) * a.col_tiles, st);
}

}  // namespace headloss
