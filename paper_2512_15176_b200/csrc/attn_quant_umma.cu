// Block attention against an 8-bit paged cache on the 5th-generation tensor cores (head_dim 128).
//
// The work is split as in the bf16 kernel: a unit is one (sequence, KV head, row tile of 128 query rows), its keys come in
// tiles of 64 -- four full pages, and one last tile for what is bf16, the tail rows and the block's own -- and the tiles
// of all units, laid end to end, are cut into one equal share per thread block (attn_share.cuh).  Beginning and ending a
// unit costs as much as several tiles (its queries are split, two accumulators joined, and the pipeline runs dry), so every
// unit's tiles are preceded in that list by HEAD places with no work in them.
//
//   S = Q K^T   on the codes as the cache holds them.  Q is split into two e4m3 terms per row, q = 2^x (q1 + q2): a bf16 value
//               has 8 significant bits, e4m3 has 4, so the two terms are exact except for elements below 2^-9 of their row's
//               largest (absolute error at most 2^-17 of that).  Two e4m3 MMAs at twice the bf16 rate cost what one bf16 MMA would,
//               and K needs half the shared memory and no conversion.
//   O += P V    in fp16: four warps turn the codes of V into fp16 (exact) in shared memory.  The weights P need eleven bits and
//               a range that 8-bit terms only reach with three of them (built: splitting P cost the softmax twice the
//               instructions of the exponentials, V's conversion costs a quarter of that).
// A page's K scale multiplies its 16 score columns, its V scale its 16 columns of P, both in the softmax.  The bf16 tile has
// the same form, K as two e4m3 terms and V as fp16, but a power of two for every token in the place of the scales: not every row
// sees every token, and what a row does not see must not take its bits.
//
// Exponentials are taken against a reference per row, chosen in the first tile and raised only when a tile outgrows 2^15: O and l
// are then rescaled in place.  The weights of O, which hold a V scale, have one of their own: m_ref is the row's largest score, and
// v_ref the power of two above the largest product of a weight and its V scale, both held as 2^11.  (With the largest V scale
// as v_ref, a page of large values that weighs next to nothing would take the others' bits.)
//
// Two groups of four softmax warps take alternate tiles of a segment, each with an accumulator, a sum and a reference of
// its own, so that neither waits for the other; they meet at the segment's end.  Warp roles: 0 loader of Q and K, 1 issuer of
// S and 3 its gate, 2 issuer of O, 4..7 and 8..11 softmax (and, as a segment begins, its queries' terms), 12..15 V and the
// bf16 tile.
// All waits are bounded: one that runs out raises the block's abort flag and the cache's status word, and every role leaves.
//
// What bounds it: not a unit but the way of a tile through the roles (16 ragged sequences of 2048 to 16384 tokens, 32 query
// and 4 KV heads, 32 rows: 113 us in a graph of twenty calls, 119 to 122 in a long row of calls; 0.9 us a tile and block, where
// its MMAs take 0.45, its exponentials 0.27 and its bytes 0.2).  Taking away half of any one role's work changes the time by
// 5 % at most; the four score buffers that tensor memory has room for are what is in flight.  32 rows over 4096 tokens, 8 KV
// heads: 22.5 us (23 in a row of calls), 27000 cycles of them in a block: 9000 until the queries are there, 4500 on their terms,
// 7500 on four tiles, 6000 on joining.

#include <cfloat>
#include <cuda_fp16.h>

#include "attn_quant.cuh"
#include "attn_share.cuh"
#include "sm100.cuh"

namespace attnq {
namespace umma {

using namespace sm100;
using attn::AttnParams;
using attn::MAX_SEGS;
using attn::Seg;

constexpr int HD = 128;
constexpr int TILE = 64;                       // keys per tile
constexpr int PAGES = TILE / PAGE;
constexpr int T_BYTES = TILE * HD;             // one 8-bit operand tile, 8 KB
constexpr int NK = 5;                          // ring slots of K tiles
constexpr int VR_BYTES = 2 * PAGE * HD;        // a converting warp's two pages of a tile, as codes; two of them per warp
constexpr int NVH = 3;                         // tiles of V in fp16
constexpr int NSCALE = 16;                      // page tiles whose scales are kept: the loader of K is at most NK tiles ahead of the
                                               // issuer of S, and that one NS ahead of O, so none is overwritten too early
constexpr int VH_BYTES = 2 * T_BYTES;          // V of a tile in fp16: [dim half][64 tokens][128 B]
constexpr int VH_HALF = T_BYTES;
constexpr int Q_BYTES = 2 * 128 * HD;          // both terms, 32 KB; two of them: the next segment's queries are split early
constexpr int BT_BYTES = 2 * T_BYTES + VH_BYTES;   // bf16 tile: K terms, V in fp16
constexpr int THREADS = 512;
constexpr int TMEM_COLS = 512;                 // S, and P in its place (columns 0..31 of it): [b * 64, +64) b < 4;  O [256 + g * 128, +128)
constexpr int NS = 4;                          // a tile's buffer is free once O has taken P from it
constexpr int O_COL = 256;
constexpr int HEAD = 12;                        // what a unit costs beside its tiles, in tiles
constexpr float BIAS = 11.f;                   // the reference weight is 2^11: 2^4 below the raise, 2^35 above fp16's last bit

// mbarrier indices
constexpr int BAR_Q_FULL = 0;                  // [2]  count 8: the softmax warps
constexpr int BAR_Q_EMPTY = 2;                 // [2]  count 9: the issuer of S, the softmax warps (they have read the factors)
constexpr int BAR_BT_FULL = 4;                 // count 4: the warps that convert
constexpr int BAR_BT_EMPTY = 5;                // the issuer of O
constexpr int BAR_S_FULL = 6;                  // [NS]  count 2: the issuer's MMAs, and the gate, who has seen the tile's scales arrive
constexpr int BAR_S_FREE = BAR_S_FULL + NS;    // [NS]  the issuer of O
constexpr int BAR_P_READY = BAR_S_FREE + NS;   // [NS]  count 4: the warps of the group that has the tile
constexpr int BAR_O_DONE = BAR_P_READY + NS;   // [2]   per group
constexpr int BAR_MEET = BAR_O_DONE + 2;       // [4]  count 2: the two warps of a lane quarter
constexpr int BAR_PART = BAR_MEET + 4;         // [4]  count 2
constexpr int BAR_K_FULL = BAR_PART + 4;       // [NK]
constexpr int BAR_K_EMPTY = BAR_K_FULL + NK;   // [NK]  the issuer of S
constexpr int BAR_VH_FULL = BAR_K_EMPTY + NK;  // [NVH]  count 2: the two warps that convert the tile
constexpr int BAR_VH_EMPTY = BAR_VH_FULL + NVH;      // [NVH]  the issuer of O
constexpr int BAR_Q_RAW = BAR_VH_EMPTY + NVH;    // [2]  the queries as bf16
constexpr int BAR_GO = BAR_Q_RAW + 2;          // [NS]  the gate: everything that S of a tile needs is there
constexpr int BAR_SEG = BAR_GO + NS;           // the issuer of O: a segment's products are all in O
constexpr int N_BARS = BAR_SEG + 1;

struct Shared {                                // behind the operand buffers
    uint64_t bars[N_BARS];
    float q_factor[2][128];                    // per query row: scale * log2(e) * the power of two taken out of it
    float bt_k[TILE], bt_lv[TILE];             // powers of two taken out of the bf16 tile's tokens: of K, log2 of V's
    float scales[NSCALE][3 * PAGES];           // K scales, V scales of a page tile's pages, log2 of those
    float meet[2][3][128];                     // per group and row: reference, sum, V reference
    uint32_t tmem_slot;
    int abort_flag;
    int n_seg;
    int bt_bad[2];                             // bf16 tile number x has a NaN or an infinity among its values: [x & 1] == x + 1
    long long cursor;
    Seg segs[MAX_SEGS];
};
constexpr int SMEM_BYTES = 2 * Q_BYTES + NK * T_BYTES + 8 * VR_BYTES + NVH * VH_BYTES + BT_BYTES + 1024 + (int)sizeof(Shared);
static_assert(SMEM_BYTES <= 227 * 1024, "a block's shared memory");

struct QParams {
    AttnParams a;
    deer_kv_quant_desc kq;
};

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A wait that usually need not wait is one instruction here; the rest is out of line (instruction fetches are what this
// kernel has least of).
__device__ __noinline__ bool wait_slowly(uint32_t bar, uint32_t parity, volatile int* abort_flag) { return mbar_wait(bar, parity, abort_flag); }
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    return mbar_try_wait(bar, parity) || wait_slowly(bar, parity, abort_flag);
}

// A value that is the same in every lane, told to the compiler: what follows from it can live in uniform registers.
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

// Places in the list for sequence b: HEAD, its full pages four at a time, the bf16 tile; 0 if the sequence cannot be used.
__device__ __forceinline__ int seq_tiles(const AttnParams& p, int b, int* n_out, int* s_out) {
    const int s = p.seq_ids[b];
    int n = -1;
    if (s >= 0 && s < p.kv.max_seqs) n = p.kv.seq_len[s];
    if (n_out) *n_out = n;
    if (s_out) *s_out = s;
    if (n < 0 || n > p.max_seq_len) return 0;
    return HEAD + (n / PAGE + PAGES - 1) / PAGES + 1;
}

__device__ __forceinline__ float power_of_two(float e) { return __uint_as_float((uint32_t)((int)e + 127) << 23); }   // 2^e, -126 <= e <= 127
// log2 of the reference of the weights of O from that of the largest product of a weight and its V scale, both against m_ref.
__device__ __forceinline__ float log2_reference(float j) { return fminf(fmaxf(ceilf(j), -126.f), 126.f); }
// This thread's row of an accumulator times a factor.  (Out of line: two places need it, neither often.)
__device__ __noinline__ void scale_accumulator(uint32_t taddr, float by) {
#pragma unroll 1
    for (int cc = 0; cc < HD / 16; ++cc) {
        uint32_t o[16];
        TMEM_LD_X16(taddr + (uint32_t)(cc * 16), o);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * by);
        TMEM_ST_X16(taddr + (uint32_t)(cc * 16), o);
    }
    tmem_wait_st();
}

// Power of two that brings a group's largest magnitude to [128, 256) (nothing but zeros: 1).
__device__ __forceinline__ float to_256(uint32_t amax_bits) {
    const int f = amax_bits ? 127 + 7 + 127 - (int)(amax_bits >> 23) : 127;
    return __uint_as_float((uint32_t)min(max(f, 1), 254) << 23);
}
// Sixteen bf16 values times `up`, as two terms of e4m3 codes: the leading four significant bits, cut off, and the four
// behind them.  Below e4m3's normal range (2^-6) the second term takes the value as a whole.
__device__ __forceinline__ void split16(const float (&v)[16], float up, bool bad, uint4* t1, uint4* t2) {
    uint32_t a[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t lo[2], hi[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x[2], y[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                x[e] = v[j * 4 + h * 2 + e] * up;
                y[e] = fabsf(x[e]) < 0.015625f ? 0.f : __uint_as_float(__float_as_uint(x[e]) & 0xfff00000u);
            }
            lo[h] = __nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3);
            hi[h] = __nv_cvt_float2_to_fp8x2(make_float2(x[0] - y[0], x[1] - y[1]), __NV_SATFINITE, __NV_E4M3);
        }
        a[j] = bad ? 0x7f7f7f7fu : (lo[0] | (lo[1] << 16));
        b[j] = bad ? 0u : (hi[0] | (hi[1] << 16));
    }
    *t1 = make_uint4(a[0], a[1], a[2], a[3]);
    *t2 = make_uint4(b[0], b[1], b[2], b[3]);
}

// A 16-dim piece of a bf16 row that lies in two halves of 64 dims (128-byte rows, swizzled), `half` bytes apart.
__device__ __forceinline__ const uint4* piece(const unsigned char* tile, int half, int r, int c16, int x) {
    return reinterpret_cast<const uint4*>(tile + (c16 >> 2) * half + r * 128 + ((((c16 & 3) * 2 + x) ^ (r & 7)) << 4));
}
// The query rows first, first + step, ... (four rows per warp at a time, eight lanes each) of a tile that TMA has brought as
// bf16 [dim half][128 rows][128 B], in place as two terms [term][128 rows][128 B], and the factor that turns their products
// into scores in the log2 domain.  A row's raw form and its terms are the same 256 bytes.  Whole-warp call; the caller
// makes the writes visible.
__device__ __forceinline__ void split_queries(unsigned char* tile, float* factor, float scale_log2, int rows, int first, int step) {
    const int c16 = threadIdx.x & 7;                               // 16-dim piece of a row
#pragma unroll 1
    for (int r = first; r < 128; r += step) {
        float v[16];
        uint4 a = *piece(tile, Q_BYTES / 2, r, c16, 0), b = *piece(tile, Q_BYTES / 2, r, c16, 1);
        if (r >= rows) a = b = make_uint4(0, 0, 0, 0);             // whatever was there
        quant::unpack_bf16x8(a, v);
        quant::unpack_bf16x8(b, v + 8);
        const uint32_t m = quant::max8(quant::amax16(v));          // (every lane of the row has read its piece)
        const float up = to_256(m);
        uint4 t1, t2;
        split16(v, up, m >= 0x7f800000u, &t1, &t2);
        unsigned char* dst = tile + r * HD + ((c16 ^ (r & 7)) << 4);
        *reinterpret_cast<uint4*>(dst) = t1;
        *reinterpret_cast<uint4*>(dst + Q_BYTES / 2) = t2;
        if (c16 == 0) factor[r] = scale_log2 / up;
    }
}

// Sixteen tokens (tok0 ..) of the bf16 tile's K in place as two terms, with a power of two for each; a token with a NaN or an
// infinity gets NaN codes.  Whole-warp call, for rows that this warp's lanes have brought, each its pieces.
__device__ __forceinline__ void split_keys(unsigned char* tile, float* scale, int tok0) {
    const int lane = threadIdx.x & 31, c16 = lane & 7;
#pragma unroll 1
    for (int x = 0; x < 4; ++x) {
        const int tok = tok0 + x * 4 + (lane >> 3);
        float v[16];
        quant::unpack_bf16x8(*piece(tile, T_BYTES, tok, c16, 0), v);
        quant::unpack_bf16x8(*piece(tile, T_BYTES, tok, c16, 1), v + 8);
        const uint32_t m = quant::max8(quant::amax16(v));          // (every lane of the row has read)
        const bool bad = m >= 0x7f800000u;
        const float up = bad ? 1.f : to_256(m);
        uint4 t1, t2;
        split16(v, up, bad, &t1, &t2);
        unsigned char* dst = tile + tok * HD + ((c16 ^ (tok & 7)) << 4);
        *reinterpret_cast<uint4*>(dst) = t1;
        *reinterpret_cast<uint4*>(dst + T_BYTES) = t2;
        if (c16 == 0) scale[tok] = 1.f / up;
    }
}
// The same for V, in place as fp16 (exact down to 2^-21 of the token's largest, 2^-32 of it absolutely), and log2 of the power of
// two (-infinity for nothing but zeros: no say in the reference of the weights).  NaN and infinities become zeros -- they join the
// rows that see them at the segment's end -- and the call returns true.
__device__ __forceinline__ bool values_to_f16(unsigned char* tile, float* log2_scale, int tok0) {
    const int lane = threadIdx.x & 31, c16 = lane & 7, c8 = (c16 & 3) * 2;
    uint32_t any = 0;
#pragma unroll 1
    for (int x = 0; x < 4; ++x) {
        const int tok = tok0 + x * 4 + (lane >> 3);
        float v[16];
        quant::unpack_bf16x8(*piece(tile, VH_HALF, tok, c16, 0), v);
        quant::unpack_bf16x8(*piece(tile, VH_HALF, tok, c16, 1), v + 8);
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t mag = quant::mag_bits(v[e]);
            any = max(any, mag);
            if (mag >= 0x7f800000u) v[e] = 0.f;
            else m = max(m, mag);
        }
        m = quant::max8(m);
        const float up = to_256(m);
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const __half2 hv = __floats2half2_rn(v[2 * e] * up, v[2 * e + 1] * up);
            w[e] = *reinterpret_cast<const uint32_t*>(&hv);
        }
        unsigned char* dst = tile + (c16 >> 2) * VH_HALF + tok * 128;
        *reinterpret_cast<uint4*>(dst + ((c8 ^ (tok & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(dst + (((c8 + 1) ^ (tok & 7)) << 4)) = make_uint4(w[4], w[5], w[6], w[7]);
        if (c16 == 0) log2_scale[tok] = m != 0 ? 127.f - (float)(__float_as_uint(up) >> 23) : -INFINITY;
    }
    return __any_sync(0xffffffffu, any >= 0x7f800000u);
}

// Columns of the bf16 tile (tail rows, then block rows) that a query row of block row i_blk sees.
__device__ __forceinline__ uint64_t columns_seen(const AttnParams& p, const Seg& g, int i_blk, bool row_valid, uint32_t present, uint32_t decoded) {
    const int n_tail = g.n % PAGE, state = (p.row_state && row_valid) ? p.row_state[(size_t)g.b * p.k + i_blk] : 1;
    return ((uint64_t)(attn::visible_rows(p.mask, i_blk, state, present, decoded) & present) << n_tail) | ((1ull << n_tail) - 1ull);
}

__global__ void __launch_bounds__(THREADS, 1)
attn_quant_umma_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const QParams qp) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char* sQ = smem;                                  // [2 buffers][2 terms][128 rows][128 B]
    unsigned char* ring = sQ + 2 * Q_BYTES;                    // [NK][64 tokens][128 B]
    unsigned char* vraw = ring + NK * T_BYTES;                 // [4 warps][2][2 pages][16 tokens][128 B]
    unsigned char* vh = vraw + 8 * VR_BYTES;                   // [NVH]
    unsigned char* bt = vh + NVH * VH_BYTES;                     // [K term 1, K term 2][64][128 B], V
    Shared& sh = *reinterpret_cast<Shared*>(bt + BT_BYTES);
    volatile int* abort_flag = &sh.abort_flag;
    const AttnParams& p = qp.a;

    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
    const int Hkv = p.kv.n_kv_heads;
    const int HR = Hkv * p.row_tiles;
    const int j = blockIdx.x;
    const int jg = j / p.row_tiles, rt = j % p.row_tiles;      // group of blocks that walk the same share; my row tile
    const int ncg = p.nc / p.row_tiles;

    const uint32_t bar_base = smem_u32(sh.bars);
    auto bar = [&](int idx) { return bar_base + 8u * idx; };
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(BAR_Q_FULL + i), 8);
            mbar_init(bar(BAR_Q_RAW + i), 1);
            mbar_init(bar(BAR_Q_EMPTY + i), 9);
            mbar_init(bar(BAR_O_DONE + i), 1);
        }
        for (int i = 0; i < NS; ++i) {
            mbar_init(bar(BAR_S_FULL + i), 2);
            mbar_init(bar(BAR_S_FREE + i), 1);
            mbar_init(bar(BAR_P_READY + i), 4);
            mbar_init(bar(BAR_GO + i), 1);
        }
        mbar_init(bar(BAR_BT_FULL), 4);
        mbar_init(bar(BAR_BT_EMPTY), 1);
        mbar_init(bar(BAR_SEG), 1);
        for (int i = 0; i < 4; ++i) {
            mbar_init(bar(BAR_MEET + i), 2);
            mbar_init(bar(BAR_PART + i), 2);
        }
        for (int i = 0; i < NVH; ++i) {
            mbar_init(bar(BAR_VH_FULL + i), 2);
            mbar_init(bar(BAR_VH_EMPTY + i), 1);
        }
        for (int i = 0; i < NK; ++i) {
            mbar_init(bar(BAR_K_FULL + i), 1);
            mbar_init(bar(BAR_K_EMPTY + i), 1);
        }
        sh.abort_flag = 0;
        sh.bt_bad[0] = sh.bt_bad[1] = 0;
        mbar_init_fence();
        prefetch_tensormap(&tm_q);
        prefetch_tensormap(&tm_k);
    }
    pdl_trigger();
    pdl_wait();

    // ---- this block's share of the flattened tile list ----
    long long T = 0;
    int my_n = -1, my_s = -1, my_tiles = 0;                    // of sequence `lane`: the list of segments asks for them again
    for (int b = lane; b < p.B; b += 32) {
        int n, s;
        const int tiles = seq_tiles(p, b, &n, &s);
        if (b == lane) {
            my_n = n;
            my_s = s;
            my_tiles = tiles;
        }
        T += tiles;
        // a sequence that cannot be used has no tiles, so no block need ever list it: its units' merge entries and the report are written here
        if (tiles == 0 && j == 0 && warp == 0) {
            deer_report(p.kv.status, DEER_ERR_INVALID_ARG);
            for (int hr = 0; hr < HR; ++hr) p.unit_parts[(size_t)b * HR + hr] = make_int2(-1, -1);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) T += __shfl_xor_sync(0xffffffffu, T, o);
    T *= Hkv;
    const long long share_lo = attn::share_begin(T, jg, ncg), share_hi = attn::share_begin(T, jg + 1, ncg);
    if (j == 0 && tid == 0) *p.total_tiles = T;
    if (share_hi <= share_lo) return;

    if (warp == 1) tmem_alloc(smem_u32(&sh.tmem_slot), TMEM_COLS);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem_base = sh.tmem_slot;
    const uint32_t q_addr = smem_u32(sQ), ring_addr = smem_u32(ring), vh_addr = smem_u32(vh), bt_addr = smem_u32(bt);

    // Counters that run across segments and rounds; every role advances its own copy identically.
    int it = 0;          // tiles so far: group it & 1, that group's phase it >> 1; S buffer it % NS, its phase it / NS
    int rs = 0;          // page tiles so far: ring slot rs % NK, fp16 buffer rs % NVH
    int nb = 0;          // bf16 tiles so far
    int sg = 0;          // segments so far: Q buffer sg & 1
    long long cursor = share_lo;
    while (cursor < share_hi) {
        if (warp == 0) {
            long long next;
            const int ns = attn::build_segments(p, Hkv, rt, cursor, share_hi, sh.segs, &next, lane,
                                                [&](int b, int* n, int* s) {
                                                    if (b != lane) return seq_tiles(p, b, n, s);
                                                    if (n) *n = my_n;
                                                    if (s) *s = my_s;
                                                    return my_tiles;
                                                });
            if (lane == 0) {                                               // from places to tiles
                int kept = 0;
                for (int x = 0; x < ns; ++x) {
                    Seg g = sh.segs[x];
                    if (g.t_b <= HEAD) continue;
                    g.t_a = max(g.t_a - HEAD, 0);
                    g.t_b -= HEAD;
                    sh.segs[kept++] = g;
                }
                sh.n_seg = kept;
                sh.cursor = next;
            }
        }
        __syncthreads();
        const int n_seg = sh.n_seg;
        cursor = sh.cursor;

        if (warp == 0) {
            // ---------------- loader of Q (TMA, as bf16) and K ----------------
            // (A page is a copy of its own, and a warp gets one out every ~200 cycles: it could not bring V as well.)
            const int no_row = p.kv.num_pages * Hkv * PAGE;    // beyond the pool: reads as zero
            bool ok = true;
            for (int si = 0; si < n_seg && ok; ++si, ++sg) {
                const Seg g = sh.segs[si];
                const int kvh = g.hr / p.row_tiles, full = g.n / PAGE;
                const int last_tile = (full + PAGES - 1) / PAGES;
                const int32_t* pt_row = p.kv.page_table + (size_t)g.s * p.kv.max_pages;
                {
                    const int qb = sg & 1;
                    int okq = 1;
                    if (lane == 0) okq = wait(bar(BAR_Q_EMPTY + qb), ((uint32_t)(sg >> 1) & 1u) ^ 1u, abort_flag) ? 1 : 0;
                    if (!__shfl_sync(0xffffffffu, okq, 0)) { ok = false; break; }
                    if (lane == 0) {
                        mbar_expect_tx(bar(BAR_Q_RAW + qb), (uint32_t)(2 * p.G * min(p.ipt, p.k) * 128));
                        tma_load_3d(q_addr + qb * Q_BYTES, &tm_q, 0, kvh * p.G, g.b * p.k + rt * p.ipt, bar(BAR_Q_RAW + qb));
                        tma_load_3d(q_addr + qb * Q_BYTES + Q_BYTES / 2, &tm_q, 64, kvh * p.G, g.b * p.k + rt * p.ipt, bar(BAR_Q_RAW + qb));
                    }
                    __syncwarp();
                }
                // Page ids and scales, eight tiles at a time: lane l holds page l of the eight tiles; the scales are fetched a batch
                // ahead, the ids they need two.  (Tile by tile their latencies, one behind the other, would set the pace.)
                auto ids_at = [&](int t0) -> int {
                    const int lp = t0 * PAGES + lane;
                    if (t0 + lane / PAGES >= g.t_b || lp >= full) return -2;       // nothing there
                    return lp < p.kv.max_pages ? pt_row[lp] : -1;
                };
                auto scale_of = [&](const float* scales, int pg) -> float {
                    return pg < 0 || pg >= p.kv.num_pages ? 0.f : __ldcg(scales + (size_t)pg * Hkv + kvh);
                };
                int id_cur = ids_at(g.t_a), id_next = ids_at(g.t_a + 8), id_third = ids_at(g.t_a + 16);
                float ks_cur = scale_of(qp.kq.k_scale, id_cur), vs_cur = scale_of(qp.kq.v_scale, id_cur);
                float ks_next = scale_of(qp.kq.k_scale, id_next), vs_next = scale_of(qp.kq.v_scale, id_next);
                const int t_end = min(g.t_b, last_tile);
                for (int t = g.t_a; t < t_end; ++t) {
                    const int sl = rs % NK, at = (t - g.t_a) & 7;
                    if (at == 0 && t != g.t_a) {
                        id_cur = id_next;
                        ks_cur = ks_next;
                        vs_cur = vs_next;
                        id_next = id_third;
                        ks_next = scale_of(qp.kq.k_scale, id_next);
                        vs_next = scale_of(qp.kq.v_scale, id_next);
                        id_third = ids_at(t + 16);
                    }
                    float ks = __shfl_sync(0xffffffffu, ks_cur, at * PAGES + (lane & 3));
                    const float vs = __shfl_sync(0xffffffffu, vs_cur, at * PAGES + (lane & 3));
                    if (!(fabsf(vs) < INFINITY)) ks = NAN;             // makes every row that sees the page NaN, as vs would
                    int oks = 1;
                    if (lane == 0) oks = wait(bar(BAR_K_EMPTY + sl), ((uint32_t)(rs / NK) & 1u) ^ 1u, abort_flag) ? 1 : 0;
                    if (!__shfl_sync(0xffffffffu, oks, 0)) { ok = false; break; }
                    if (lane < 3 * PAGES) sh.scales[rs % NSCALE][lane] = lane < PAGES ? ks : lane < 2 * PAGES ? vs : __log2f(vs);
                    __syncwarp();
                    if (lane == 0) mbar_expect_tx(bar(BAR_K_FULL + sl), T_BYTES);      // (the arrival publishes the scales as well)
                    __syncwarp();
                    const int pg = __shfl_sync(0xffffffffu, id_cur, at * PAGES + (lane & 3));
                    if (lane < 4) {
                        const bool there = pg >= 0 && pg < p.kv.num_pages;
                        if (!there && pg != -2) deer_report(p.kv.status, DEER_ERR_BAD_PAGE);
                        tma_load_2d(ring_addr + sl * T_BYTES + lane * PAGE * HD, &tm_k, 0, there ? (pg * Hkv + kvh) * PAGE : no_row, bar(BAR_K_FULL + sl));
                    }
                    ++rs;
                }
            }
        } else if (warp == 3) {
            // ---------------- gate of S: does the issuer's waiting (a wait takes 100 cycles and more even when it need not wait) ----------------
            if (lane == 0) {
                bool ok = true;
                for (int si = 0; si < n_seg && ok; ++si, ++sg) {
                    const Seg g = sh.segs[si];
                    const int last_tile = (g.n / PAGE + PAGES - 1) / PAGES;
                    if (!wait(bar(BAR_Q_FULL + (sg & 1)), (uint32_t)(sg >> 1) & 1u, abort_flag)) { ok = false; break; }
                    for (int t = g.t_a; t < g.t_b; ++t, ++it) {
                        const int sb = it % NS;
                        const bool blk = t == last_tile;
                        if (!wait(blk ? bar(BAR_BT_FULL) : bar(BAR_K_FULL + rs % NK), (uint32_t)(blk ? nb : rs / NK) & 1u, abort_flag) ||
                            !wait(bar(BAR_S_FREE + sb), ((uint32_t)(it / NS) & 1u) ^ 1u, abort_flag)) {
                            ok = false;
                            break;
                        }
                        mbar_arrive(bar(BAR_GO + sb));
                        mbar_arrive(bar(BAR_S_FULL + sb));
                        if (blk) ++nb;
                        else ++rs;
                    }
                }
            }
        } else if (warp == 1) {
            // ---------------- issuer of S ----------------
            const uint32_t idesc = make_idesc_e4m3(TILE);
            const bool leader = elect_one();
            bool ok = true;
            for (int si = 0; si < n_seg && ok; ++si, ++sg) {
                const int last_tile = uniform((sh.segs[si].n / PAGE + PAGES - 1) / PAGES), t_a = uniform(sh.segs[si].t_a), t_b = uniform(sh.segs[si].t_b);
                const int qb = sg & 1;
                const uint64_t qd = smem_desc_sw128_kmajor(q_addr + qb * Q_BYTES);
                for (int t = t_a; t < t_b; ++t, ++it) {
                    const int sb = it % NS;
                    const uint32_t d_tmem = tmem_base + (uint32_t)(sb * TILE);
                    ok = __all_sync(0xffffffffu, wait(bar(BAR_GO + sb), (uint32_t)(it / NS) & 1u, abort_flag));
                    if (!ok) break;
                    tcgen05_fence_after();
                    if (t != last_tile) {
                        const int sl = rs % NK;
                        const uint64_t kd = smem_desc_sw128_kmajor(ring_addr + sl * T_BYTES);
                        if (leader) {
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)                 // four steps of 32 dims for each term of Q
                                umma_f8_ss(d_tmem, qd + (uint64_t)(((kk >> 2) * (Q_BYTES / 2) + (kk & 3) * 32) >> 4), kd + (uint64_t)((kk & 3) * 2),
                                           idesc, kk != 0 ? 1u : 0u);
                            umma_commit(bar(BAR_S_FULL + sb));
                            umma_commit(bar(BAR_K_EMPTY + sl));
                        }
                        ++rs;
                    } else {
                        const uint64_t kd = smem_desc_sw128_kmajor(bt_addr);
                        if (leader) {
#pragma unroll
                            for (int kk = 0; kk < 16; ++kk)                // and for each term of K
                                umma_f8_ss(d_tmem, qd + (uint64_t)((((kk >> 2) & 1) * (Q_BYTES / 2) + (kk & 3) * 32) >> 4),
                                           kd + (uint64_t)(((kk >> 3) * T_BYTES + (kk & 3) * 32) >> 4), idesc, kk != 0 ? 1u : 0u);
                            umma_commit(bar(BAR_S_FULL + sb));
                        }
                    }
                    __syncwarp();
                }
                if (ok && leader) umma_commit(bar(BAR_Q_EMPTY + qb));
                __syncwarp();
            }
        } else if (warp == 2) {
            // ---------------- issuer of O += P V, both groups ----------------
            const uint32_t idesc = make_idesc_f16(HD, 1);
            const bool leader = elect_one();
            bool ok = true;
            for (int si = 0; si < n_seg && ok; ++si) {
                const int last_tile = uniform((sh.segs[si].n / PAGE + PAGES - 1) / PAGES), t_a = uniform(sh.segs[si].t_a), t_b = uniform(sh.segs[si].t_b);
                for (int t = t_a; t < t_b; ++t, ++it) {
                    const int grp = it & 1;
                    const int sb = it % NS;
                    const uint32_t o_tmem = tmem_base + (uint32_t)(O_COL + grp * HD), p_tmem = tmem_base + (uint32_t)(sb * TILE);
                    const uint32_t keep = t - t_a < 2 ? 0u : 1u;           // the group's first tile of the segment starts a new sum
                    const bool blk = t == last_tile;
                    const int vb = rs % NVH;
                    ok = (blk || wait(bar(BAR_VH_FULL + vb), (uint32_t)(rs / NVH) & 1u, abort_flag)) &&
                         wait(bar(BAR_P_READY + sb), (uint32_t)(it / NS) & 1u, abort_flag);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tcgen05_fence_after();                                 // (a bf16 tile was full before its S)
                    // 16 tokens per MMA: two groups of eight, 1 KB apart; the dim halves 8 KB apart
                    const uint64_t vd = smem_desc_sw128(blk ? bt_addr + 2 * T_BYTES : vh_addr + vb * VH_BYTES, VH_HALF, 1024);
                    if (leader) {
#pragma unroll
                        for (int kk = 0; kk < TILE / 16; ++kk)
                            umma_bf16_ts(o_tmem, p_tmem + (uint32_t)(kk * 8), vd + (uint64_t)((kk * 2048) >> 4), idesc, kk != 0 ? 1u : keep);
                        umma_commit(bar(BAR_S_FREE + sb));
                        umma_commit(bar(BAR_O_DONE + grp));
                        umma_commit(blk ? bar(BAR_BT_EMPTY) : bar(BAR_VH_EMPTY + vb));
                    }
                    __syncwarp();
                    if (!blk) ++rs;
                }
                if (ok && leader) umma_commit(bar(BAR_SEG));
                __syncwarp();
            }
        } else if (warp >= 12) {
            // ---------------- V to fp16, and the bf16 tile ----------------
            // Warps 12, 13 take the even page tiles, 14, 15 the odd ones, two pages each: codes to a buffer of the warp's own (each
            // lane copies what it will convert; two tiles of its own ahead within a segment), from there as fp16 to the operand tile.
            const int w = warp - 12, c16 = lane & 7, c8 = (c16 & 3) * 2, mine = w >> 1, pair = (w & 1) * 2;
            unsigned char* my_raw = vraw + w * 2 * VR_BYTES;
            bool ok = true;
            for (int si = 0; si < n_seg && ok; ++si) {
                const Seg g = sh.segs[si];
                const int kvh = g.hr / p.row_tiles, full = g.n / PAGE, last_tile = (full + PAGES - 1) / PAGES;
                const int32_t* pt_row = p.kv.page_table + (size_t)g.s * p.kv.max_pages;
                const int t_end = min(g.t_b, last_tile), t_first = g.t_a + ((rs ^ mine) & 1);       // this warp's first tile of the segment
                auto ids_at = [&](int t0) -> int {                         // lane l: page `pair` + (l & 1) of tile t0 + (l & ~1)
                    const int t = t0 + (lane & ~1), lp = t * PAGES + pair + (lane & 1);
                    return t < t_end && lp < full && lp < p.kv.max_pages ? pt_row[lp] : -1;
                };
                int id_cur = ids_at(t_first), id_next = ids_at(t_first + 32), t_next = t_first;
                auto fetch = [&](int buf) {                                // this warp's next tile to its buffer; zeros for a page that is not there
                    const int at = (t_next - t_first) & 31;
                    if (at == 0 && t_next != t_first) {
                        id_cur = id_next;
                        id_next = ids_at(t_next + 32);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int pg = __shfl_sync(0xffffffffu, id_cur, at + h);
                        const bool there = pg >= 0 && pg < p.kv.num_pages;
                        const unsigned char* src = static_cast<const unsigned char*>(p.kv.v_pool) + ((size_t)(there ? pg : 0) * Hkv + kvh) * PAGE * HD + lane * 16;
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            cp_async16(smem_u32(my_raw + buf * VR_BYTES) + (uint32_t)(h * PAGE * HD + y * 512 + lane * 16), src + y * 512, there ? 16 : 0);
                    }
                    cp_async_commit();
                    t_next += 2;
                };
                int buf = 0;
                cp_async_wait<0>();                                        // (copies that the last segment asked for beyond its end)
                fetch(0);
                fetch(1);
                for (int t = g.t_a; t < g.t_b; ++t) {
                    if (t == (g.t_a + 2 < last_tile ? g.t_a + 2 : last_tile) && g.t_b == last_tile + 1) {
                        // The bf16 tile, as early as its buffer allows (two page tiles are on their way to O meanwhile): warp w
                        // takes 16 tokens of K, then of V.
                        const int n_tail = g.n % PAGE;
                        ok = wait(bar(BAR_BT_EMPTY), ((uint32_t)nb & 1u) ^ 1u, abort_flag);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        uint32_t present, decoded;
                        attn::row_state_sets(p.row_state, g.b, p.k, lane, &present, &decoded);
                        const size_t tail0 = (((size_t)g.s * Hkv + kvh) * DEER_TAIL_ROWS + (g.n / PAGE % 3) * PAGE) * HD;
                        const size_t blk0 = ((size_t)g.b * p.k * Hkv + kvh) * HD;
                        // rows as bf16 to where their split form will be, [dim half][64 tokens][128 B], zeros where there is no
                        // token; each lane copies what it will split
#pragma unroll 1
                        for (int x = 0; x < 8; ++x) {
                            const bool is_v = x >= 4;
                            const int tok = w * PAGE + (x & 3) * 4 + (lane >> 3), jb = tok - n_tail;
                            const __nv_bfloat16* src = nullptr;
                            if (tok < n_tail)
                                src = static_cast<const __nv_bfloat16*>(is_v ? qp.kq.v_tail : qp.kq.k_tail) + tail0 + (size_t)(tok * HD + c16 * 16);
                            else if (jb < p.k && ((present >> jb) & 1u))
                                src = (is_v ? p.v_blk : p.k_blk) + blk0 + (size_t)jb * Hkv * HD + c16 * 16;
                            unsigned char* tile = bt + (is_v ? 2 * T_BYTES : 0);
                            cp_async16(smem_u32(piece(tile, T_BYTES, tok, c16, 0)), src ? src : p.k_blk, src ? 16 : 0);
                            cp_async16(smem_u32(piece(tile, T_BYTES, tok, c16, 1)), src ? src + 8 : p.k_blk, src ? 16 : 0);
                        }
                        cp_async_commit();
                        cp_async_wait<0>();                                // (and whatever V is on its way)
                        __syncwarp();
                        split_keys(bt, sh.bt_k, w * PAGE);
                        if (values_to_f16(bt + 2 * T_BYTES, sh.bt_lv, w * PAGE) && lane == 0) *(volatile int*)&sh.bt_bad[nb & 1] = nb + 1;
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(BAR_BT_FULL));
                        ++nb;
                    }
                    if (t == last_tile) break;
                    if ((rs & 1) == mine) {
                        const int vb = rs % NVH;
                        ok = wait(bar(BAR_VH_EMPTY + vb), ((uint32_t)(rs / NVH) & 1u) ^ 1u, abort_flag);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        cp_async_wait<1>();
                        unsigned char* dst = vh + vb * VH_BYTES + (c16 >> 2) * VH_HALF;
                        const uint4* src = reinterpret_cast<const uint4*>(my_raw + buf * VR_BYTES) + lane;
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            const int tok = (pair + (x >> 2)) * PAGE + (x & 3) * 4 + (lane >> 3);
                            const uint4 codes = src[x * 32];
                            const uint32_t cw[4] = {codes.x, codes.y, codes.z, codes.w};
                            uint32_t f[8];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                f[2 * e] = codes_lo(cw[e]);
                                f[2 * e + 1] = codes_hi(cw[e]);
                            }
                            *reinterpret_cast<uint4*>(dst + tok * 128 + ((c8 ^ (tok & 7)) << 4)) = make_uint4(f[0], f[1], f[2], f[3]);
                            *reinterpret_cast<uint4*>(dst + tok * 128 + (((c8 + 1) ^ (tok & 7)) << 4)) = make_uint4(f[4], f[5], f[6], f[7]);
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(BAR_VH_FULL + vb));
                        fetch(buf);
                        buf ^= 1;
                    }
                    ++rs;
                }
            }
        } else if (warp >= 4) {
            // ---------------- softmax: one query row per thread, the group's tiles ----------------
            const int grp = (warp - 4) >> 2, quarter = warp & 3;
            const int row = quarter * 32 + lane;
            const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16);
            const int i_blk = rt * p.ipt + row / p.G, g_row = row % p.G, rows = min(p.ipt, p.k - rt * p.ipt) * p.G;      // this row's block row and head
            const bool row_valid = row < rows;
            bool alive = true;
            for (int si = 0; si < n_seg && alive; ++si, ++sg) {
                const Seg& g = sh.segs[si];
                const int full = g.n / PAGE, last_tile = (full + PAGES - 1) / PAGES, t_b = g.t_b;
                float m_ref = 0.f, lv_ref = 0.f, i_ref = 1.f, l_run = 0.f;      // lv_ref: log2 of v_ref, i_ref: 1 / v_ref
                bool first = true;
                const int qb = sg & 1;
                {
                    const bool raw = wait(bar(BAR_Q_RAW + qb), (uint32_t)(sg >> 1) & 1u, abort_flag);
                    if (!__all_sync(0xffffffffu, raw)) { alive = false; break; }
                    split_queries(sQ + qb * Q_BYTES, sh.q_factor[qb], p.scale_log2, rows, (warp - 4) * 4 + (lane >> 3), 32);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(BAR_Q_FULL + qb));
                }
                {
                    const bool got = wait(bar(BAR_Q_FULL + qb), (uint32_t)(sg >> 1) & 1u, abort_flag);
                    if (!__all_sync(0xffffffffu, got)) { alive = false; break; }
                }
                const float f_row = sh.q_factor[qb][row];
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(BAR_Q_EMPTY + qb));         // (a short segment's MMAs may all be done before this point)
                for (int t = g.t_a; t < t_b; ++t, ++it) {
                    const bool is_bt = t == last_tile;
                    const int sb = it % NS;
                    const float* kv_scale = sh.scales[rs % NSCALE];        // (of a page tile)
                    if (!is_bt) ++rs;
                    if ((it & 1) != grp) continue;
                    const int n_pages = min(PAGES, full - t * PAGES);
                    const uint32_t s_tmem = t_lane + (uint32_t)(sb * TILE);
                    // The scores, and with them the scales.  (Not K_FULL or BT_FULL for those: a slot may be on its next tile but one
                    // by now, and a parity wait cannot tell.)
                    const bool got = wait(bar(BAR_S_FULL + sb), (uint32_t)(it / NS) & 1u, abort_flag);
                    if (!__all_sync(0xffffffffu, got)) { alive = false; break; }
                    tcgen05_fence_after();
                    // O times a factor.  Phase (it >> 1) - 1 of o_done: the group's previous tile is in O.  (The one before it is: its
                    // buffer is the one that this tile's scores are in.)
                    auto shrink = [&](float by) {
                        const bool od = wait(bar(BAR_O_DONE + grp), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag);
                        if (!__all_sync(0xffffffffu, od)) return false;
                        tcgen05_fence_after();
                        scale_accumulator(t_lane + (uint32_t)(O_COL + grp * HD), by);
                        return true;
                    };
                    if (is_bt) {
                        // Every column has factors of its own, and not every row sees it.  Whether a row's references have to rise is seen
                        // before its weights are made, for the row alone; P takes the scores' place sixteen columns at a time.
                        uint32_t present, decoded;
                        attn::row_state_sets(p.row_state, g.b, p.k, lane, &present, &decoded);
                        const uint64_t see = columns_seen(p, g, i_blk, row_valid, present, decoded);
                        auto load = [&](int q, float (&sc)[16]) {          // scores in the log2 domain
                            uint32_t r[16];
                            TMEM_LD_X16(s_tmem + (uint32_t)(q * 16), r);
                            tmem_wait_ld();
                            const uint32_t bits = (uint32_t)(see >> (q * 16));
#pragma unroll
                            for (int c = 0; c < 16; ++c) sc[c] = (bits >> c) & 1u ? __uint_as_float(r[c]) * (f_row * sh.bt_k[q * 16 + c]) : -INFINITY;
                        };
                        float m_t = -INFINITY, j_t = -INFINITY;            // largest score; largest score + log2 of its value's factor
#pragma unroll 1
                        for (int q = 0; q < TILE / 16; ++q) {
                            float sc[16];
                            load(q, sc);
#pragma unroll
                            for (int c = 0; c < 16; ++c) {
                                m_t = fmaxf(m_t, sc[c]);
                                j_t = fmaxf(j_t, sc[c] + sh.bt_lv[q * 16 + c]);
                            }
                        }
                        // (nothing visible, or not finite: the references stay)
                        const bool rise = fabsf(m_t) < INFINITY && (first || m_t > m_ref + 28.f || j_t > m_ref + lv_ref + 4.f);
                        if (!first) {
                            m_t = fmaxf(m_t, m_ref);
                            j_t = fmaxf(j_t, m_ref + lv_ref);
                        }
                        const float m_n = rise ? m_t : m_ref, lv_n = rise ? log2_reference(j_t - m_t) : lv_ref;
                        if (!first && __any_sync(0xffffffffu, rise)) {
                            l_run *= ex2_approx(m_ref - m_n);
                            if (!shrink(ex2_approx((m_ref - m_n) + (lv_ref - lv_n)))) { alive = false; break; }
                        }
                        m_ref = m_n;
                        lv_ref = lv_n;
                        first = false;
#pragma unroll 1
                        for (int q = 0; q < TILE / 16; ++q) {
                            float sc[16];
                            uint32_t w[8];
                            load(q, sc);
#pragma unroll
                            for (int c = 0; c < 16; c += 2) {
                                const float p0 = sc[c] + (BIAS - m_ref), p1 = sc[c + 1] + (BIAS - m_ref);
                                l_run += ex2_approx(p0) + ex2_approx(p1);
                                const __half2 hw = __floats2half2_rn(ex2_approx(p0 + (sh.bt_lv[q * 16 + c] - lv_ref)),
                                                                     ex2_approx(p1 + (sh.bt_lv[q * 16 + c + 1] - lv_ref)));
                                w[c >> 1] = *reinterpret_cast<const uint32_t*>(&hw);
                            }
                            TMEM_ST_X8(s_tmem + (uint32_t)(q * 8), w);
                        }
                        tmem_wait_st();
                        tcgen05_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(BAR_P_READY + sb));
                        continue;                                          // (the unit's last tile)
                    }
                    // 32 scores: column c of half h in the log2 domain = sr[c] * factor * its page's K scale
                    uint32_t sr[32];
                    auto load_half = [&](int h) {
                        TMEM_LD_X32(s_tmem + (uint32_t)(h * 32), sr);
                        tmem_wait_ld();
                    };
                    // The group's first tile sets the references.  Later a weight of 2^15 (0x7800 in fp16) or a sum of 2^40 raises
                    // them: O and l shrink in place, the tile is done again (P has not taken the scores' place yet).
                    bool set = first, stop = false;
                    float tile_sum;
                    uint32_t pr[TILE / 2];
#pragma unroll 1
                    for (int pass = 0; pass < 2; ++pass) {
                        if (set) {
                            float m_t = -INFINITY, j_t = -INFINITY;        // largest score; largest score + log2 of its V scale
#pragma unroll 1
                            for (int h = 0; h < 2; ++h) {
                                load_half(h);
#pragma unroll
                                for (int x = 0; x < 2; ++x) {
                                    if (h * 2 + x >= n_pages) break;
                                    float mx = -INFINITY;
#pragma unroll
                                    for (int c = 0; c < PAGE; ++c) mx = fmaxf(mx, __uint_as_float(sr[x * PAGE + c]));
                                    mx *= f_row * kv_scale[h * 2 + x];
                                    m_t = fmaxf(m_t, mx);
                                    j_t = fmaxf(j_t, mx + kv_scale[2 * PAGES + h * 2 + x]);
                                }
                            }
                            if (!(fabsf(m_t) < INFINITY)) {                // not finite
                                m_t = m_ref;
                                j_t = m_ref + lv_ref;
                            }
                            if (!first) {
                                m_t = fmaxf(m_t, m_ref);
                                j_t = fmaxf(j_t, m_ref + lv_ref);
                            }
                            const float lv_t = log2_reference(j_t - m_t);
                            if (!first) {
                                l_run *= ex2_approx(m_ref - m_t);
                                if (!shrink(ex2_approx((m_ref - m_t) + (lv_ref - lv_t)))) { stop = true; break; }
                            }
                            m_ref = m_t;
                            lv_ref = lv_t;
                            i_ref = power_of_two(-lv_ref);
                        }
                        // weights 2^(score - m_ref + 11), and in fp16 those times V scale / v_ref
                        uint64_t sum2[2] = {0, 0};
                        __half2 top2 = __float2half2_rn(0.f);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            load_half(h);
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const float nm = h * 2 + x < n_pages ? BIAS - m_ref : -INFINITY;
                                const float ka = f_row * kv_scale[h * 2 + x];
                                const float va = fminf(kv_scale[PAGES + h * 2 + x] * i_ref, FLT_MAX);      // (beyond that: masked, or next to nothing)
                                const uint64_t nm2 = pack_f32x2(nm, nm), ka2 = pack_f32x2(ka, ka), va2 = pack_f32x2(va, va);
#pragma unroll
                                for (int c = x * PAGE; c < (x + 1) * PAGE; c += 2) {
                                    float p0, p1, w0, w1;
                                    unpack_f32x2(fma2(pack_f32x2(__uint_as_float(sr[c]), __uint_as_float(sr[c + 1])), ka2, nm2), p0, p1);
                                    const uint64_t p2 = pack_f32x2(ex2_approx(p0), ex2_approx(p1));
                                    sum2[(c >> 1) & 1] = add2(sum2[(c >> 1) & 1], p2);
                                    unpack_f32x2(mul2(p2, va2), w0, w1);
                                    const __half2 hw = __floats2half2_rn(w0, w1);
                                    top2 = __hmax2(top2, hw);
                                    pr[h * 16 + (c >> 1)] = *reinterpret_cast<const uint32_t*>(&hw);
                                }
                            }
                        }
                        float a, b;
                        unpack_f32x2(add2(sum2[0], sum2[1]), a, b);
                        tile_sum = a + b;
                        const uint32_t tb = *reinterpret_cast<const uint32_t*>(&top2);
                        set = __any_sync(0xffffffffu, max(tb & 0x7fffu, (tb >> 16) & 0x7fffu) >= 0x7800u || !(tile_sum < 1.0995116e12f));
                        if (first || !set) break;
                    }
                    if (stop) { alive = false; break; }
                    first = false;
                    l_run += tile_sum;
                    TMEM_ST_X32(s_tmem, pr);
                    tmem_wait_st();
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(BAR_P_READY + sb));
                }
                if (!alive) break;
                if (t_b == last_tile + 1) ++nb;

                // ---- the segment's result: the groups meet; each takes half of the columns of both accumulators ----
                // (one phase per segment: the phases of o_done are not all waited for, so the last one could not be told)
                const bool done = wait(bar(BAR_SEG), (uint32_t)sg & 1u, abort_flag);
                if (!__all_sync(0xffffffffu, done)) { alive = false; break; }
                sh.meet[grp][0][row] = first ? -INFINITY : m_ref;
                sh.meet[grp][1][row] = first ? 0.f : l_run;
                sh.meet[grp][2][row] = power_of_two(lv_ref);
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(BAR_MEET + quarter));
                {
                    const bool got = wait(bar(BAR_MEET + quarter), (uint32_t)sg & 1u, abort_flag);
                    if (!__all_sync(0xffffffffu, got)) { alive = false; break; }
                }
                tcgen05_fence_after();
                const float m0 = sh.meet[0][0][row], m1 = sh.meet[1][0][row], l0 = sh.meet[0][1][row], l1 = sh.meet[1][1][row];
                const float mx = fmaxf(m0, m1);                            // one of the groups had a tile
                const float e0 = m0 == -INFINITY ? 0.f : ex2_approx(m0 - mx), e1 = m1 == -INFINITY ? 0.f : ex2_approx(m1 - mx);
                const float l = e0 * l0 + e1 * l1;
                const int kvh = g.hr / p.row_tiles, n_tail = g.n % PAGE;
                // no query row, or an absent one
                const bool gone = !row_valid || (p.row_state && p.row_state[(size_t)g.b * p.k + i_blk] < 0);
                const float inv = l != 0.f ? 1.f / l : 0.f;
                const float w0 = e0 * sh.meet[0][2][row] * inv, w1 = e1 * sh.meet[1][2][row] * inv;
                const bool has0 = m0 != -INFINITY, has1 = m1 != -INFINITY;
                const bool bad_v = g.t_b == last_tile + 1 && *(volatile int*)&sh.bt_bad[(nb - 1) & 1] == nb;
                const int hq = kvh * p.G + g_row;
                const size_t unit = (size_t)g.b * HR + g.hr;
                const bool whole = g.t_a == 0 && g.t_b == last_tile + 1;
                const size_t slot = ((size_t)g.b * Hkv + kvh + jg) * p.row_tiles + rt;
                uint64_t see = 0;
                if (bad_v) {                                               // (warp-uniform)
                    uint32_t present, decoded;
                    attn::row_state_sets(p.row_state, g.b, p.k, lane, &present, &decoded);
                    see = columns_seen(p, g, i_blk, row_valid, present, decoded);
                }
                __nv_bfloat16* out_row = row_valid && whole ? p.out + ((size_t)(g.b * p.k + i_blk) * p.Hq + hq) * HD + grp * 64 : nullptr;
                // partial results [four dims][row][4]: the lanes of a warp, who have a row each, write side by side
                float* part_row = row_valid && !whole ? p.part_o + slot * 128 * HD + (size_t)(grp * 16 * 128 + row) * 4 : nullptr;
#pragma unroll 1
                for (int cc = 0; cc < 4; ++cc) {
                    uint32_t a[16], b[16];
                    TMEM_LD_X16(t_lane + (uint32_t)(O_COL + grp * 64 + cc * 16), a);
                    TMEM_LD_X16(t_lane + (uint32_t)(O_COL + HD + grp * 64 + cc * 16), b);
                    tmem_wait_ld();
                    float v[16];
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        v[c] = has0 ? __uint_as_float(a[c]) * w0 : 0.f;
                        if (has1) v[c] = fmaf(__uint_as_float(b[c]), w1, v[c]);
                    }
                    if (bad_v) {                                           // what the bf16 tile's values could not carry
                        for (int x = 0; x < n_tail + p.k; ++x) {
                            if (!((see >> x) & 1u)) continue;
                            const __nv_bfloat16* src = x < n_tail
                                ? static_cast<const __nv_bfloat16*>(qp.kq.v_tail) + (((size_t)g.s * Hkv + kvh) * DEER_TAIL_ROWS + (full % 3) * PAGE + x) * HD
                                : p.v_blk + ((size_t)(g.b * p.k + x - n_tail) * Hkv + kvh) * HD;
                            src += grp * 64 + cc * 16;
#pragma unroll
                            for (int c = 0; c < 16; ++c) {
                                const float f = __bfloat162float(src[c]);
                                if (quant::mag_bits(f) >= 0x7f800000u) v[c] += f;
                            }
                        }
                    }
                    if (gone) {                                            // (zero times a NaN would be one)
#pragma unroll
                        for (int c = 0; c < 16; ++c) v[c] = 0.f;
                    }
                    if (out_row) {
#pragma unroll
                        for (int c = 0; c < 16; c += 8)
                            *reinterpret_cast<uint4*>(out_row + cc * 16 + c) = make_uint4(pack_bf16(v[c], v[c + 1]), pack_bf16(v[c + 2], v[c + 3]),
                                                                                          pack_bf16(v[c + 4], v[c + 5]), pack_bf16(v[c + 6], v[c + 7]));
                    }
                    if (part_row) {
#pragma unroll
                        for (int c = 0; c < 16; c += 4) *reinterpret_cast<float4*>(part_row + (cc * 4 + c / 4) * 128 * 4) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
                    }
                }
                if (grp == 0) {
                    if (whole) {
                        if (row == 0) p.unit_parts[unit] = make_int2(-1, -1);       // nothing for the merge kernel to do
                    } else {
                        // a NaN sum must reach the output: the merge gives such a piece all the weight
                        if (row_valid) p.part_lse[slot * 128 + row] = gone || l == 0.f ? -INFINITY : l != l ? 3.0e38f : mx + log2f(l) - BIAS;
                        if (g.t_a == 0 && row == 0) {                      // tells the merge kernel which blocks share the unit
                            const long long u0 = g.u0 + HEAD;              // the groups that hold its first and its last tile
                            const int j_lo = (int)(((u0 + 1) * ncg + T - 1) / T) - 1;
                            const int j_hi = (int)(((u0 + last_tile + 1) * ncg + T - 1) / T) - 1;
                            p.unit_parts[unit] = make_int2(j_lo, j_hi);
                        }
                    }
                }
                // both groups have read both accumulators before either goes on to overwrite its own
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(BAR_PART + quarter));
                const bool parted = wait(bar(BAR_PART + quarter), (uint32_t)sg & 1u, abort_flag);
                if (!__all_sync(0xffffffffu, parted)) { alive = false; break; }
            }
        }
        __syncthreads();                                                   // every role is done with this list
        if (*abort_flag) break;
    }

    tcgen05_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (tid == 0) deer_report(p.kv.status, DEER_ERR_TIMEOUT);
        for (int i = 0; i < 64; ++i) __nanosleep(10000);                   // copies still in flight land before the memory goes away
        __syncthreads();
    }
    if (warp == 1) {
        __syncwarp();
        tcgen05_fence_after();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// Thread blocks for a call: one per SM, fewer when the tiles would not give each of them a few.
static int pick_blocks(int B, int Hkv, int row_tiles, int max_seq_len) {
    const long long t_max = (long long)B * Hkv * ((max_seq_len / PAGE + PAGES - 1) / PAGES + 1);
    long long groups = t_max / 4, most = deer_sm_count() / row_tiles;
    if (groups > most) groups = most;
    if (groups < 1) groups = 1;
    return (int)groups * row_tiles;
}

// Joins the pieces of the units that were cut: a thread per row and four dims, the pieces' sums and results eight at a time
// (they come from L2, and a load of one at a time would cost its latency eighteen times over in a long context).  Blocks
// small enough to sit beside the attention kernel's, waiting for it.  (C2 block: joined by a warp per row, two pieces at a
// time, and stored by rows 27.0 us; like this 22.5.)
__global__ void __launch_bounds__(128, 8) attn_quant_merge_kernel(const AttnParams p) {
    const int unit = blockIdx.x >> 5, c4 = blockIdx.x & 31, r = threadIdx.x;
    const int Hkv = p.kv.n_kv_heads, HR = Hkv * p.row_tiles, RT = p.row_tiles, ncg = p.nc / RT;
    const int b = unit / HR, hr = unit % HR, kvh = hr / RT, rt = hr % RT;
    const int rows = min(p.ipt, p.k - rt * p.ipt) * p.G;
    pdl_trigger();
    pdl_wait();                                                   // the attention kernel's partial results
    const int2 parts = p.unit_parts[unit];
    const long long T = *p.total_tiles;
    // (a block that gave up on a wait may have left its units' entries unwritten: nothing outside the workspace is read then)
    if (parts.x < 0 || parts.y < parts.x || parts.y >= ncg || r >= rows) return;
    const int nj = parts.y - parts.x + 1;
    const size_t slot0 = ((size_t)b * Hkv + kvh + parts.x) * RT + rt;      // the pieces of a unit sit RT slots apart
    const float* lse = p.part_lse + slot0 * 128 + r;
    const float* o = p.part_o + slot0 * 128 * HD + (size_t)(c4 * 128 + r) * 4;
    const bool dense = T >= ncg;                                  // with fewer tiles than groups some shares are empty
    float m = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < nj; j0 += 8) {
        float l[8];
        float4 v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int jj = j0 + e;
            const bool on = jj < nj && (dense || attn::share_begin(T, parts.x + jj + 1, ncg) > attn::share_begin(T, parts.x + jj, ncg));
            l[e] = on ? lse[(size_t)jj * RT * 128] : -INFINITY;
            v[e] = on ? *reinterpret_cast<const float4*>(o + (size_t)jj * RT * 128 * HD) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float top = m;
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, l[e]);
        if (top == -INFINITY) continue;
        const float corr = m == -INFINITY ? 0.f : exp2f(m - top);
        sum *= corr;
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] *= corr;
        m = top;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (l[e] == -INFINITY) continue;
            const float w = exp2f(l[e] - m);
            sum += w;
            acc[0] = fmaf(w, v[e].x, acc[0]);
            acc[1] = fmaf(w, v[e].y, acc[1]);
            acc[2] = fmaf(w, v[e].z, acc[2]);
            acc[3] = fmaf(w, v[e].w, acc[3]);
        }
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    __nv_bfloat16* dst = p.out + ((size_t)(b * p.k + rt * p.ipt + r / p.G) * p.Hq + kvh * p.G + r % p.G) * HD + c4 * 4;
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv));
}

}  // namespace umma

// More query rows than a warp's tile of 16 hold share the KV stream here; fewer leave the 128 lanes idle while the
// warp-level kernel reads the same bytes with less latency.
// This kernel takes about 15 us for any call, however short (its pipeline's start, the queries' split, two joins); the
// warp-level one 6 to 8, and then the time for its pages, of which each costs 16 query rows as much as this one spends on
// 128.  Measured in us, warp-level against this, 32 query and 8 KV heads, tokens: 32 rows x 1003 13.3 / 18, x 2048
// 18.9 / 18.3, x 4096 27.1 / 22.4, x 8192 45 / 27.0; 8 rows x 8192 21.9 / 21; 8 sequences of 8 rows x 1003 19.7 / 23,
// x 4096 47.7 / 40.6; and with more row tiles than fit the SMs at once (16 sequences, 4 KV heads, 32 rows x 200) 36.0 / 17.
bool use_umma(int B, int D, int k, int Hq, int Hkv, int max_seq_len, float scale) {
    const int G = Hq / Hkv;
    if (D != umma::HD || G > 128 || !(scale > 0.f) || k * G <= ROWS_SMALL) return false;
    const long long tiles = (long long)B * Hkv * ((k * G + ROWS_SMALL - 1) / ROWS_SMALL);    // the warp-level kernel's
    return tiles > 2LL * deer_sm_count() || tiles * (max_seq_len / PAGE + 3) > 9000;
}

size_t umma_workspace_bytes(int B, int k, int Hq, int Hkv, int max_seq_len) {
    const int row_tiles = attn::umma_row_tiles(k, Hq / Hkv);
    const size_t units = (size_t)B * Hkv * row_tiles, slots = units + umma::pick_blocks(B, Hkv, row_tiles, max_seq_len);
    return slots * 128 * (umma::HD + 1) * sizeof(float) + units * sizeof(int2) + sizeof(long long);
}

int launch_umma(const Params& q, void* workspace, cudaStream_t st) {
    using namespace umma;
    QParams qp = {};
    AttnParams& p = qp.a;
    qp.kq = q.kq;
    p.kv = q.kv;
    p.seq_ids = q.seq_ids;
    p.row_state = q.row_state;
    p.q = q.q;
    p.k_blk = q.k_blk;
    p.v_blk = q.v_blk;
    p.out = q.out;
    p.B = q.B;
    p.k = q.k;
    p.Hq = q.Hq;
    p.G = q.G;
    p.R = q.G * q.k;
    p.mask = q.mask;
    p.scale_log2 = q.scale_log2;
    p.max_seq_len = q.max_seq_len;
    p.ipt = 128 / p.G;
    p.row_tiles = attn::umma_row_tiles(p.k, p.G);
    const int Hkv = p.kv.n_kv_heads;
    p.nc = pick_blocks(p.B, Hkv, p.row_tiles, p.max_seq_len);
    const size_t units = (size_t)p.B * Hkv * p.row_tiles, slots = units + p.nc;
    p.part_o = static_cast<float*>(workspace);
    p.part_lse = p.part_o + slots * 128 * HD;
    p.total_tiles = reinterpret_cast<long long*>(p.part_lse + slots * 128);
    p.unit_parts = reinterpret_cast<int2*>(p.total_tiles + 1);
    CUtensorMap tm_q, tm_k;
    const uint64_t dims[2] = {HD, (uint64_t)p.kv.num_pages * Hkv * PAGE}, str[1] = {HD};
    const uint32_t box[2] = {HD, PAGE};
    // q [B*k][Hq][128]: a box brings G heads of box_i block rows, 64 dims wide -> shared-memory row = i * G + g
    const uint64_t dims_q[3] = {HD, (uint64_t)p.Hq, (uint64_t)p.B * p.k}, str_q[2] = {HD * 2, (uint64_t)p.Hq * HD * 2};
    const uint32_t box_q[3] = {64, (uint32_t)p.G, (uint32_t)(p.ipt < p.k ? p.ipt : p.k)};
    int rc = make_map_bf16(&tm_q, p.q, 3, dims_q, str_q, box_q);
    if (rc != DEER_OK) return rc;
    rc = make_map_u8(&tm_k, p.kv.k_pool, 2, dims, str, box);
    if (rc != DEER_OK) return rc;
    DEER_CUDA(cudaFuncSetAttribute(attn_quant_umma_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES));
    DEER_CUDA(launch_pdl(attn_quant_umma_kernel, dim3((unsigned)p.nc), dim3(THREADS), (size_t)SMEM_BYTES, st, tm_q, tm_k, qp));
    DEER_CUDA(launch_pdl(attn_quant_merge_kernel, dim3((unsigned)(units * 32)), dim3(128), 0, st, p));
    return DEER_OK;
}

}  // namespace attnq
