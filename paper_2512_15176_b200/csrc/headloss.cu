// The losses of the LM head and their gradients: entry points, workspace, and the kernels that work by rows.
//
// A row's target is a distribution t over a list of tokens (cross entropy: one token, t = 1; distillation: the softmax of
// the teacher's logits of the list).  With z = h w^T / tau and lse = log sum exp z over the vocabulary,
//     loss    = a tau^2 sum_j t_j (log t_j - z_j + lse)          (j: tokens; what a list names twice has the sum of both)
//     G[m][v] = a g tau (exp(z_v - lse) - t_v),     dh = G w,     dw = G^T h
// (a: the row's weight, g: the upstream gradient of its loss).  The logits are never kept: the forward pass reduces each
// tile of z to (max, sum exp) per row, the backward pass computes z a second time, a piece of the vocabulary at a time,
// and keeps only that piece's G.  Four products of 2 live V hid operations in all bound both, at every size but the
// smallest; at few rows it is the reading of w (three times) and the writing of dw.
//
// The loss is linear in the rows, and rows without a target are common (positions that are not masked, padding), so the
// live rows are moved together first and everything behind works on those alone.  Their number stays on the device.
#include <limits.h>
#include <math.h>

#include "headloss.cuh"

namespace headloss {

constexpr int ROW_THREADS = 256, ROW_WARPS = ROW_THREADS / 32;
constexpr int ROW_BLOCKS = 512;            // blocks of the kernel that moves the rows, at most: each of them counts all rows
constexpr size_t PIECE_BYTES = size_t(256) << 20;      // of G at a time, but 1024 columns at least (more pieces: more part-filled
                                           // waves; fewer: more memory)
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f, LN2_LOW = (float)(0.6931471805599453 - (double)LN2);

// Columns of a tile, a multiple of `unit` up to 256: the one whose tiles over `rows` row tiles and `cols` columns keep
// the busiest block or pair shortest, a tile costing what 32 columns do beside its own (151936 columns at one row tile:
// 594 tiles of 256 take 148 blocks 5 rounds = 1280 columns, 731 of 208 take 5 as well = 1040).
static int tile_columns(long rows, long cols, int unit, int groups) {
    int best = 256;
    long best_cost = LONG_MAX;
    for (int n = 256; n >= 64; n -= unit) {
        const long cost = (rows * ((cols + n - 1) / n) + groups - 1) / groups * (n + 32);
        if (cost < best_cost) {
            best_cost = cost;
            best = n;
        }
    }
    return best;
}

Space lay_out(void* base, int M, int hid, int V, int K, bool grad) {
    Space s = {};
    const int pairs = deer_sm_count() / 2;
    s.Mp = (M + TILE - 1) / TILE * TILE;
    const int mt = s.Mp / TILE, groups = M > ONE_BLOCK ? pairs : deer_sm_count();
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? static_cast<char*>(base) + at : nullptr;
        at += (bytes + 1023) / 1024 * 1024;
        return p;
    };
    s.hdr = (int*)take(32);
    s.slot = (int*)take((size_t)M * 4);
    s.row = (int*)take((size_t)s.Mp * 4);
    s.ids = (int*)take((size_t)K * s.Mp * 4);
    s.h = (__nv_bfloat16*)take((size_t)s.Mp * hid * 2);
    if (!grad) {
        s.stats_n = tile_columns(mt, V, 16, groups);
        s.piece = V;
        s.piece_tiles = (V + s.stats_n - 1) / s.stats_n;
        s.first_pitch = (s.piece_tiles + 3) / 4 * 4;
        s.first = (uint8_t*)take(takes_rows_as_they_are(M, K) ? 0 : (size_t)s.Mp * s.first_pitch);
        s.place = (int*)take((size_t)K * s.Mp * 4);
        s.z = (float*)take((size_t)K * s.Mp * 4);
        s.part = (float2*)take((size_t)s.Mp * ((V + s.stats_n - 1) / s.stats_n) * STATS_SHARE * 8);
        s.bytes = at;
        return s;
    }
    // equal pieces, whole tiles of dw
    const long room = (long)(PIECE_BYTES / ((size_t)s.Mp * 2)) / TILE * TILE;
    const long most = room < 1024 ? 1024 : room;
    s.pieces = (int)((V + most - 1) / most);
    s.piece = (int)(((V + s.pieces - 1) / s.pieces + TILE - 1) / TILE * TILE);
    s.pieces = (V + s.piece - 1) / s.piece;
    s.grad_n = tile_columns(mt, s.piece < V ? s.piece : V, 16, groups);
    s.hid_n = tile_columns(1, hid, 32, 1);
    // space for dh's partial sums: as many ranges as two rounds of tiles take
    const int ht = (hid + s.hid_n - 1) / s.hid_n;
    s.slab_tiles = 2 * pairs / ht > mt ? 2 * pairs / ht : mt;
    s.coef = (float*)take((size_t)s.Mp * 4);
    s.lse2 = (float*)take((size_t)s.Mp * 4);
    s.piece_tiles = (s.piece + s.grad_n - 1) / s.grad_n;
    s.first_pitch = (s.pieces * s.piece_tiles + 3) / 4 * 4;
    s.first = (uint8_t*)take((size_t)s.Mp * s.first_pitch);
    s.rounding = (float*)take((size_t)ROW_BLOCKS * 32 * 4);
    s.gval = (float*)take((size_t)K * s.Mp * 4);
    s.g = (__nv_bfloat16*)take((size_t)s.Mp * s.piece * 2);
    s.slab = (float*)take((size_t)s.slab_tiles * TILE * hid * 4);
    s.bytes = at;
    return s;
}

struct RowArgs {
    int M, hid, V, K, per_block;
    const __nv_bfloat16* h;
    const int* ids;              // [M][K]
    const float* teacher;        // [M][K] or NULL (K = 1, t = 1)
    const float* weight;         // [M] or NULL
    const float* grad;           // [M] or NULL                     (gradient)
    const float* lse;            // [M]                             (loss: out; gradient: in)
    const float* target_logit;   // [M][K]
    float tau;
    int tile_n;                  // columns of a tile of STATS or GRAD
    int ht, steps, dw_tiles, pairs, slab_tiles;
    Space s;
};

__device__ __forceinline__ bool is_live(const RowArgs& a, int m) { return is_live(a.ids, a.weight, a.K, m); }
__device__ __forceinline__ float row_coef(const RowArgs& a, int m) {
    return (a.weight ? a.weight[m] : 1.f) * (a.grad ? a.grad[m] : 1.f) * a.tau;
}
// A row's coefficient relative to the call's largest finite one.  Without a finite one other than 0 it stays as it is: what is
// not finite must reach the gradients.
__device__ __forceinline__ float relative(float coef, float top) { return top > 0.f ? coef / top : coef; }
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ int warp_sum(int v) { return __reduce_add_sync(0xffffffffu, v); }

// Ranges that dh's contraction is cut into: as many as give every pair of blocks a tile, so that all of them read w at once
// (77 rows, hid 2048: nine ranges and then dw's tiles 290 us, four beside dw's tiles 305 us), and from there on the count
// with the shortest run of the launch, dw's tiles evening out what dh's leave; ranges of four steps at least, as many as
// there is space for their partial sums.  The lanes of a warp try one count each.
__device__ int dh_ranges(const RowArgs& a, int live, int lane) {
    const int mt = (live + TILE - 1) / TILE, tiles = mt * a.ht;
    if (mt == 0) return 1;
    const int dw_steps = dw_contraction(live);
    const int most = max(1, min(a.slab_tiles / mt, a.steps / 4)), least = max(1, min(a.pairs / tiles, most));
    const uint64_t dw_cost = (uint64_t)a.dw_tiles * dw_tile_cost(dw_steps);
    uint64_t best = ~uint64_t(0);              // cost, then the count
    for (int s = least + lane; s <= most; s += 32) {
        const uint32_t c = (uint32_t)dh_tile_cost(a.steps, s), n = (uint32_t)tiles * s;
        const uint64_t longest = (uint64_t)((n + a.pairs - 1) / a.pairs) * a.pairs * c, all = (uint64_t)n * c + dw_cost;
        const uint64_t cost = (longest > all ? longest : all) << 16 | (uint32_t)s;
        if (cost < best) best = cost;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, best, o);
        if (other < best) best = other;
    }
    return (int)(best & 0xffff);
}

// A warp's view of one row's list: lane l holds entries l, l + 32, ...
struct List {
    int n;                       // entries in front of the first negative id
    bool beyond;                 // an id of V or more among them
    int id[MAX_TOP / 32];
    float log_t[MAX_TOP / 32];   // the teacher's logits; after targets(): log t, -inf behind the list's end
    float z[MAX_TOP / 32];       // target_logit
    // Only loads, none of which waits for another.
    __device__ __forceinline__ void load(const RowArgs& a, const float* target_logit, int m, int lane) {
#pragma unroll
        for (int i = 0; i < MAX_TOP / 32; ++i) {
            const int j = i * 32 + lane;
            const size_t at = (size_t)m * a.K + j;
            id[i] = j < a.K ? a.ids[at] : -1;
            log_t[i] = j < a.K && a.teacher ? a.teacher[at] : 0.f;
            z[i] = j < a.K && target_logit ? target_logit[at] : 0.f;
        }
    }
    __device__ __forceinline__ void find_end(const RowArgs& a, int lane) {
        n = a.K;
        bool out = false;
#pragma unroll
        for (int i = 0; i < MAX_TOP / 32; ++i) {
            const unsigned end = __ballot_sync(0xffffffffu, id[i] < 0);
            if (end && i * 32 + __ffs(end) - 1 < n) n = i * 32 + __ffs(end) - 1;
        }
#pragma unroll
        for (int i = 0; i < MAX_TOP / 32; ++i) out |= i * 32 + lane < n && id[i] >= a.V;
        beyond = __any_sync(0xffffffffu, out);
    }
    // log t: the log-softmax of teacher / tau over the list, 0 for a list without a teacher.  False: the list holds no entry
    // above -inf, so that there is no distribution (the row then has neither loss nor gradient).
    __device__ __forceinline__ bool targets(const RowArgs& a, int lane) {
        float top = -INFINITY, sum = 0.f;
        bool some = false;
#pragma unroll
        for (int i = 0; i < MAX_TOP / 32; ++i) {
            if (i * 32 + lane >= n) log_t[i] = -INFINITY;
            some |= !(log_t[i] == -INFINITY);
            top = fmaxf(top, log_t[i]);
        }
        if (!a.teacher) return true;
        top = warp_max(top);
        if (!__any_sync(0xffffffffu, some)) return false;
#pragma unroll
        for (int i = 0; i < MAX_TOP / 32; ++i) {
            log_t[i] = (log_t[i] - top) / a.tau;           // (NaN where the teacher's is, or the largest is infinite)
            if (i * 32 + lane < n) sum += expf(log_t[i]);
        }
        const float log_sum = logf(warp_sum(sum));
#pragma unroll
        for (int i = 0; i < MAX_TOP / 32; ++i) log_t[i] -= log_sum;
        return true;
    }
};

__device__ __forceinline__ float factor_of(int i) { return 1.f + i * 0.03125f; }

// Sorts N x 32 keys of a warp, key i * 32 + lane in key[i], by a bitonic network.
template <int N>
__device__ __forceinline__ void sort_warp(uint64_t (&key)[MAX_TOP / 32], int lane) {
#pragma unroll
    for (int size = 2; size <= N * 32; size <<= 1)
#pragma unroll
        for (int step = size >> 1; step > 0; step >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool rising = ((i * 32 + lane) & size) == 0;
                if (step < 32) {
                    const uint64_t other = __shfl_xor_sync(0xffffffffu, key[i], step);
                    const bool keep_less = ((lane & step) == 0) == rising;
                    key[i] = (other < key[i]) == keep_less ? other : key[i];
                } else if ((i & (step / 32)) == 0) {
                    const uint64_t a = key[i], b = key[i | (step / 32)];
                    const bool swap = (b < a) == rising;
                    key[i] = swap ? b : a;
                    key[i | (step / 32)] = swap ? a : b;
                }
            }
}

// Moves the live rows together and lists their tokens by rising id.  A block takes `per_block` rows and counts the live
// ones among all rows itself (M flags from L2: less than the launch of a kernel that counts); a warp takes a row.
// GRAD: also what the products' epilogue needs of a row and of its listed tokens.
template <bool GRAD>
__global__ void __launch_bounds__(ROW_THREADS) head_rows_kernel(const RowArgs a) {
    __shared__ int sums[2][ROW_WARPS];
    __shared__ float tops[ROW_WARPS];
    __shared__ float list_g[GRAD ? ROW_WARPS : 1][MAX_TOP];        // G by rising id
    __shared__ float taken[GRAD ? ROW_WARPS : 1][32];
    __shared__ int list_id[GRAD ? ROW_WARPS : 1][MAX_TOP], sorted_id[ROW_WARPS][MAX_TOP];
    __shared__ float2 list_t[GRAD ? ROW_WARPS : 1][MAX_TOP];       // t and z by the list's order
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_trigger();
    pdl_wait();
    const int base = blockIdx.x * a.per_block;
    // what a row brings is on its way one row ahead, the first one's beside the counting
    const int chunks = a.hid / 8;                          // 16 bytes each
    List l;
    float lse = 0.f;
    uint4 x[4];
    auto load_row = [&](int m) {
        if (m >= a.M) return;
        l.load(a, a.target_logit, m, lane);
        if (GRAD) lse = a.lse[m];
        const uint4* src = reinterpret_cast<const uint4*>(a.h + (size_t)m * a.hid);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = lane + 32 * i < chunks ? src[lane + 32 * i] : make_uint4(0, 0, 0, 0);
    };
    load_row(base + warp);
    int before = 0, total = 0;
    float top = 0.f;                           // the largest finite coefficient: what G is relative to
#pragma unroll 4
    for (int m = tid; m < a.M; m += ROW_THREADS) {
        const int f = is_live(a, m);
        total += f;
        before += m < base ? f : 0;
        if (GRAD) {
            const float c = fabsf(row_coef(a, m));
            if (f && c < INFINITY) top = fmaxf(top, c);
        }
    }
    before = warp_sum(before);
    total = warp_sum(total);
    top = warp_max(top);
    if (lane == 0) {
        sums[0][warp] = before;
        sums[1][warp] = total;
        tops[warp] = top;
    }
    __syncthreads();
    before = total = 0;
#pragma unroll
    for (int i = 0; i < ROW_WARPS; ++i) {
        before += sums[0][i];
        total += sums[1][i];
        top = fmaxf(top, tops[i]);
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.s.hdr[HDR_LIVE] = total;
        a.s.hdr[HDR_GAVE_UP] = 0;
        a.s.hdr[HDR_SCALE] = __float_as_int(top > 0.f ? top : 1.f);
        a.s.hdr[HDR_FACTOR] = __float_as_int(1.f);
    }
    if (GRAD && blockIdx.x == 0 && warp == ROW_WARPS - 1) {
        const int ranges = dh_ranges(a, total, lane);
        if (lane == 0) a.s.hdr[HDR_RANGES] = ranges;
    }
    // what dw's contraction meets behind the live rows is zeros; the second term's rows of G meet a copy of h
    const int low = GRAD && total <= TWO_TERMS ? low_term(total) : 0;
    const int fill_end = low ? low : (total + STEP - 1) / STEP * STEP;
    const float factor = factor_of(lane);
    float lost = 0.f;
    for (int g = 0; g < a.per_block; g += 32) {
        const int here = min(32, a.per_block - g);
        const unsigned mask = __ballot_sync(0xffffffffu, lane < here && base + g + lane < a.M && is_live(a, base + g + lane));
        for (int r = warp; r < here; r += ROW_WARPS) {
            const int m = base + g + r;
            if (GRAD && m >= total && m < fill_end) {
                uint4* dst = reinterpret_cast<uint4*>(a.s.h + (size_t)m * a.hid);
                for (int c = lane; c < chunks; c += 32) {
                    dst[c] = make_uint4(0, 0, 0, 0);
                    if (low) dst[(size_t)low * chunks + c] = make_uint4(0, 0, 0, 0);
                }
            }
            if (m >= a.M) continue;
            if (!((mask >> r) & 1u)) {
                if (lane == 0) a.s.slot[m] = -1;
                load_row(m + ROW_WARPS);
                continue;
            }
            const int slot = before + __popc(mask & ((1u << r) - 1u));
            l.find_end(a, lane);
            float coef = 0.f;
            if (GRAD) {
                const bool some = l.targets(a, lane);
                coef = some && !l.beyond ? relative(row_coef(a, m), top) : 0.f;
            }
            if (lane == 0) {
                a.s.slot[m] = slot;
                a.s.row[slot] = m;
                if (GRAD) {
                    a.s.coef[slot] = coef;
                    a.s.lse2[slot] = lse * LOG2E;
                }
            }
            const uint4* src = reinterpret_cast<const uint4*>(a.h + (size_t)m * a.hid);
            uint4* dst = reinterpret_cast<uint4*>(a.s.h + (size_t)slot * a.hid);
            for (int c0 = lane; c0 < chunks; c0 += 128) {
                if (c0 >= 128)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = c0 + 32 * i < chunks ? src[c0 + 32 * i] : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c0 + 32 * i < chunks) {
                        dst[c0 + 32 * i] = x[i];
                        if (low) dst[(size_t)low * chunks + c0 + 32 * i] = x[i];
                    }
            }
            // the list by rising id (and by its own order among equals): an entry is its id and where it stood
            uint64_t key[MAX_TOP / 32];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < MAX_TOP / 32; ++i) {
                const int j = i * 32 + lane;
                key[i] = (uint64_t)(j < l.n ? (uint32_t)l.id[i] : 0x7fffffffu) << 32 | (uint32_t)j;
                if (GRAD) list_t[warp][j] = make_float2(expf(l.log_t[i]), l.z[i]);
            }
            __syncwarp();
            if (a.K <= 32) sort_warp<1>(key, lane);
            else if (a.K <= 64) sort_warp<2>(key, lane);
            else sort_warp<4>(key, lane);
            bool repeats = false;
            if (GRAD) {
#pragma unroll
                for (int i = 0; i < MAX_TOP / 32; ++i) {
                    const int id = (int)(key[i] >> 32);
                    int left = __shfl_up_sync(0xffffffffu, id, 1);
                    const int behind = i > 0 ? (int)(__shfl_sync(0xffffffffu, key[i > 0 ? i - 1 : 0], 31) >> 32) : -1;
                    if (lane == 0) left = behind;
                    repeats |= i * 32 + lane < l.n && left == id;
                    list_id[warp][i * 32 + lane] = l.id[i];
                }
                repeats = __any_sync(0xffffffffu, repeats);
                __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < MAX_TOP / 32; ++i) {
                const int place = i * 32 + lane, id = (int)(key[i] >> 32), j = (int)(key[i] & 0x7f);
                int left = __shfl_up_sync(0xffffffffu, id, 1);
                const int behind = i > 0 ? (int)(__shfl_sync(0xffffffffu, key[i > 0 ? i - 1 : 0], 31) >> 32) : -1;
                if (lane == 0) left = behind;
                if (place >= a.K) continue;
                a.s.ids[(size_t)slot * a.K + place] = sorted_id[warp][place] = place < l.n ? id : INT_MAX;
                if (!GRAD) a.s.place[(size_t)slot * a.K + j] = left == id ? -1 : place;
                if (GRAD && place < l.n) {
                    float t = list_t[warp][j].x;           // the token's probability, wherever the list names it
                    if (repeats) {
                        t = 0.f;
                        for (int o = 0; o < l.n; ++o) t += list_id[warp][o] == id ? list_t[warp][o].x : 0.f;
                    }
                    const float g = coef == 0.f ? 0.f : coef * (expf(list_t[warp][j].y / a.tau - lse) - t);
                    a.s.gval[(size_t)slot * a.K + place] = g;
                    list_g[warp][place] = g;
                }
            }
            __syncwarp();
            // where the list stands at each of the products' tiles: a lane walks a run of them, four to a store
            const int run = (a.s.first_pitch / 4 + 31) / 32 * 4, tile0 = lane * run, tile1 = min(tile0 + run, a.s.first_pitch);
            if (tile0 < tile1) {
                int piece = tile0 / a.s.piece_tiles, in_piece = tile0 - piece * a.s.piece_tiles;
                int from = piece * a.s.piece + in_piece * a.tile_n, e = 0, hi = l.n;
                while (e < hi) {
                    const int mid = (e + hi) >> 1;
                    if (sorted_id[warp][mid] < from) e = mid + 1;
                    else hi = mid;
                }
                int next = e < l.n ? sorted_id[warp][e] : INT_MAX;
                for (int tile = tile0; tile < tile1; tile += 4) {
                    uint32_t four = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        while (next < from) next = ++e < l.n ? sorted_id[warp][e] : INT_MAX;
                        four |= (uint32_t)e << (8 * i);
                        from += a.tile_n;
                        if (++in_piece == a.s.piece_tiles) {
                            in_piece = 0;
                            from = ++piece * a.s.piece;
                        }
                    }
                    *reinterpret_cast<uint32_t*>(a.s.first + (size_t)slot * a.s.first_pitch + tile) = four;
                }
            }
            if (GRAD && total > DW_TERMS) {                // a lane tries one factor
                for (int o = 0; o < l.n; ++o) {
                    const float g = list_g[warp][o] * factor, off = g - __bfloat162float(__float2bfloat16(g));
                    lost = fmaf(off, off, lost);
                }
            }
            load_row(m + ROW_WARPS);
        }
        before += __popc(mask);
    }
    if (GRAD && total > DW_TERMS) {
        taken[warp][lane] = lost / (factor * factor);
        __syncthreads();
        if (warp == 0) {
            float all = 0.f;
#pragma unroll
            for (int i = 0; i < ROW_WARPS; ++i) all += taken[i][lane];
            a.s.rounding[(size_t)blockIdx.x * 32 + lane] = all;
        }
    }
}

// The factor that goes with the call's largest coefficient: what rounding takes of G at the listed tokens depends on where
// their values lie between two powers of two, and their common scale is free.  Of 32 scales the one that loses least.
__global__ void __launch_bounds__(1024) head_factor_kernel(const RowArgs a, int blocks) {
    __shared__ float sums[32][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();
    pdl_wait();
    float lost = 0.f;
    if (a.s.hdr[HDR_LIVE] > DW_TERMS)
        for (int b = warp; b < blocks; b += 32) lost += a.s.rounding[(size_t)b * 32 + lane];
    sums[warp][lane] = lost;
    __syncthreads();
    if (warp > 0 || a.s.hdr[HDR_LIVE] <= DW_TERMS) return;
    lost = 0.f;
    for (int i = 0; i < 32; ++i) lost += sums[i][lane];
    // (a sum is not negative: its bits are in its order; NaN, of a row that is not finite, behind all)
    const uint32_t best = __reduce_min_sync(0xffffffffu, __float_as_uint(lost));
    const int which = __ffs(__ballot_sync(0xffffffffu, __float_as_uint(lost) == best)) - 1;
    if (lane == 0) {
        a.s.hdr[HDR_FACTOR] = __float_as_int(factor_of(which));
        a.s.hdr[HDR_SCALE] = __float_as_int(__int_as_float(a.s.hdr[HDR_SCALE]) / factor_of(which));
    }
}

// lse and loss of every row from its tiles' partial sums: a warp per row, or (few rows, which may have thousands) a block.
__global__ void __launch_bounds__(ROW_THREADS) head_loss_kernel(const RowArgs a, int as_is, int wide, int tiles, float2 plain, float2 tile, float* loss, float* lse_out, float* target_logit) {
    __shared__ float2 warps[ROW_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m = wide ? blockIdx.x : blockIdx.x * ROW_WARPS + warp;
    pdl_trigger();
    pdl_wait();
    if (m >= a.M) return;                                  // (never a part of a block, where wide)
    const int slot = as_is ? (is_live(a, m) ? m : -1) : a.s.slot[m];       // (as STATS took them)
    List l;
    l.load(a, target_logit, m, lane);
    l.find_end(a, lane);
    if (slot < 0) {
        if (wide && warp > 0) return;
        for (int j = lane; j < a.K; j += 32) target_logit[(size_t)m * a.K + j] = 0.f;
        if (lane == 0) loss[m] = lse_out[m] = 0.f;
        return;
    }
    // in powers of two, relative to the largest of the tiles' references
    const float2* part = a.s.part + (size_t)slot * tiles;
    float top = -INFINITY, sum = 0.f;                      // (a lane's, and its sum relative to that)
    const int step = wide ? ROW_THREADS : 32;
    for (int i0 = wide ? threadIdx.x : lane; i0 < tiles; i0 += 4 * step) {
        float2 p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = i0 + i * step < tiles ? part[i0 + i * step] : make_float2(-INFINITY, 0.f);
        const float m2 = fmaxf(fmaxf(fmaxf(p[0].x, p[1].x), fmaxf(p[2].x, p[3].x)), top), shift = m2 == -INFINITY ? 0.f : m2;
        sum *= exp2f(top - shift);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = fmaf(p[i].y, exp2f(p[i].x - shift), sum);
        top = m2;
    }
    float all = warp_max(top);
    sum = warp_sum(sum * (top == -INFINITY ? 0.f : exp2f(top - all)));
    if (wide) {                                            // the first warp goes on with the block's
        if (lane == 0) warps[warp] = make_float2(all, sum);
        __syncthreads();
        if (warp > 0) return;
        const float2 p = lane < ROW_WARPS ? warps[lane] : make_float2(-INFINITY, 0.f);
        all = warp_max(p.x);
        sum = warp_sum(p.y * (p.x == -INFINITY ? 0.f : exp2f(p.x - all)));
    }
    const bool some = l.targets(a, lane);
#pragma unroll
    for (int i = 0; i < MAX_TOP / 32; ++i) {
        const int j = i * 32 + lane;
        if (j < a.K && (j >= l.n || l.id[i] >= a.V)) target_logit[(size_t)m * a.K + j] = 0.f;
    }
    // the listed tokens' z: by plain sums in target_logit, as the tiles have it in s.z; each token once.  A low temperature makes
    // their difference large: a plain one far above the reference becomes the reference.
    float beyond = 0.f;
#pragma unroll
    for (int i = 0; i < MAX_TOP / 32; ++i) {
        if (i * 32 + lane >= l.n || l.id[i] >= a.V) continue;
        l.z[i] = fmaf(l.z[i], plain.y, fmaf(l.z[i], plain.x, -all));
        beyond = fmaxf(beyond, l.z[i]);
    }
    if (__any_sync(0xffffffffu, beyond > 64.f)) {          // (out of range else)
        beyond = warp_max(beyond);
        all += beyond;
        sum *= exp2f(-beyond);
    } else {
        beyond = 0.f;
    }
    float more = 0.f;
    bool repeats = false;
#pragma unroll
    for (int i = 0; i < MAX_TOP / 32; ++i) {
        const int j = i * 32 + lane;
        if (j >= l.n || l.id[i] >= a.V) continue;
        int at = j;                                        // (as they are: each token at its first entry)
        if (as_is)
            for (int o = 0; o < j; ++o) at = a.ids[(size_t)m * a.K + o] == l.id[i] ? -1 : at;
        else at = a.s.place[(size_t)slot * a.K + j];
        l.z[i] -= beyond;
        repeats |= at < 0;
        if (at < 0) continue;
        const float tile_z = a.s.z[(size_t)slot * a.K + at];
        more += exp2f(l.z[i]) - exp2f(fmaf(tile_z, tile.y, fmaf(tile_z, tile.x, -all)));
    }
    const float log_sum = logf(sum + warp_sum(more));
    float t[MAX_TOP / 32], each = 0.f;
#pragma unroll
    for (int i = 0; i < MAX_TOP / 32; ++i) t[i] = i * 32 + lane < l.n ? expf(l.log_t[i]) : 0.f;
    if (__any_sync(0xffffffffu, repeats)) {                // log t of a token is that of the sum over its entries
        float token[MAX_TOP / 32] = {};
#pragma unroll
        for (int c = 0; c < MAX_TOP / 32; ++c)
            for (int from = 0; from < 32; ++from) {
                const int id = __shfl_sync(0xffffffffu, l.id[c], from);
                const float some_t = __shfl_sync(0xffffffffu, t[c], from);
#pragma unroll
                for (int i = 0; i < MAX_TOP / 32; ++i) token[i] += c * 32 + from < l.n && l.id[i] == id ? some_t : 0.f;
            }
#pragma unroll
        for (int i = 0; i < MAX_TOP / 32; ++i)
            if (token[i] > t[i]) l.log_t[i] = logf(token[i]);
    }
#pragma unroll
    for (int i = 0; i < MAX_TOP / 32; ++i)
        if (i * 32 + lane < l.n && l.id[i] < a.V && !(t[i] == 0.f)) each += t[i] * (l.log_t[i] + fmaf(l.z[i], -LN2, log_sum));
    each = warp_sum(each);
    if (lane == 0) {
        const float x = (a.weight ? a.weight[m] : 1.f) * (a.tau * a.tau) * each;
        loss[m] = l.beyond ? NAN : some ? x : 0.f;
        lse_out[m] = fmaf(all, LN2, fmaf(all, LN2_LOW, log_sum));
    }
}

// dh of every row: the partial sums of its ranges in a fixed order, zeros for a dead row.  A block takes 128 columns of
// up to eight rows; where there are many partial sums its warps share a row's, so that they are all on their way at once.
// As the call's last kernel it also marks what a product that gave up has left: dh and dw all NaN.  dh, dw: NULL where not
// asked for.
__global__ void __launch_bounds__(ROW_THREADS) head_dh_kernel(const RowArgs a, int per_block, __nv_bfloat16* dh, __nv_bfloat16* dw) {
    __shared__ float4 sums[ROW_WARPS][ROW_WARPS][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int m0 = blockIdx.x * per_block, rows = min(per_block, a.M - m0), c = (blockIdx.y * 32 + lane) * 4;
    const bool in = c < a.hid;
    pdl_trigger();
    pdl_wait();
    const int gave_up = a.s.hdr[HDR_GAVE_UP], live = a.s.hdr[HDR_LIVE], ranges = a.s.hdr[HDR_RANGES];
    const float call_scale = __int_as_float(a.s.hdr[HDR_SCALE]);
    if (dw && gave_up) {
        uint4* to = reinterpret_cast<uint4*>(dw);          // (rows are a multiple of 16 bytes)
        const size_t n = (size_t)a.V * a.hid / 8, threads = (size_t)gridDim.x * gridDim.y * ROW_THREADS;
        for (size_t i = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * ROW_THREADS + threadIdx.x; i < n; i += threads)
            to[i] = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
    }
    if (!dh) return;
    // few live rows: a range's tile holds the two terms' products, 128 rows each; nothing is read behind a product that gave up
    const int parts = gave_up ? 0 : live <= TWO_TERMS ? 2 * ranges : ranges;
    const size_t part_rows = live <= TWO_TERMS ? TILE / 2 : (size_t)((live + TILE - 1) / TILE) * TILE;
    const float scale = gave_up ? NAN : call_scale;
    auto part_sum = [&](int slot, int first, int step) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        const float* src = a.s.slab + (size_t)slot * a.hid + c;
#pragma unroll 8
        for (int r = first; r < parts; r += step) {
            const float4 x = *reinterpret_cast<const float4*>(src + (size_t)r * part_rows * a.hid);
            v.x += x.x;
            v.y += x.y;
            v.z += x.z;
            v.w += x.w;
        }
        return v;
    };
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    const bool share = parts > 4;
    if (share && in)
        for (int r = 0; r < rows; ++r) {
            const int slot = a.s.slot[m0 + r];
            if (slot >= 0) sums[r][warp][lane] = part_sum(slot, warp, ROW_WARPS);
        }
    __syncthreads();
    if (warp >= rows || !in) return;
    const int slot = a.s.slot[m0 + warp];
    float4 v = zero;
    if (slot >= 0 && !share) v = part_sum(slot, 0, 1);
    if (slot >= 0 && share)
#pragma unroll
        for (int i = 0; i < ROW_WARPS; ++i) {
            const float4 x = sums[warp][i][lane];
            v.x += x.x;
            v.y += x.y;
            v.z += x.z;
            v.w += x.w;
        }
    *reinterpret_cast<uint2*>(dh + (size_t)(m0 + warp) * a.hid + c) = make_uint2(pack_bf16(v.x * scale, v.y * scale), pack_bf16(v.z * scale, v.w * scale));
}

static int check_sizes(const char* call, int K, float tau, int M, int hid, int V) {
    DEER_CHECK_ARG(M >= 0 && V >= 1, DEER_ERR_INVALID_ARG, "%s: M must not be negative, V at least 1", call);
    DEER_CHECK_ARG(M <= (1 << 18) && V <= (1 << 30), DEER_ERR_UNSUPPORTED, "%s: more than 2^18 rows or 2^30 tokens", call);
    DEER_CHECK_ARG(hid >= 64 && hid % 64 == 0 && hid <= 65536, DEER_ERR_UNSUPPORTED, "%s: hid must be a multiple of 64, at most 65536", call);
    DEER_CHECK_ARG(K >= 1 && K <= MAX_TOP, DEER_ERR_UNSUPPORTED, "%s: a list has 1 to %d entries", call, MAX_TOP);
    DEER_CHECK_ARG(tau > 0.f && tau < INFINITY, DEER_ERR_INVALID_ARG, "%s: temperature must be positive and finite", call);
    // (beyond these fp32 logits have no bits left for a loss: |z| / tau below, z - z' above)
    DEER_CHECK_ARG(tau >= 0x1p-20f && tau <= 0x1p20f, DEER_ERR_UNSUPPORTED, "%s: temperature must be 2^-20 to 2^20", call);
    return DEER_OK;
}
static int check_pointers(const char* call, const void* h, const void* w, const int32_t* ids, const float* teacher, bool needs_teacher,
                          const float* row_weight, const float* lse, const float* target_logit) {
    DEER_CHECK_ARG(h && w && ids && lse && target_logit && (teacher || !needs_teacher), DEER_ERR_INVALID_ARG, "%s: null pointer", call);
    DEER_CHECK_ARG(deer_aligned16(h) && deer_aligned16(w), DEER_ERR_INVALID_ARG, "%s: h and w must be 16-byte aligned", call);
    DEER_CHECK_ARG(deer_aligned4(ids) && deer_aligned4(teacher) && deer_aligned4(row_weight) && deer_aligned4(lse) && deer_aligned4(target_logit),
                   DEER_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    return DEER_OK;
}

static bool overlap(const void* p, size_t n, const void* q, size_t m) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return p && q && a < b + m && b < a + n;
}

// The kernels by rows run between products that use an SM's whole shared memory: with the same split of its memory they
// may start beside the end of one, and the SM need not drain to change the split.
template <typename Kernel>
static cudaError_t keep_split(Kernel* kernel, bool (&done)[64]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && done[dev])) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (dev < 64) done[dev] = e == cudaSuccess;
    return e;
}

static RowArgs row_args(const Space& s, const void* h, const int32_t* ids, const float* teacher, int K, float tau, const float* row_weight,
                        int M, int hid, int V) {
    RowArgs a = {};
    a.M = M;
    a.hid = hid;
    a.V = V;
    a.K = K;
    a.per_block = ROW_WARPS * (((M + STEP - 1) / STEP * STEP + ROW_WARPS * ROW_BLOCKS - 1) / (ROW_WARPS * ROW_BLOCKS));
    a.h = static_cast<const __nv_bfloat16*>(h);
    a.ids = ids;
    a.teacher = teacher;
    a.weight = row_weight;
    a.tau = tau;
    a.s = s;
    return a;
}
static unsigned row_blocks(const RowArgs& a) {             // all rows, and the places that are filled up behind them
    return (unsigned)(((a.M + STEP - 1) / STEP * STEP + a.per_block - 1) / a.per_block);
}

static int loss_call(const char* call, const void* h, const void* w, const int32_t* ids, const float* teacher, bool needs_teacher, int K,
                     float tau, const float* row_weight, int M, int hid, int V, float* loss, float* lse, float* target_logit,
                     void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(call, K, tau, M, hid, V);
    if (rc != DEER_OK || M == 0) return rc;
    rc = check_pointers(call, h, w, ids, teacher, needs_teacher, row_weight, lse, target_logit);
    if (rc != DEER_OK) return rc;
    DEER_CHECK_ARG(loss && deer_aligned4(loss), DEER_ERR_INVALID_ARG, "%s: loss is null or misaligned", call);
    const Space s = lay_out(workspace, M, hid, V, K, false);
    DEER_CHECK_ARG(workspace && deer_aligned16(workspace) && workspace_bytes >= s.bytes, DEER_ERR_WORKSPACE,
                   "%s: needs a 16-byte aligned workspace of %zu bytes", call, s.bytes);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    RowArgs a = row_args(s, h, ids, teacher, K, tau, row_weight, M, hid, V);
    a.tile_n = s.stats_n;
    float2 plain, tile;
    scale_of(tau, plain.x, plain.y);
    tile_scale_of(tau, hid, tile.x, tile.y);
    static bool rows_set[64] = {}, loss_set[64] = {};
    DEER_CUDA(keep_split(head_rows_kernel<false>, rows_set));
    DEER_CUDA(keep_split(head_loss_kernel, loss_set));
    const bool as_is = takes_rows_as_they_are(M, K);
    if (!as_is) DEER_CUDA(launch_pdl(head_rows_kernel<false>, dim3(row_blocks(a)), dim3(ROW_THREADS), 0, st, a));
    rc = launch_product(STATS, s, h, w, ids, row_weight, M, hid, V, K, 0, tau, target_logit, false, nullptr, st);
    if (rc != DEER_OK) return rc;
    const bool wide = M <= 512;
    DEER_CUDA(launch_pdl(head_loss_kernel, dim3(wide ? M : (M + ROW_WARPS - 1) / ROW_WARPS), dim3(ROW_THREADS), 0, st, a, (int)as_is, (int)wide, (V + s.stats_n - 1) / s.stats_n * STATS_SHARE, plain, tile,
                         loss, lse, target_logit));
    return DEER_OK;
}

// What is behind the products of a gradient call.
static int finish_grad(const RowArgs& a, void* dh, void* dw, cudaStream_t st) {
    static bool dh_set[64] = {};
    DEER_CUDA(keep_split(head_dh_kernel, dh_set));
    const int per_block = a.M <= 512 ? 1 : ROW_WARPS;      // (few rows may have many partial sums each)
    const dim3 grid = dh ? dim3((unsigned)((a.M + per_block - 1) / per_block), (unsigned)((a.hid + 127) / 128)) : dim3((unsigned)deer_sm_count());
    DEER_CUDA(launch_pdl(head_dh_kernel, grid, dim3(ROW_THREADS), 0, st, a, per_block, static_cast<__nv_bfloat16*>(dh), static_cast<__nv_bfloat16*>(dw)));
    return DEER_OK;
}

static int grad_call(const char* call, const void* h, const void* w, const int32_t* ids, const float* teacher, bool needs_teacher, int K,
                     float tau, const float* row_weight, const float* grad_loss, const float* lse, const float* target_logit, int M, int hid,
                     int V, void* dh, void* dw, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(call, K, tau, M, hid, V);
    if (rc != DEER_OK) return rc;
    DEER_CHECK_ARG(deer_aligned16(dh) && deer_aligned16(dw), DEER_ERR_INVALID_ARG, "%s: dh and dw must be 16-byte aligned", call);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (M == 0) {
        if (dw) DEER_CUDA(cudaMemsetAsync(dw, 0, (size_t)V * hid * 2, st));
        return DEER_OK;
    }
    rc = check_pointers(call, h, w, ids, teacher, needs_teacher, row_weight, lse, target_logit);
    if (rc != DEER_OK) return rc;
    DEER_CHECK_ARG(dh || dw, DEER_ERR_INVALID_ARG, "%s: neither dh nor dw is asked for", call);
    DEER_CHECK_ARG(deer_aligned4(grad_loss), DEER_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    const Space s = lay_out(workspace, M, hid, V, K, true);
    DEER_CHECK_ARG(workspace && deer_aligned16(workspace) && workspace_bytes >= s.bytes, DEER_ERR_WORKSPACE,
                   "%s: needs a 16-byte aligned workspace of %zu bytes", call, s.bytes);
    const size_t h_bytes = (size_t)M * hid * 2, w_bytes = (size_t)V * hid * 2, rows = (size_t)M * 4;
    auto clear = [&](const void* out, size_t n) {          // of every input and of the workspace
        return !(overlap(out, n, h, h_bytes) || overlap(out, n, w, w_bytes) || overlap(out, n, ids, rows * K) || overlap(out, n, teacher, rows * K) ||
                 overlap(out, n, row_weight, rows) || overlap(out, n, grad_loss, rows) || overlap(out, n, lse, rows) ||
                 overlap(out, n, target_logit, rows * K) || overlap(out, n, workspace, s.bytes));
    };
    DEER_CHECK_ARG(clear(dh, h_bytes) && clear(dw, w_bytes) && !overlap(dh, h_bytes, dw, w_bytes), DEER_ERR_INVALID_ARG,
                   "%s: a gradient overlaps an operand, the other gradient or the workspace", call);
    RowArgs a = row_args(s, h, ids, teacher, K, tau, row_weight, M, hid, V);
    a.tile_n = s.grad_n;
    a.grad = grad_loss;
    a.lse = lse;
    a.target_logit = target_logit;
    a.ht = (hid + s.hid_n - 1) / s.hid_n;
    a.steps = (s.piece + STEP - 1) / STEP;
    a.dw_tiles = dw ? (s.piece + TILE - 1) / TILE * a.ht : 0;
    a.pairs = deer_sm_count() / 2;
    a.slab_tiles = s.slab_tiles;
    static bool rows_set[64] = {}, factor_set[64] = {};
    DEER_CUDA(keep_split(head_factor_kernel, factor_set));
    DEER_CUDA(keep_split(head_rows_kernel<true>, rows_set));
    DEER_CUDA(launch_pdl(head_rows_kernel<true>, dim3(row_blocks(a)), dim3(ROW_THREADS), 0, st, a));
    if (M > DW_TERMS) DEER_CUDA(launch_pdl(head_factor_kernel, dim3(1), dim3(1024), 0, st, a, (int)row_blocks(a)));
    for (int p = 0; p < s.pieces; ++p) {
        rc = launch_product(GRAD, s, h, w, ids, row_weight, M, hid, V, K, p, tau, nullptr, false, nullptr, st);
        if (rc == DEER_OK) rc = launch_product(BACK, s, h, w, ids, row_weight, M, hid, V, K, p, tau, nullptr, dh != nullptr, dw, st);
        if (rc != DEER_OK) return rc;
    }
    return finish_grad(a, dh, dw, st);
}

// The end of a gradient call again, as if one of its products had given up.
static int selftest_gave_up(int M, int hid, int V, int K, void* dh, void* dw, void* workspace, size_t workspace_bytes, void* stream) {
    const char* call = "deer_selftest_lmhead_gave_up";
    const int rc = check_sizes(call, K, 1.f, M, hid, V);
    if (rc != DEER_OK) return rc;
    DEER_CHECK_ARG(M > 0 && (dh || dw) && deer_aligned16(dh) && deer_aligned16(dw), DEER_ERR_INVALID_ARG, "%s: no rows, no gradient or a misaligned one", call);
    const Space s = lay_out(workspace, M, hid, V, K, true);
    DEER_CHECK_ARG(workspace && deer_aligned16(workspace) && workspace_bytes >= s.bytes, DEER_ERR_WORKSPACE,
                   "%s: needs a 16-byte aligned workspace of %zu bytes", call, s.bytes);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    DEER_CUDA(cudaMemsetAsync(s.hdr + HDR_GAVE_UP, 1, 4, st));
    return finish_grad(row_args(s, nullptr, nullptr, nullptr, K, 1.f, nullptr, M, hid, V), dh, dw, st);
}

}  // namespace headloss

extern "C" {

int deer_selftest_lmhead_gave_up(int M, int hid, int V, int K, void* dh, void* dw, void* workspace, size_t workspace_bytes, void* stream) {
    return headloss::selftest_gave_up(M, hid, V, K, dh, dw, workspace, workspace_bytes, stream);
}

size_t deer_lmhead_loss_workspace_bytes(int M, int hid, int V, int K, int grad) {
    if (M <= 0 || M > (1 << 18) || hid < 64 || hid % 64 || hid > 65536 || V < 1 || V > (1 << 30) || K < 1 || K > headloss::MAX_TOP) return 0;
    return headloss::lay_out(nullptr, M, hid, V, K, grad != 0).bytes;
}

int deer_lmhead_loss(const void* h, const void* w, const int32_t* targets, const float* row_weight, int M, int hid, int V, float* loss,
                     float* lse, float* target_logit, void* workspace, size_t workspace_bytes, void* stream) {
    return headloss::loss_call("deer_lmhead_loss", h, w, targets, nullptr, false, 1, 1.f, row_weight, M, hid, V, loss, lse, target_logit, workspace,
                               workspace_bytes, stream);
}

int deer_lmhead_loss_grad(const void* h, const void* w, const int32_t* targets, const float* row_weight, const float* grad_loss,
                          const float* lse, const float* target_logit, int M, int hid, int V, void* dh, void* dw, void* workspace,
                          size_t workspace_bytes, void* stream) {
    return headloss::grad_call("deer_lmhead_loss_grad", h, w, targets, nullptr, false, 1, 1.f, row_weight, grad_loss, lse, target_logit, M, hid, V, dh,
                               dw, workspace, workspace_bytes, stream);
}

int deer_lmhead_distill(const void* h, const void* w, const int32_t* ids, const float* teacher, int K, float temperature,
                        const float* row_weight, int M, int hid, int V, float* loss, float* lse, float* target_logit, void* workspace,
                        size_t workspace_bytes, void* stream) {
    return headloss::loss_call("deer_lmhead_distill", h, w, ids, teacher, true, K, temperature, row_weight, M, hid, V, loss, lse, target_logit,
                               workspace, workspace_bytes, stream);
}

int deer_lmhead_distill_grad(const void* h, const void* w, const int32_t* ids, const float* teacher, int K, float temperature,
                             const float* row_weight, const float* grad_loss, const float* lse, const float* target_logit, int M, int hid,
                             int V, void* dh, void* dw, void* workspace, size_t workspace_bytes, void* stream) {
    return headloss::grad_call("deer_lmhead_distill_grad", h, w, ids, teacher, true, K, temperature, row_weight, grad_loss, lse, target_logit, M, hid,
                               V, dh, dw, workspace, workspace_bytes, stream);
}

}  // extern "C"
