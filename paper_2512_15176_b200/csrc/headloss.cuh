// What the files of the LM head's losses share: the workspace of a call and the launcher of its products.
//
// A loss call works on the live rows only (rows that have a target and a weight other than 0), moved together at the
// start of the workspace; how many there are is known on the device alone, so every kernel reads it from `hdr`.
#pragma once

#include <math.h>

#include "common.cuh"

namespace headloss {

constexpr int STEP = 64;                   // contraction of one pipeline stage
constexpr int TILE = 256;                  // rows of a product's tile: 128 in each block of a pair
constexpr int ONE_BLOCK = 128;             // up to this many rows STATS and GRAD work by single blocks: a pair would leave half of its
                                           // lanes empty and the products, not the reading of w, would bound the call
constexpr int SHORT = 8;                   // lists of up to so many entries are searched as they are: with them single blocks of
                                           // STATS take the call's rows themselves (a dead one costs nothing in a tile that is
                                           // not full), which saves a launch
inline bool takes_rows_as_they_are(int M, int K) { return M <= ONE_BLOCK && K <= SHORT; }
constexpr int MAX_TOP = 128;               // entries of a row's list
constexpr int STATS_SHARE = 2;             // warps that share a tile's columns in STATS: partial sums a row has of a tile
constexpr int HDR_LIVE = 0, HDR_RANGES = 1, HDR_GAVE_UP = 2, HDR_SCALE = 3, HDR_FACTOR = 4;
// Up to this many live rows G is kept as two bf16 terms, rows [0, low) and [low, 2 low) with low = low_term(live).  In dh's
// product the second takes the places of the second block's rows, idle then.  In dw's it lengthens the contraction: that
// covers its first 128 places, all of both terms up to 64 live rows, and beyond them (where rows' errors begin to be
// independent) what is left of its second step.  With all of both terms up to 128 rows the gradients take 401 us instead of 391
// (77 rows x 151936 x 2048) to 607 instead of 566 (128 rows, hid 2688); dw's error at 77 rows is 1.96e-3 so, its own rounding 1.66e-3.
constexpr int TWO_TERMS = 128, DW_TERMS = 64;
__host__ __device__ inline int low_term(int live) { return (live + 31) / 32 * 32; }
// Steps of dw's contraction.
__host__ __device__ inline int dw_contraction(int live) {
    if (live > TWO_TERMS) return (live + STEP - 1) / STEP;
    const int rows = 2 * low_term(live) < 2 * DW_TERMS ? 2 * low_term(live) : 2 * DW_TERMS;
    return (rows + STEP - 1) / STEP;
}

enum Product {
    STATS,      // z = h w^T, reduced to (max, sum exp) per row and vocabulary tile, and the listed tokens' z
    GRAD,       // the same z, as G = coef (exp(z / tau - lse) - t), bf16; coef is relative to HDR_SCALE
    BACK        // dh / scale = G w, fp32, added up over pieces and ranges, and dw = scale G^T h, bf16
};

// The arrays of one call, all in its workspace.
struct Space {
    int* hdr;                  // [5]
    int* slot;                 // [M]        place of a row among the live ones, -1: dead
    int* row;                  // [Mp]       the row at a place
    int* ids;                  // [Mp][K]    a live row's list by rising id, INT_MAX behind its end
    uint8_t* first;            // [Mp][tiles] entries of a row's list in front of a tile of STATS or GRAD
    int* place;                // [Mp][K]    an entry's place among the rising ids, -1: a token listed before    (loss)
    float* z;                  // [Mp][K]    by rising id (as they are: by the list): the token's z as the tiles have it  (loss)
    float2* part;              // [Mp][tiles] (m, sum 2^(z log2(e) / tau - m))            (loss)
    float* coef;               // [Mp]       what a row's probabilities count            (gradient)
    float* lse2;               // [Mp]       lse log2(e)                                 (gradient)
    float* rounding;           // [blocks][32] squares of what rounding takes of G at the listed tokens, by factor   (gradient)
    float* gval;               // [Mp][K]    G at the listed tokens                      (gradient)
    __nv_bfloat16* h;          // [Mp][hid]  live rows
    __nv_bfloat16* g;          // [Mp][piece]                                            (gradient)
    float* slab;               // [slab_tiles * 256][hid]  partial dh                    (gradient)
    size_t bytes;
    int first_pitch, piece_tiles;      // tiles of a row, of a piece
    int Mp, pieces, piece, stats_n, grad_n, hid_n, slab_tiles;
};

// Sizes and offsets for M rows, lists of K; `base` may be null (sizes only).
Space lay_out(void* base, int M, int hid, int V, int K, bool grad);

struct ProductArgs {
    int M;
    int as_is;                 // STATS: the call's rows and lists, not the live ones moved together
    const int* list;           // the call's lists and row weights
    const float* weight;
    const int* hdr_in;
    int* hdr;
    int hid, V, v0, vn;        // vn columns of the vocabulary from v0 on
    int n;                     // columns of a tile
    int col_tiles;             // tiles along the columns (vocabulary or hid)
    int want_dh, row_tiles;    // BACK: whether dh is asked for; dw's tiles along the vocabulary (0: not asked for)
    int a_rows;                // rows of the 128-row operand one block loads (fewer than 128 only where M is)
    int K, tiles;
    int add;                   // BACK: a piece behind the first
    float c2, c2_low;          // tile_scale_of tau
    const int* ids;
    const int* row;
    const __nv_bfloat16* h;
    const __nv_bfloat16* w;
    float* target_logit;
    float* z;
    float2* part;
    const float* coef;
    const float* lse2;
    const float* gval;
    const uint8_t* first;
    int first_pitch, first_tile;
    __nv_bfloat16* g;
    __nv_bfloat16* dw;
    int g_pitch;
};

// Launches one product of the call: `piece` counts the pieces of the vocabulary (STATS: the whole of it).
// h, list, weight: the call's own; dh and dw: what is asked for (BACK).
int launch_product(Product what, const Space& s, const void* h, const void* w, const int* list, const float* weight, int M, int hid, int V, int K,
                   int piece, float tau, float* target_logit, bool want_dh, void* dw, cudaStream_t st);

// log2(e) / tau as two fp32 terms, both above 0 (a z of -inf stays one).
inline void scale_of(double tau, float& c2, float& c2_low) {
    const double c = 1.4426950408889634 / tau;
    c2 = (float)c;
    if (c2 >= c) c2 = nextafterf(c2, 0.f);
    c2_low = (float)(c - c2);
}
// The same for a z that comes from the tensor cores, whose accumulation rounds towards zero: measured against 64 bits from hid 64
// to 65536, each of its steps of 16 leaves z short by 1.5e-8 to 1.7e-8 of itself where the products' signs mix (at hid 2048 z of a
// row's whole vocabulary is 1.8e-6 of itself too near to zero), by 1.3e-8 to 2.2e-8 where z stands out, and where all products have
// one sign by 2.5e-8 (hid 512) to 9.2e-8 (hid 65536).  1.5e-8, the mean of the ordinary case and about the least of all, is given
// back: it takes lse's error at hid 2048 to that of an fp32 product (6.7e-6 and 6.2e-6 for logits of 20) and overshoots nowhere
// by more than 6e-9 a step (hid 64, sums that rise and fall again).
inline void tile_scale_of(double tau, int hid, float& c2, float& c2_low) { scale_of(tau / (1.0 + 1.5e-8 * (hid / 16)), c2, c2_low); }

__device__ __forceinline__ bool is_live(const int* list, const float* weight, int K, int m) {
    const int id = list[(size_t)m * K];
    const float a = weight ? weight[m] : 1.f;
    return id >= 0 && a != 0.f;
}

// What a tile of dh's and of dw's product costs, in steps of its contraction: filling the pipeline and storing the tile
// cost eight steps beside them, and a short contraction waits for the tile before it to be stored.
__host__ __device__ inline int dh_tile_cost(int steps, int ranges) { return (steps + ranges - 1) / ranges + 8; }
__host__ __device__ inline int dw_tile_cost(int steps) { return steps > 7 ? steps : 7; }

}  // namespace headloss
