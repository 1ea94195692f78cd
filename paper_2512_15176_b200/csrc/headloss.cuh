// What the files of the LM head's losses share: the workspace of a call and the launcher of its products.
//
// A loss call works on the live rows only (rows that have a target and a weight other than 0), moved together at the
// start of the workspace; how many there are is known on the device alone, so every kernel reads it from `hdr`.
#pragma once

#include "common.cuh"

namespace headloss {

constexpr int TILE = 256;                  // rows of a product's tile: 128 in each block of a pair
constexpr int ONE_BLOCK = 128;             // up to this many rows STATS and GRAD work by single blocks: a pair would leave half of its
                                           // lanes empty and the products, not the reading of w, would bound the call
constexpr int STEP = 64;                   // contraction of one pipeline stage
constexpr int MAX_TOP = 128;               // entries of a row's list
constexpr int HDR_LIVE = 0, HDR_RANGES = 1, HDR_GAVE_UP = 2, HDR_SCALE = 3;
// Up to this many live rows G is kept as two bf16 terms: the second takes the places of the second block's rows in DH, idle
// then, and the contraction that DW's steps of 64 leave free.  DW sees rows [0, gap) and [gap, 2 gap), gap = low_term(live).
constexpr int TWO_TERMS = 128;
__host__ __device__ inline int low_term(int live) { return (live + 31) / 32 * 32; }

enum Product {
    STATS,      // z = h w^T, reduced to (max, sum exp) per row and vocabulary tile, and the listed tokens' z
    GRAD,       // the same z, as G = coef (exp(z / tau - lse) - t), bf16; coef is relative to the largest, HDR_SCALE
    DH,         // dh / scale = G w, fp32, added up over pieces and ranges
    DW          // dw = scale G^T h, bf16
};

// The arrays of one call, all in its workspace.
struct Space {
    int* hdr;                  // [4]
    int* slot;                 // [M]        place of a row among the live ones, -1: dead
    int* row;                  // [Mp]       the row at a place
    int* ids;                  // [K][Mp]    a live row's list by rising id, INT_MAX behind its end
    int* pos;                  // [K][Mp]    where an entry stood in the list            (loss)
    float* z;                  // [K][Mp]    a listed token's z as the tiles have it      (loss)
    float2* part;              // [Mp][tiles] (max z, sum exp((z - max) / tau))           (loss)
    float* coef;               // [Mp]       what a row's probabilities count            (gradient)
    float* lse2;               // [Mp]       lse log2(e)                                 (gradient)
    float* gval;               // [K][Mp]    G at the listed tokens                      (gradient)
    __nv_bfloat16* h;          // [Mp][hid]  live rows
    __nv_bfloat16* g;          // [Mp][piece]                                            (gradient)
    float* slab;               // [slab_tiles * 256][hid]  partial dh                    (gradient)
    size_t bytes;
    int Mp, pieces, piece, stats_n, grad_n, hid_n, slab_tiles;
};

// Sizes and offsets for M rows, lists of K; `base` may be null (sizes only).
Space lay_out(void* base, int M, int hid, int V, int K, bool grad);

struct ProductArgs {
    const int* hdr_in;
    int* hdr;
    int hid, V, v0, vn;        // vn columns of the vocabulary from v0 on
    int n;                     // columns of a tile
    int col_tiles;             // tiles along the columns (vocabulary or hid)
    int row_tiles;             // DW: tiles along the vocabulary
    int a_rows;                // rows of the 128-row operand one block loads (fewer than 128 only where M is)
    int Mp, K, tiles;
    int add;                   // DH: a piece behind the first
    float c2;                  // log2(e) / tau
    const int* ids;
    const int* pos;
    const int* row;
    const __nv_bfloat16* h;
    const __nv_bfloat16* w;
    float* target_logit;
    float* z;
    float2* part;
    const float* coef;
    const float* lse2;
    const float* gval;
    __nv_bfloat16* g;
    int g_pitch;
};

// Launches one product of the call: `piece` counts the pieces of the vocabulary (STATS: the whole of it).
int launch_product(Product what, const Space& s, const void* w, int M, int hid, int V, int K, int piece, float c2, float* target_logit,
                   void* dw, cudaStream_t st);

// Ranges that dh's contraction is cut into, so that mt x ht tiles of `steps` steps fill `pairs` pairs of blocks: the
// count with the shortest busiest pair, a range costing 24 steps beside its own (filling the pipeline, storing the
// tile).  At most `cap` tiles in all, for their partial sums' space, and ranges of 8 steps at least.
__host__ __device__ inline int dh_ranges(int mt, int ht, int steps, int pairs, int cap) {
    const uint32_t P = (uint32_t)pairs, tiles = (uint32_t)(mt * ht), all = (uint32_t)steps;
    int best = 1;
    uint64_t best_cost = (uint64_t)((tiles + P - 1) / P) * (all + 24);
    for (uint32_t s = 2; (int)s * mt <= cap && s * 8 <= all; ++s) {
        const uint64_t cost = (uint64_t)((tiles * s + P - 1) / P) * ((all + s - 1) / s + 24);
        if (cost < best_cost) {
            best_cost = cost;
            best = (int)s;
        }
    }
    return best;
}

}  // namespace headloss
