// Shared declarations of the block-attention kernels over an 8-bit paged cache.
#pragma once

#include "attn.cuh"
#include "quant.cuh"

namespace attnq {

using attn::LOG2E;
constexpr int PAGE = DEER_PAGE_SIZE;

struct Params {
    deer_kv_desc kv;
    deer_kv_quant_desc kq;
    const int32_t* seq_ids;
    const int32_t* row_state;  // [B][k] or null: 1 masked, 0 decoded, -1 absent (bidirectional mask only)
    const __nv_bfloat16* q;
    const __nv_bfloat16* k_blk;
    const __nv_bfloat16* v_blk;
    __nv_bfloat16* out;
    float* part_o;             // [parts][B*k*Hq][D]  normalised partial outputs, one per cluster of context chunks
    float* part_lse;           // [parts][B*k*Hq]     their log2-sum-exp
    int B, k, Hq, G, mask;
    int max_seq_len;
    float scale_log2;
    int row_tiles;             // tiles of 16 query rows (block row major, then query head) per KV head
    int chunk_pages;           // full pages per context chunk
    int cluster;               // chunks (thread blocks) that meet in a cluster
};

constexpr int ROWS_SMALL = 16;   // query rows of a warp-level tile

// tcgen05 variant (attn_quant_umma.cu).
bool use_umma(int B, int D, int k, int Hq, int Hkv, int max_seq_len, float scale);
size_t umma_workspace_bytes(int B, int k, int Hq, int Hkv, int max_seq_len);
int launch_umma(const Params& p, void* workspace, cudaStream_t st);

#ifdef __CUDACC__
// Two e4m3 codes (the low or the high half of w) as fp16, exactly.
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) {
    uint32_t r;
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 %0, l;}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) {
    uint32_t r;
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 %0, h;}" : "=r"(r) : "r"(w));
    return r;
}
// Sequence of index b in the call: its cache slot and committed length; false (and the status word) if it cannot be used.
__device__ __forceinline__ bool sequence_of(const Params& p, int b, int* s, int* n, bool report) {
    *s = p.seq_ids[b];
    *n = -1;
    if (*s >= 0 && *s < p.kv.max_seqs) *n = p.kv.seq_len[*s];
    if (*n >= 0 && *n <= p.max_seq_len) return true;
    if (report) deer_report(p.kv.status, DEER_ERR_INVALID_ARG);
    return false;
}
__device__ __forceinline__ int chunks_of(const Params& p, int n) {
    const int full = n / PAGE;
    return full > p.chunk_pages ? (full + p.chunk_pages - 1) / p.chunk_pages : 1;
}
#endif

}  // namespace attnq
