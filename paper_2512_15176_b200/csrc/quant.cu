// The row-wise quantisers of the 8-bit verifier layer -- residual + RMSNorm, a plain copy, the SiLU gate, each with
// e4m3 codes and one scale per 128 columns as output -- and the store of a step's kept rows into an 8-bit paged cache.
// All are one pass over their data.  With few rows a launch and two dependent memory round trips bound them (32 x 4096
// normalised 2.2 us, copied 1.3 us, the store of 16 blocks 3.2 us); with many the bytes, and close behind them the
// instructions (2048 x 4096 normalised 12.1 us = 4.9 TB/s; 512 x 12288 gated 8.2 us = 3.9 TB/s; four prompts' store
// 14.9 us = 3.8 TB/s).

#include "quant.cuh"

namespace quant {

using namespace sm100;

// 1 / rms of a row whose squares fp32 does not hold, from the squares of its values times `by`, a power of two.  By all threads
// of the block.  (Out of line, and from memory: with the row's registers kept for it 2048 x 4096 took 13.7 us, like this 12.2, without 11.8.)
__device__ __noinline__ float inverse_rms_of_far_row(const __nv_bfloat16* x, const __nv_bfloat16* residual, int hid, float eps, float by, float* part) {
    float ss = 0.f;
#pragma unroll 1
    for (int c = threadIdx.x; c < hid; c += blockDim.x) {
        const float v = (__bfloat162float(x[c]) + (residual ? __bfloat162float(residual[c]) : 0.f)) * by;
        ss = fmaf(v, v, ss);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    __syncthreads();                                               // (everyone has the first sum)
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = ss;
    __syncthreads();                                               // (and has read the row: `total` may be it)
    ss = 0.f;
#pragma unroll 1
    for (int w = 0; w < blockDim.x / 32; ++w) ss += part[w];
    return rsqrtf(ss / (float)hid + eps * by * by) * by;
}

// y = (x + residual) / rms * gamma per row.  A thread keeps its columns, CHUNKS pieces of 8, in registers between the two
// phases -- the sum of squares over the row, the codes of the sixteen-lane groups -- so a row is read once; with one or two
// pieces all loads, the gain's too, are on their way before the first value is used (more would not fit the registers).
template <int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS) rmsnorm_quant_kernel(const __nv_bfloat16* x, const __nv_bfloat16* residual,
                                                                const __nv_bfloat16* __restrict__ gamma, __nv_bfloat16* total,
                                                                uint8_t* __restrict__ codes, float* __restrict__ scales, int hid, float eps) {
    __shared__ float part[THREADS / 32];
    const size_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int groups = (hid + GROUP - 1) / GROUP;
    pdl_trigger();
    pdl_wait();
    constexpr bool EARLY = CHUNKS <= 2;
    uint4 xv[CHUNKS], rv[CHUNKS], gv[CHUNKS];
    auto piece = [&](const __nv_bfloat16* p, int c) {
        const int col = (c * THREADS + tid) * 8;
        return col < hid && p ? *reinterpret_cast<const uint4*>(p + col) : make_uint4(0, 0, 0, 0);
    };
    const __nv_bfloat16 *x_row = x + row * hid, *r_row = residual ? residual + row * hid : nullptr;
    if (EARLY) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            xv[c] = piece(x_row, c);
            rv[c] = piece(r_row, c);
            gv[c] = piece(gamma, c);
        }
    }
    V8 h[CHUNKS];
    uint64_t ss2 = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * THREADS + tid) * 8;
        if (!EARLY) {
            xv[c] = piece(x_row, c);
            rv[c] = piece(r_row, c);
        }
        h[c] = unpack8(xv[c]);
        if (residual) {
            const V8 r = unpack8(rv[c]);
#pragma unroll
            for (int j = 0; j < 4; ++j) h[c].p[j] = add2(h[c].p[j], r.p[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) ss2 = fma2(h[c].p[j], h[c].p[j], ss2);
    }
    float ss, ss_hi;
    unpack_f32x2(ss2, ss, ss_hi);
    ss += ss_hi;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (lane == 0) part[warp] = ss;
    __syncthreads();
    float tot = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) tot += part[w];
    float inv = rsqrtf(tot / (float)hid + eps);
    if (!(tot < 1e36f) || (tot < 1e-24f && eps < 1e-24f))
        inv = inverse_rms_of_far_row(x_row, r_row, hid, eps, tot < 1.f ? 1.26765060e30f : 7.88860905e-31f, part);       // 2^100, 2^-100
    const uint64_t inv2 = pack_f32x2(inv, inv);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int col = (c * THREADS + tid) * 8;
        if (c * THREADS * 8 >= hid) break;
        if (!EARLY) gv[c] = piece(gamma, c);
        if (total && col < hid) *reinterpret_cast<uint4*>(total + row * hid + col) = to_bf16(h[c]);
        const V8 g = unpack8(gv[c]);
#pragma unroll
        for (int j = 0; j < 4; ++j) h[c].p[j] = mul2(mul2(h[c].p[j], inv2), g.p[j]);
        const Divisor by(scale_of(max_mag_of<16>(col < hid ? max_mag(h[c]) : 0.f)));
        if (col < hid) {
            *reinterpret_cast<uint2*>(codes + row * hid + col) = codes8(h[c], by);
            if ((lane & 15) == 0) scales[row * groups + col / GROUP] = by.s;
        }
    }
}

// v / (1 + exp(-v)) * u for two values.
//
// 2^t with t = a multiple of log2(e) to twice fp32's precision: what the product's rounding left out (an fma has it exactly, and
// the part of log2(e) that fp32 does not hold is added) comes back as a factor 1 + rest * ln 2.
__device__ __forceinline__ uint64_t exp_of(uint64_t x, float l, float l_lo) {
    constexpr float LN2 = 0.693147182f;
    const uint64_t t = mul2(x, pack_f32x2(-l, -l));
    const uint64_t lack = fma2(x, pack_f32x2(l_lo, l_lo), fma2(x, pack_f32x2(l, l), t));     // t - (-x log2(e))
    float t0, t1, e0, e1;
    unpack_f32x2(t, t0, t1);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(t0));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(t1));
    const uint64_t e = pack_f32x2(e0, e1);
    return fma2(mul2(e, pack_f32x2(-LN2, -LN2)), lack, e);
}
// -n / d by an approximate reciprocal, corrected once by its remainder.
__device__ __forceinline__ uint64_t neg_quotient(uint64_t n, uint64_t d) {
    float d0, d1, r0, r1;
    unpack_f32x2(d, d0, d1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(-d0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(-d1));
    const uint64_t neg_r = pack_f32x2(r0, r1), neg_q = mul2(n, neg_r);
    return fma2(fma2(neg_q, d, n), neg_r, neg_q);
}
// Gates below GATE_NEAR in magnitude: exp(-v) is at most 2^93, and nothing on the way leaves fp32's normal range.  Off by about
// what the last two products round away, as close as the same formula in fp32 with a full exp and a division (512 x 12288:
// 10.7 us with those, 8.2 like this, 9.0 with the form below for all).
constexpr float GATE_NEAR = 64.f;
__device__ __forceinline__ uint64_t gate_near2(uint64_t v, uint64_t neg_u) {
    const uint64_t e = exp_of(v, 1.44269502f, 1.92596299e-8f);
    return mul2(neg_quotient(v, add2(e, pack_f32x2(1.f, 1.f))), neg_u);
}
// Gates of any size.  With w = exp(-|v|) the quotient is v / (1 + w) or, below zero, v w / (1 + w) -- the larger of v and v w over
// 1 + w -- so nothing overflows; and w is multiplied in as two factors exp(-|v| / 2), so that the quotient leaves fp32 gradually,
// as a number does, and not where w would.  |v| stops at 400, where the factors are 0, so that t stays finite.  -inf gives a NaN.
__device__ __forceinline__ uint64_t gate_any2(uint64_t v, uint64_t neg_u) {
    float v0, v1, n0, n1;
    unpack_f32x2(v, v0, v1);
    const uint64_t h = exp_of(pack_f32x2(fminf(fabsf(v0), 400.f), fminf(fabsf(v1), 400.f)), 0.72134751f, 9.62981496e-9f);
    unpack_f32x2(mul2(mul2(v, h), h), n0, n1);
    return mul2(neg_quotient(pack_f32x2(fmaxf(v0, n0), fmaxf(v1, n1)), fma2(h, h, pack_f32x2(1.f, 1.f))), neg_u);
}

// Sixteen lanes per group of 128 columns, groups of all rows laid end to end.
template <bool GATED>
__global__ void __launch_bounds__(256) quantize_kernel(const __nv_bfloat16* __restrict__ x, uint8_t* __restrict__ codes,
                                                       float* __restrict__ scales, int M, int K) {
    const int groups = (K + GROUP - 1) / GROUP;
    const size_t item = (size_t)blockIdx.x * 16 + (threadIdx.x >> 4);          // group index over all rows
    const size_t row = item <= 0xffffffffu ? (uint32_t)item / (uint32_t)groups : item / (size_t)groups;   // (32 bits where they do)
    const int g = (int)(item - row * (size_t)groups);
    const int col = g * GROUP + (threadIdx.x & 15) * 8;
    pdl_trigger();
    pdl_wait();
    const bool on = row < (size_t)M && col < K;
    V8 v = {};
    if (on) {
        const __nv_bfloat16* src = x + row * (size_t)(GATED ? 2 * (size_t)K : K) + col;
        const uint4 a = *reinterpret_cast<const uint4*>(src);
        v = unpack8(a);
        if (GATED) {
            uint4 b = *reinterpret_cast<const uint4*>(src + K);
            b.x ^= 0x80008000u;
            b.y ^= 0x80008000u;
            b.z ^= 0x80008000u;
            b.w ^= 0x80008000u;
            const V8 neg_u = unpack8(b);
            if (max_mag(v) < GATE_NEAR) {                  // (not for a NaN)
#pragma unroll
                for (int j = 0; j < 4; ++j) v.p[j] = gate_near2(v.p[j], neg_u.p[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v.p[j] = gate_any2(v.p[j], neg_u.p[j]);
            }
        }
    }
    const Divisor by(scale_of(max_mag_of<16>(max_mag(v))));
    if (on) {
        *reinterpret_cast<uint2*>(codes + row * K + col) = codes8(v, by);
        if ((threadIdx.x & 15) == 0) scales[row * groups + g] = by.s;
    }
}

// ---- the store into an 8-bit paged cache -----------------------------------------------------------------------
// One thread block per (run of PP pages that the new rows can touch, KV head, sequence), its first half for K, its second
// for V; a thread holds 16 dims of one token, and the next page's while it works on one.  Page 0 is the one that seq_len
// stands in; its block alone reads tail rows, and it also writes the new ones, last, because the page behind the last full
// one may share their places (page mod 3).
template <int D>
__global__ void __launch_bounds__(2 * D) kv_store_kernel(deer_kv_desc kv, deer_kv_quant_desc q, const int32_t* __restrict__ seq_ids,
                                                         const __nv_bfloat16* __restrict__ k_rows, const __nv_bfloat16* __restrict__ v_rows,
                                                         const int32_t* __restrict__ keep, int k, int pages_per_block) {
    constexpr int PER_ROW = D / 16;                       // threads of a token
    __shared__ float part[2][2 * D / 32];
    const int tid = threadIdx.x;
    const bool is_v = tid >= D;
    const int t16 = (tid % D) / PER_ROW, col = (tid % PER_ROW) * 16;
    const int Hkv = kv.n_kv_heads;
    const int h = (int)(blockIdx.x % (unsigned)Hkv), run = (int)(blockIdx.x / (unsigned)Hkv), b = blockIdx.y;   // the heads of a token are neighbours in memory
    pdl_trigger();
    pdl_wait();
    const int s = seq_ids[b];
    const int kp = keep ? min(max(keep[b], 0), k) : k;
    if (s < 0 || s >= kv.max_seqs) {
        if (tid == 0) deer_report(kv.status, DEER_ERR_INVALID_ARG);
        return;
    }
    const int n = kv.seq_len[s];
    if (n < 0 || n / DEER_PAGE_SIZE > kv.max_pages) {
        if (tid == 0) deer_report(kv.status, DEER_ERR_INVALID_ARG);
        return;
    }
    if (kp == 0) return;
    const int end = n + kp, full_pages = end / DEER_PAGE_SIZE;
    const __nv_bfloat16* rows = (is_v ? v_rows : k_rows) + (size_t)b * k * Hkv * D;
    __nv_bfloat16* tail = static_cast<__nv_bfloat16*>(is_v ? q.v_tail : q.k_tail) + ((size_t)s * Hkv + h) * DEER_TAIL_ROWS * D;
    uint8_t* pool = static_cast<uint8_t*>(is_v ? kv.v_pool : kv.k_pool);
    const int first = n / DEER_PAGE_SIZE + run * pages_per_block, last = min(first + pages_per_block, full_pages);
    uint4 next[2];
    int pg_next = -1;
    auto bring = [&](int page) {                          // this thread's token of a full page, and the page's number
        const int t = page * DEER_PAGE_SIZE + t16;
        const uint4* src = reinterpret_cast<const uint4*>(t < n ? tail + (size_t)(t % DEER_TAIL_ROWS) * D + col
                                                                : rows + ((size_t)(t - n) * Hkv + h) * D + col);
        next[0] = src[0];
        next[1] = src[1];
        pg_next = page < kv.max_pages ? kv.page_table[(size_t)s * kv.max_pages + page] : -1;
    };
    if (first < last) bring(first);
    for (int page = first; page < last; ++page) {
        const V8 v0 = unpack8(next[0]), v1 = unpack8(next[1]);
        const int pg = pg_next;
        if (page + 1 < last) bring(page + 1);
        const float mine = max_mag_of<32>(max_mag(v1, max_mag(v0)));
        if ((tid & 31) == 0) part[page & 1][tid >> 5] = mine;
        __syncthreads();                                  // (the first time also: the tail rows are in registers)
        float m = 0.f;
#pragma unroll
        for (int w = 0; w < D / 32; w += 2) m = max_mag(m, part[page & 1][(is_v ? D / 32 : 0) + w], part[page & 1][(is_v ? D / 32 : 0) + w + 1]);
        const Divisor by(scale_of(m));
        if (pg < 0 || pg >= kv.num_pages) {
            if (tid == 0) deer_report(kv.status, DEER_ERR_BAD_PAGE);
            continue;
        }
        const size_t slab = (size_t)pg * Hkv + h;
        const uint2 lo = codes8(v0, by), hi = codes8(v1, by);
        *reinterpret_cast<uint4*>(pool + (slab * DEER_PAGE_SIZE + t16) * D + col) = make_uint4(lo.x, lo.y, hi.x, hi.y);
        if (tid % D == 0) (is_v ? q.v_scale : q.k_scale)[slab] = by.s;
    }
    if (run == 0) {                                       // the rows behind the last full page
        const int tt = full_pages * DEER_PAGE_SIZE + t16;
        if (tt >= n && tt < end) {
            const uint4* src = reinterpret_cast<const uint4*>(rows + ((size_t)(tt - n) * Hkv + h) * D + col);
            uint4* dst = reinterpret_cast<uint4*>(tail + (size_t)(tt % DEER_TAIL_ROWS) * D + col);
            dst[0] = src[0];
            dst[1] = src[1];
        }
    }
}

}  // namespace quant

using namespace quant;

extern "C" int deer_rmsnorm_quant(const void* x, const void* residual, const void* gamma, void* total, void* codes, float* scales,
                                  int M, int hid, float eps, void* stream) {
    DEER_CHECK_ARG(x && gamma && codes && scales, DEER_ERR_INVALID_ARG, "deer_rmsnorm_quant: null argument");
    DEER_CHECK_ARG(deer_aligned16(x) && deer_aligned16(residual) && deer_aligned16(gamma) && deer_aligned16(total) && deer_aligned16(codes) &&
                       deer_aligned4(scales),
                   DEER_ERR_INVALID_ARG, "deer_rmsnorm_quant: pointers must be 16-byte aligned (scales: 4)");
    DEER_CHECK_ARG(M >= 0, DEER_ERR_INVALID_ARG, "deer_rmsnorm_quant: M must be >= 0");
    DEER_CHECK_ARG(hid >= 16 && hid % 16 == 0 && hid <= 65536, DEER_ERR_UNSUPPORTED,
                   "deer_rmsnorm_quant: hid must be a multiple of 16 in [16, 65536]");
    if (M == 0) return DEER_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto run = [&](auto kernel, int threads) {
        return launch_pdl(kernel, dim3((unsigned)M), dim3((unsigned)threads), 0, st, static_cast<const __nv_bfloat16*>(x),
                          static_cast<const __nv_bfloat16*>(residual), static_cast<const __nv_bfloat16*>(gamma),
                          static_cast<__nv_bfloat16*>(total), static_cast<uint8_t*>(codes), scales, hid, eps);
    };
    if (hid <= 1024) DEER_CUDA(run(rmsnorm_quant_kernel<128, 1>, 128));
    else if (hid <= 2048) DEER_CUDA(run(rmsnorm_quant_kernel<256, 1>, 256));
    else if (hid <= 4096) DEER_CUDA(run(rmsnorm_quant_kernel<256, 2>, 256));
    else if (hid <= 8192) DEER_CUDA(run(rmsnorm_quant_kernel<512, 2>, 512));
    else if (hid <= 16384) DEER_CUDA(run(rmsnorm_quant_kernel<512, 4>, 512));
    else DEER_CUDA(run(rmsnorm_quant_kernel<1024, 8>, 1024));      // (64 values a thread spill: 512 x 20000 33.8 us, 512 x 16384 16.0)
    return DEER_OK;
}

extern "C" int deer_quantize(const void* x, int gated, void* codes, float* scales, int M, int K, void* stream) {
    DEER_CHECK_ARG(x && codes && scales, DEER_ERR_INVALID_ARG, "deer_quantize: null argument");
    DEER_CHECK_ARG(deer_aligned16(x) && deer_aligned16(codes) && deer_aligned4(scales), DEER_ERR_INVALID_ARG,
                   "deer_quantize: pointers must be 16-byte aligned (scales: 4)");
    DEER_CHECK_ARG(M >= 0, DEER_ERR_INVALID_ARG, "deer_quantize: M must be >= 0");
    DEER_CHECK_ARG(K >= 16 && K % 16 == 0, DEER_ERR_UNSUPPORTED, "deer_quantize: K must be a multiple of 16");
    if (M == 0) return DEER_OK;
    const long long items = (long long)M * ((K + GROUP - 1) / GROUP), blocks = (items + 15) / 16;
    DEER_CHECK_ARG(blocks <= 0x7fffffffLL, DEER_ERR_UNSUPPORTED, "deer_quantize: too many rows");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    DEER_CUDA(launch_pdl(gated ? quantize_kernel<true> : quantize_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st,
                         static_cast<const __nv_bfloat16*>(x), static_cast<uint8_t*>(codes), scales, M, K));
    return DEER_OK;
}

extern "C" int deer_kv_store(deer_kv* kv, const int32_t* seq_ids, const void* k_rows, const void* v_rows, const int32_t* keep, int B, int k,
                             void* stream) {
    DEER_CHECK_ARG(kv && seq_ids && k_rows && v_rows, DEER_ERR_INVALID_ARG, "deer_kv_store: null argument");
    DEER_CHECK_ARG(kv->quant, DEER_ERR_UNSUPPORTED, "deer_kv_store: the cache holds bf16 pools (deer_block_attn appends to those)");
    DEER_CHECK_ARG(deer_aligned16(k_rows) && deer_aligned16(v_rows), DEER_ERR_INVALID_ARG, "deer_kv_store: pointers must be 16-byte aligned");
    DEER_CHECK_ARG(B >= 0 && B <= 65535, DEER_ERR_UNSUPPORTED, "deer_kv_store: B must be in [0, 65535]");
    DEER_CHECK_ARG(k >= 0 && k <= (1 << 24), DEER_ERR_UNSUPPORTED, "deer_kv_store: k must be in [0, 2^24]");
    DEER_CHECK_ARG(kv->d.n_kv_heads <= 65535, DEER_ERR_UNSUPPORTED, "deer_kv_store: too many KV heads");
    if (B == 0 || k == 0) return DEER_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // k rows that start anywhere in a page fill at most (15 + k) / 16 pages to their end (at least one: k >= 1).  A page per
    // block while all blocks fit the SMs at once; a block starts with three loads that wait for one another, so long
    // prompts give it up to eight (4 prompts of 4096 rows, a random part of each kept, 8 heads of 128: 1 page 24.1, 2 18.8,
    // 8 15.7, 16 21.5 us, the last because blocks behind the kept rows have nothing to do).
    const long long pages = (15 + k) / DEER_PAGE_SIZE, blocks = pages * kv->d.n_kv_heads * B;
    const long long rounds = (blocks + 4LL * deer_sm_count() - 1) / (4LL * deer_sm_count());
    const int per = rounds > 8 ? 8 : (int)rounds;
    const long long runs = (pages + per - 1) / per * kv->d.n_kv_heads;
    DEER_CHECK_ARG(runs <= 0x7fffffffLL, DEER_ERR_UNSUPPORTED, "deer_kv_store: too many rows");
    const dim3 grid((unsigned)runs, (unsigned)B);
    auto run = [&](auto kernel, int threads) {
        return launch_pdl(kernel, grid, dim3((unsigned)threads), 0, st, kv->d, kv->q, seq_ids, static_cast<const __nv_bfloat16*>(k_rows),
                          static_cast<const __nv_bfloat16*>(v_rows), keep, k, per);
    };
    if (kv->d.head_dim == 128) DEER_CUDA(run(kv_store_kernel<128>, 256));
    else DEER_CUDA(run(kv_store_kernel<64>, 128));
    return DEER_OK;
}
