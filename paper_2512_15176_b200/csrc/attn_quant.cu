// Block attention against an 8-bit paged cache (Section 3.2's parallel pass with the KV stream at half its bytes).
//
// The keys of a sequence with n committed tokens: floor(n / 16) full pages of e4m3 codes with one scale per page and
// head, n mod 16 tail rows in bf16, and the block's own k rows in bf16.
//
// Warp-level kernel.  A page of one KV head is 16 tokens: exactly one contraction step of the second product and two
// column tiles of the first.  A warp takes whole pages: each lane copies, pages ahead and asynchronously, the
// 16-byte pieces of K and V that it will use to shared memory of its own -- the pieces are laid out so that they ARE the
// operand fragments (the contraction index of q . k and the column index of p v may be permuted freely, as long as the
// other side is permuted alike), so the lanes exchange nothing -- and the codes become fp16 exactly.  The page's K scale multiplies the 16 scores; its V scale
// multiplies the page's product before it joins the fp32 sums, so scales of any size work.  Queries are brought to
// fp16 by a power of two per row (exact to 2^-24 of the row's largest), probabilities are taken against their page's maximum, at
// most 2^12, and keep fp16's 11 bits down to 2^-26 of it; the page's own weight joins its product in fp32.  The warps of a block take pages in turn with running maxima of their
// own, and meet in shared memory at the end.  A context is cut into chunks over thread blocks; up to eight of them form
// a cluster and meet in its shared memory, and where a context has more a second kernel joins the clusters' parts.
//
// What bounds it: latencies in short contexts (one token, 32 query and 8 KV heads, over 1003: 8.0 us, two pages per warp,
// most of it the chain length -> page number -> page -> products -> meeting in the cluster), the instructions of a page
// (about 400 a warp, and their latencies) in long ones: 16 x 4096 tokens 44.4 us = 3.0 TB/s, one token over 32768 29.5 us; and, for many rows over heads of 64, that each 16 of them read the pages again (16 x 32 rows,
// 32 query and 4 KV heads of 64, 2048 to 16384 tokens 305 us).

#include <cuda_fp16.h>

#include "attn_quant.cuh"
#include "sm100.cuh"

namespace attnq {

constexpr int ROWS = ROWS_SMALL;
constexpr int WARPS = 4;
constexpr int CLUSTER_MAX = 8;                 // the portable limit
constexpr int RESIDENT = 2;                    // blocks per SM
constexpr int STAGES = 4;                      // pages of a warp under way or in use

// Shared memory of a block: a ring of pages per warp, then (over it) the warps' results.
template <int D>
struct Smem {
    static constexpr int LANE = D / 64 * 32 + D / 32 * 16;       // bytes of K and V of a page that a lane uses
    static constexpr int STAGE = LANE * 32 + 16;                 // and the two scales
    static constexpr int RING = WARPS * STAGES * STAGE;
    static constexpr int QD = D / 4 + 1;       // a lane's dims of a row, one word apart from the next lane's: no two lanes share a bank
    static constexpr int RESULTS = (WARPS * ROWS * 4 * QD + 2 * WARPS * ROWS + ROWS) * 4;
    static constexpr int BYTES = RING > RESULTS ? RING : RESULTS;
};
constexpr float P_BIAS = 12.f;                 // probabilities are held as 2^12 p

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// 2^x of differences to a maximum; 0 below 2^-126.
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}

// Lane (g8, t4) = (lane / 4, lane % 4).  Contraction step (hc, w) of q . k: this lane's four contraction indices are
// the dims hc * 64 + t4 * 16 + w * 4 + 0..3.  Column tile j of p v: column g8 is dim g8 * (D / 8) + j, so that this
// lane's accumulators are the dims t4 * (D / 4) + 0 .. D / 4 - 1 of rows g8 and g8 + 8.
template <int D>
__global__ void __launch_bounds__(WARPS * 32, RESIDENT) attn_quant_kernel(const Params p) {
    constexpr int HC = D / 64;                 // 16-byte pieces of a key row per lane
    constexpr int ND = D / 8;                  // column tiles of the output
    constexpr int VW = D / 32;                 // 32-bit words of a value row per lane (16-byte or 8-byte piece)
    constexpr int QD = Smem<D>::QD;
    extern __shared__ __align__(16) unsigned char smem[];
    float (*s_o)[ROWS][4 * QD] = reinterpret_cast<float (*)[ROWS][4 * QD]>(smem);
    float (*s_m)[ROWS] = reinterpret_cast<float (*)[ROWS]>(s_o + WARPS), (*s_l)[ROWS] = s_m + WARPS;
    float* s_lse = s_l[WARPS];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, t4 = lane & 3;
    const int Hkv = p.kv.n_kv_heads;
    const int c = blockIdx.x, kvh = blockIdx.y / p.row_tiles, rt = blockIdx.y % p.row_tiles, b = blockIdx.z;
    pdl_trigger();
    pdl_wait();
    const int page_lo = c * p.chunk_pages;
    // the sequence's length and the numbers of this warp's pages (lane j: its j-th one) are on their way together
    const int slot_id = p.seq_ids[b];
    const bool known = slot_id >= 0 && slot_id < p.kv.max_seqs;
    const int32_t* pt_row = p.kv.page_table + (size_t)(known ? slot_id : 0) * p.kv.max_pages;
    auto page_numbers = [&](int j0) {
        const int page = page_lo + warp + (j0 + lane) * WARPS;
        return page < p.kv.max_pages ? __ldcg(pt_row + page) : -1;
    };
    int pgs = page_numbers(0);
    int s, n;
    if (!sequence_of(p, b, &s, &n, c == 0 && blockIdx.y == 0 && tid == 0)) return;
    const int n_chunks = chunks_of(p, n);
    if (c / p.cluster * p.cluster >= n_chunks) return;         // none of the cluster's blocks has a chunk
    const int R = p.G * p.k;
    const bool busy = c < n_chunks;
    const int n_pages = busy ? max(0, (min(n / PAGE - page_lo, p.chunk_pages) - warp + WARPS - 1) / WARPS) : 0;   // this warp's
    const int n_tail = n % PAGE;

    // Page j of this warp into its ring: the next call's page numbers are fetched with every 32nd.
    int pgs_next = n_pages > 32 ? page_numbers(32) : -1;
    auto bring = [&](int j) {
        if (j > 0 && (j & 31) == 0) {
            pgs = pgs_next;
            pgs_next = n_pages > j + 32 ? page_numbers(j + 32) : -1;
        }
        int pg = __shfl_sync(0xffffffffu, pgs, j & 31);
        if (pg < 0 || pg >= p.kv.num_pages) {
            if (lane == 0) deer_report(p.kv.status, DEER_ERR_BAD_PAGE);
            pg = 0;                                            // inside the pool; the status word flags the result
        }
        const size_t slab = (size_t)pg * Hkv + kvh;
        const uint8_t* kp = static_cast<const uint8_t*>(p.kv.k_pool) + slab * PAGE * D;
        const uint8_t* vp = static_cast<const uint8_t*>(p.kv.v_pool) + slab * PAGE * D;
        const uint32_t st = smem_u32(smem + (warp * STAGES + j % STAGES) * Smem<D>::STAGE);
#pragma unroll
        for (int t = 0; t < 2; ++t)            // keys g8, g8 + 8 of the page
#pragma unroll
            for (int hc = 0; hc < HC; ++hc) cp_async16(st + ((t * HC + hc) * 32 + lane) * 16, kp + (t * 8 + g8) * D + hc * 64 + t4 * 16, 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {          // values 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9
            const uint8_t* src = vp + (2 * t4 + (e & 1) + (e >> 1) * 8) * D + g8 * (D / 8);
            const uint32_t dst = st + 2 * HC * 512 + (e * 32 + lane) * (VW * 4);
            if (D == 128) cp_async16(dst, src, 16);
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(dst), "l"(src));
        }
        if (lane < 2) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(st + Smem<D>::LANE * 32 + lane * 4), "l"((lane ? p.kq.v_scale : p.kq.k_scale) + slab));
    };
    if (n_pages > 0) bring(0);
    if (n_pages > 1) bring(1);
    cp_async_commit();

    uint32_t present, decoded;
    attn::row_state_sets(p.row_state, b, p.k, lane, &present, &decoded);

    // ---- this lane's two query rows ----
    int row[2], blk_row[2];
    const __nv_bfloat16* q_row[2];
    uint32_t cols[2];                                          // block rows that the row sees
    bool live[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        row[u] = rt * ROWS + g8 + u * 8;
        const int rr = min(row[u], R - 1);
        blk_row[u] = rr / p.G;
        const int st = p.row_state ? p.row_state[(size_t)b * p.k + blk_row[u]] : 1;
        live[u] = row[u] < R && st >= 0;
        cols[u] = attn::visible_rows(p.mask, blk_row[u], st, present, decoded);
        q_row[u] = p.q + ((size_t)(b * p.k + blk_row[u]) * p.Hq + kvh * p.G + rr % p.G) * D;
    }
    uint32_t qf[HC * 4][4];
    float f_row[2];                                            // scale * log2(e) * the power of two taken out of the row
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        float qv[HC][16];
        uint32_t m = 0;
#pragma unroll
        for (int hc = 0; hc < HC; ++hc) {
            quant::load_bf16x16(q_row[u] + hc * 64 + t4 * 16, qv[hc]);
            m = max(m, quant::amax16(qv[hc]));
        }
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        // 2^-e with 2^e <= max < 2^(e+1); a row with a NaN or an infinity stays as it is (and gives NaN)
        int e = (int)(m >> 23) - 127;
        if (e == 128) e = 0;
        const float down = __uint_as_float((uint32_t)max(127 - e, 1) << 23);
        f_row[u] = p.scale_log2 / down;
#pragma unroll
        for (int hc = 0; hc < HC; ++hc)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                qf[hc * 4 + w][u] = pack_f16(qv[hc][w * 4] * down, qv[hc][w * 4 + 1] * down);
                qf[hc * 4 + w][2 + u] = pack_f16(qv[hc][w * 4 + 2] * down, qv[hc][w * 4 + 3] * down);
            }
    }

    float o[ND][4];
#pragma unroll
    for (int j = 0; j < ND; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};     // l: this lane's columns only, until the end

    // Scores (N groups of two column tiles of 8 keys each) in the log2 domain -> probabilities against their group's maximum, and
    // the weight of each group against the running maximum, which rises.  (A page's probabilities are rounded to fp16 before
    // its V scale joins them: against the running maximum a page of large values and little weight would lose them.)
    auto softmax = [&](auto& sc, auto& weight) {
        constexpr int N = sizeof(sc) / sizeof(sc[0]) / 2;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float mx[N], mn = m_run[u];
#pragma unroll
            for (int x = 0; x < N; ++x) {
                mx[x] = quad_max(fmaxf(fmaxf(sc[2 * x][2 * u], sc[2 * x][2 * u + 1]), fmaxf(sc[2 * x + 1][2 * u], sc[2 * x + 1][2 * u + 1])));
                mn = fmaxf(mn, mx[x]);
            }
            if (__any_sync(0xffffffffu, mn > m_run[u])) {
                const float corr = mn == -INFINITY ? 1.f : exp2f(m_run[u] - mn);
                l_run[u] *= corr;
#pragma unroll
                for (int j = 0; j < ND; ++j) {
                    o[j][2 * u] *= corr;
                    o[j][2 * u + 1] *= corr;
                }
                m_run[u] = mn;
            }
#pragma unroll
            for (int x = 0; x < N; ++x) {
                const float base = (mx[x] == -INFINITY ? 0.f : mx[x]) - P_BIAS;
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float& s = sc[2 * x + (e >> 1)][2 * u + (e & 1)];
                    s = ex2(s - base);
                    sum += s;
                }
                weight[x][u] = mx[x] == -INFINITY ? 1.f : ex2(mx[x] - mn);
                l_run[u] = fmaf(sum, weight[x][u], l_run[u]);
            }
        }
    };

    // ---- full pages, two at a time: one page's chain of products and shuffles hides the other's ----
    for (int j = 0; j < n_pages; j += 2) {
        const bool two = j + 1 < n_pages;
        cp_async_wait<0>();
        __syncwarp();
        const unsigned char* st[2] = {smem + (warp * STAGES + j % STAGES) * Smem<D>::STAGE, smem + (warp * STAGES + (j + 1) % STAGES) * Smem<D>::STAGE};
        // (the pair before has been used by every lane: its places take the pair after this one)
        if (j + 2 < n_pages) bring(j + 2);
        if (j + 3 < n_pages) bring(j + 3);
        cp_async_commit();
        float sc[4][4], vs[2], weight[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (x == 1 && !two) {
                vs[1] = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[2][e] = sc[3][e] = -INFINITY;
                break;
            }
            const float ks = *reinterpret_cast<const float*>(st[x] + Smem<D>::LANE * 32);
            vs[x] = *reinterpret_cast<const float*>(st[x] + Smem<D>::LANE * 32 + 4);
            const float f0 = f_row[0] * ks, f1 = f_row[1] * ks;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float (&d)[4] = sc[2 * x + t];
                d[0] = d[1] = d[2] = d[3] = 0.f;
#pragma unroll
                for (int hc = 0; hc < HC; ++hc) {
                    const uint4 kw = *reinterpret_cast<const uint4*>(st[x] + ((t * HC + hc) * 32 + lane) * 16);
                    const uint32_t w[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) mma_f16_16816(d, qf[hc * 4 + i], codes_lo(w[i]), codes_hi(w[i]));
                }
                d[0] *= f0; d[1] *= f0; d[2] *= f1; d[3] *= f1;
            }
        }
        softmax(sc, weight);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (x == 1 && !two) break;
            const float f[2] = {vs[x] * weight[x][0], vs[x] * weight[x][1]};
            const uint32_t pa[4] = {pack_f16(sc[2 * x][0], sc[2 * x][1]), pack_f16(sc[2 * x][2], sc[2 * x][3]), pack_f16(sc[2 * x + 1][0], sc[2 * x + 1][1]),
                                    pack_f16(sc[2 * x + 1][2], sc[2 * x + 1][3])};
            uint32_t v[4][VW];                 // values 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned char* src = st[x] + 2 * HC * 512 + (e * 32 + lane) * (VW * 4);
                if (D == 128) {
                    const uint4 w = *reinterpret_cast<const uint4*>(src);
                    v[e][0] = w.x; v[e][1] = w.y; v[e][VW - 2] = w.z; v[e][VW - 1] = w.w;
                } else {
                    const uint2 w = *reinterpret_cast<const uint2*>(src);
                    v[e][0] = w.x; v[e][1] = w.y;
                }
            }
#pragma unroll
            for (int w = 0; w < VW; ++w) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // dims 4 w + 2 h, + 1: the codes of two tokens side by side
                    const uint32_t a = __byte_perm(v[0][w], v[1][w], h ? 0x7362 : 0x5140);
                    const uint32_t d = __byte_perm(v[2][w], v[3][w], h ? 0x7362 : 0x5140);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float r[4] = {0.f, 0.f, 0.f, 0.f};
                        mma_f16_16816(r, pa, e ? codes_hi(a) : codes_lo(a), e ? codes_hi(d) : codes_lo(d));
                        const int i = w * 4 + h * 2 + e;
#pragma unroll
                        for (int z = 0; z < 4; ++z) o[i][z] = fmaf(r[z], f[z >> 1], o[i][z]);
                    }
                }
            }
        }
    }

    // ---- what is bf16: the tail rows and the block's own, 16 at a time, with the chunk that is last ----
    if (c == n_chunks - 1) {                                   // (a block without a chunk has nothing here either)
        const int n_blk = (p.k + PAGE - 1) / PAGE;
        for (int it = (n_tail ? 0 : 1) + warp; it <= n_blk; it += WARPS) {         // 0: the tail, 1 ..: block rows
            const bool is_tail = it == 0;
            const int j0 = (it - 1) * PAGE;                                        // first block row
            const int valid = is_tail ? n_tail : min(PAGE, p.k - j0);
            const size_t stride = is_tail ? D : (size_t)Hkv * D;
            const size_t off = is_tail ? (((size_t)s * Hkv + kvh) * DEER_TAIL_ROWS + (n / PAGE % 3) * PAGE) * D
                                       : ((size_t)(b * p.k + j0) * Hkv + kvh) * D;
            const __nv_bfloat16* kr = (is_tail ? static_cast<const __nv_bfloat16*>(p.kq.k_tail) : p.k_blk) + off;
            const __nv_bfloat16* vr = (is_tail ? static_cast<const __nv_bfloat16*>(p.kq.v_tail) : p.v_blk) + off;
            // rows that hold something, and those that each of my two query rows sees, as bits of this group of 16
            const uint32_t has = is_tail ? (1u << valid) - 1u : (present >> j0) & ((1u << valid) - 1u);
            const uint32_t see[2] = {is_tail ? has : (cols[0] >> j0) & has, is_tail ? has : (cols[1] >> j0) & has};
            float sc[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
                const int tok = t * 8 + g8;
                const bool on = (has >> tok) & 1u;
#pragma unroll
                for (int hc = 0; hc < HC; ++hc)
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const int d0 = hc * 64 + t4 * 16 + z * 8;                  // two contraction steps of four dims each
                        const uint4 kv = on ? *reinterpret_cast<const uint4*>(kr + (size_t)tok * stride + d0) : make_uint4(0, 0, 0, 0);
                        const uint4 qa = *reinterpret_cast<const uint4*>(q_row[0] + d0), qb = *reinterpret_cast<const uint4*>(q_row[1] + d0);
                        const uint32_t a0[4] = {qa.x, qb.x, qa.y, qb.y}, a1[4] = {qa.z, qb.z, qa.w, qb.w};
                        mma_bf16_16816(sc[t], a0, kv.x, kv.y);
                        mma_bf16_16816(sc[t], a1, kv.z, kv.w);
                    }
#pragma unroll
                for (int z = 0; z < 4; ++z)
                    sc[t][z] = (see[z >> 1] >> (t * 8 + t4 * 2 + (z & 1))) & 1u ? sc[t][z] * p.scale_log2 : -INFINITY;
            }
            float weight[1][2];
            softmax(sc, weight);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int z = 0; z < 4; ++z) sc[t][z] *= weight[0][z >> 1];         // (fp32, and bf16's range below)
            // values: a NaN or an infinity must reach only the rows that see it, so such a group of rows goes element by element
            uint4 vv[4][D / 64];               // D / 8 bf16 of four tokens
            uint32_t worst = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int tok = 2 * t4 + (e & 1) + (e >> 1) * 8;
                const bool on = (has >> tok) & 1u;
#pragma unroll
                for (int z = 0; z < D / 64; ++z) {
                    vv[e][z] = on ? *reinterpret_cast<const uint4*>(vr + (size_t)tok * stride + g8 * (D / 8) + z * 8) : make_uint4(0, 0, 0, 0);
                    const uint32_t w[4] = {vv[e][z].x, vv[e][z].y, vv[e][z].z, vv[e][z].w};
#pragma unroll
                    for (int y = 0; y < 4; ++y) worst = max(worst, max(w[y] & 0x7fffu, (w[y] >> 16) & 0x7fffu));
                }
            }
            if (!__any_sync(0xffffffffu, worst >= 0x7f80u)) {
                // bf16 probabilities would lose three bits against the pages' fp16: two terms carry 16
                uint32_t pa[4], pb[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const float x0 = sc[z >> 1][(z & 1) * 2], x1 = sc[z >> 1][(z & 1) * 2 + 1];
                    pa[z] = pack_bf16(x0, x1);
                    pb[z] = pack_bf16(x0 - __uint_as_float(pa[z] << 16), x1 - __uint_as_float(pa[z] & 0xffff0000u));
                }
#pragma unroll
                for (int z = 0; z < D / 64; ++z) {
                    const uint32_t w0[4] = {vv[0][z].x, vv[0][z].y, vv[0][z].z, vv[0][z].w}, w1[4] = {vv[1][z].x, vv[1][z].y, vv[1][z].z, vv[1][z].w};
                    const uint32_t w2[4] = {vv[2][z].x, vv[2][z].y, vv[2][z].z, vv[2][z].w}, w3[4] = {vv[3][z].x, vv[3][z].y, vv[3][z].z, vv[3][z].w};
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t b0 = __byte_perm(w0[y], w1[y], e ? 0x7632 : 0x5410), b1 = __byte_perm(w2[y], w3[y], e ? 0x7632 : 0x5410);
                            mma_bf16_16816(o[z * 8 + y * 2 + e], pa, b0, b1);
                            mma_bf16_16816(o[z * 8 + y * 2 + e], pb, b0, b1);
                        }
                }
            } else {
                for (int tok = 0; tok < valid; ++tok) {
                    const int src = (g8 << 2) | ((tok & 7) >> 1);
                    float pr[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float x0 = __shfl_sync(0xffffffffu, sc[0][2 * u], src), x1 = __shfl_sync(0xffffffffu, sc[0][2 * u + 1], src);
                        const float x2 = __shfl_sync(0xffffffffu, sc[1][2 * u], src), x3 = __shfl_sync(0xffffffffu, sc[1][2 * u + 1], src);
                        pr[u] = tok < 8 ? ((tok & 1) ? x1 : x0) : ((tok & 1) ? x3 : x2);
                    }
                    const __nv_bfloat16* v = vr + (size_t)tok * stride + t4 * (D / 4);
#pragma unroll
                    for (int j = 0; j < ND; ++j) {
                        const float v0 = __bfloat162float(v[j]), v1 = __bfloat162float(v[ND + j]);
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            if ((see[u] >> tok) & 1u) {
                                o[j][2 * u] = fmaf(pr[u], v0, o[j][2 * u]);
                                o[j][2 * u + 1] = fmaf(pr[u], v1, o[j][2 * u + 1]);
                            }
                    }
                }
            }
        }
    }

    // ---- the warps meet (every page that was brought has been used) ----
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const float l = quad_sum(l_run[u]);
        if (t4 == 0) {
            s_m[warp][g8 + u * 8] = m_run[u];
            s_l[warp][g8 + u * 8] = live[u] ? l : 0.f;
        }
#pragma unroll
        for (int j = 0; j < ND; ++j) {
            s_o[warp][g8 + u * 8][t4 * QD + j] = o[j][2 * u];
            s_o[warp][g8 + u * 8][t4 * QD + ND + j] = o[j][2 * u + 1];
        }
    }
    __syncthreads();
    // 8 threads per row, D / 8 dims each
    const int r = tid >> 3, d0 = (tid & 7) * (D / 8), rr = rt * ROWS + r;
    const int i = min(rr, R - 1) / p.G;
    const bool absent = rr >= R || (p.row_state && p.row_state[(size_t)b * p.k + i] < 0);
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) mx = fmaxf(mx, s_m[w][r]);
    const float base = mx == -INFINITY ? 0.f : mx;
    float l = 0.f, wt[WARPS];
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        wt[w] = s_m[w][r] == -INFINITY ? 0.f : exp2f(s_m[w][r] - base);
        if (s_l[w][r] != s_l[w][r]) wt[w] = 1.f;               // a NaN passes on, whatever the maxima are
        l += wt[w] * s_l[w][r];
    }
    const float inv = (absent || l == 0.f) ? 0.f : 1.f / l;
    float acc[D / 8];
    float* mine = &s_o[0][r][(tid & 7) / 2 * QD + (tid & 1) * ND];                 // where dim d0 of row r is, with each warp's copy
#pragma unroll
    for (int d = 0; d < D / 8; ++d) {
        acc[d] = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) acc[d] = wt[w] != 0.f ? fmaf(wt[w], mine[w * ROWS * 4 * QD + d], acc[d]) : acc[d];
        acc[d] = absent ? 0.f : acc[d] * inv;
    }
    if (p.cluster == 1) {
        if (rr >= R) return;
        __nv_bfloat16* dst = p.out + ((size_t)(b * p.k + i) * p.Hq + kvh * p.G + rr % p.G) * D + d0;
#pragma unroll
        for (int d = 0; d < D / 8; d += 8)
            *reinterpret_cast<uint4*>(dst + d) = make_uint4(pack_bf16(acc[d], acc[d + 1]), pack_bf16(acc[d + 2], acc[d + 3]),
                                                            pack_bf16(acc[d + 4], acc[d + 5]), pack_bf16(acc[d + 6], acc[d + 7]));
        return;
    }

    // ---- the cluster's blocks meet: each joins its share of the rows, two dims a thread ----
#pragma unroll
    for (int d = 0; d < D / 8; ++d) mine[d] = acc[d];          // (this thread alone reads these words above)
    if ((tid & 7) == 0) s_lse[r] = (absent || l == 0.f) ? -INFINITY : mx + log2f(l);
    sm100::cluster_sync();
    const int part = c / p.cluster, rank = c % p.cluster;
    const int in_part = min(p.cluster, n_chunks - part * p.cluster), n_parts = (n_chunks + p.cluster - 1) / p.cluster;
    const uint32_t lse_addr = smem_u32(s_lse), o_addr = smem_u32(&s_o[0][0][0]);
    for (int it = rank * WARPS * 32 + tid; it < min(ROWS, R - rt * ROWS) * (D / 2); it += p.cluster * WARPS * 32) {
        const int jr = it / (D / 2), jd = it % (D / 2) * 2;    // row of the tile, dim
        const uint32_t at = o_addr + (uint32_t)((jr * 4 * QD + jd / (D / 4) * QD + jd % (D / 4)) * 4);
        float lse[CLUSTER_MAX], x0[CLUSTER_MAX], x1[CLUSTER_MAX], top = -INFINITY;
#pragma unroll
        for (int q = 0; q < CLUSTER_MAX; ++q) {
            lse[q] = q < in_part ? sm100::ld_cluster_f32(sm100::map_to_cta(lse_addr + (uint32_t)jr * 4u, (uint32_t)q)) : -INFINITY;
            x0[q] = q < in_part ? sm100::ld_cluster_f32(sm100::map_to_cta(at, (uint32_t)q)) : 0.f;
            x1[q] = q < in_part ? sm100::ld_cluster_f32(sm100::map_to_cta(at + 4u, (uint32_t)q)) : 0.f;
        }
#pragma unroll
        for (int q = 0; q < CLUSTER_MAX; ++q) top = fmaxf(top, lse[q]);
        float sum = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
        for (int q = 0; q < CLUSTER_MAX; ++q) {
            const float w = lse[q] == -INFINITY ? 0.f : exp2f(lse[q] - (top == -INFINITY ? 0.f : top));   // a NaN joins
            sum += w;
            y0 = w != 0.f ? fmaf(w, x0[q], y0) : y0;
            y1 = w != 0.f ? fmaf(w, x1[q], y1) : y1;
        }
        const float norm = sum == 0.f ? 0.f : 1.f / sum;
        y0 *= norm;
        y1 *= norm;
        const int jrr = rt * ROWS + jr;
        const size_t orow = (size_t)(b * p.k + jrr / p.G) * p.Hq + kvh * p.G + jrr % p.G;
        if (n_parts == 1) {
            *reinterpret_cast<__nv_bfloat162*>(p.out + orow * D + jd) = __floats2bfloat162_rn(y0, y1);
        } else {
            const size_t slot = (size_t)part * p.B * p.k * p.Hq + orow;
            *reinterpret_cast<float2*>(p.part_o + slot * D + jd) = make_float2(y0, y1);
            if (jd == 0) p.part_lse[slot] = sum == 0.f ? -INFINITY : top + log2f(sum);
        }
    }
    sm100::cluster_sync();                                     // nobody's shared memory goes away while it is being read
}

// One warp per output row: joins the clusters' partial results.
template <int D>
__global__ void __launch_bounds__(256) attn_quant_merge_kernel(const Params p) {
    constexpr int PER = D / 32;
    const int lane = threadIdx.x & 31;
    const size_t n_rows = (size_t)p.B * p.k * p.Hq;
    const size_t orow = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    pdl_trigger();
    pdl_wait();
    if (orow >= n_rows) return;
    int s, n;
    if (!sequence_of(p, (int)(orow / ((size_t)p.k * p.Hq)), &s, &n, false)) return;
    const int n_parts = (chunks_of(p, n) + p.cluster - 1) / p.cluster;
    if (n_parts == 1) return;                                  // written by its only cluster
    float mx = -INFINITY;
    for (int c = lane; c < n_parts; c += 32) mx = fmaxf(mx, p.part_lse[(size_t)c * n_rows + orow]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float base = mx == -INFINITY ? 0.f : mx;
    float acc[PER], sum = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] = 0.f;
    for (int c = 0; c < n_parts; ++c) {
        const float lse = p.part_lse[(size_t)c * n_rows + orow];
        const float w = lse == -INFINITY ? 0.f : exp2f(lse - base);
        const float* src = p.part_o + ((size_t)c * n_rows + orow) * D + lane * PER;
        sum += w;
        if (w != 0.f) {                                        // a NaN joins
#pragma unroll
            for (int e = 0; e < PER; ++e) acc[e] = fmaf(w, src[e], acc[e]);
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    __nv_bfloat16* dst = p.out + orow * D + lane * PER;
#pragma unroll
    for (int e = 0; e < PER; e += 2) *reinterpret_cast<__nv_bfloat162*>(dst + e) = __floats2bfloat162_rn(acc[e] * inv, acc[e + 1] * inv);
}

struct Plan {
    int row_tiles, chunk_pages, chunks, cluster, parts;
};
// The context is cut so that the blocks of all units fill the SMs once (clusters of eight do not quite: they stay within
// groups of SMs), in chunks of two pages per warp at least.  One cluster without a second kernel is the better choice up
// to six pages per warp (one token, 8 heads: 10.2 against 11.9 us at 2048 tokens, 13.6 against 12.2 at 4096).
static Plan plan(int B, int k, int Hq, int Hkv, int max_seq_len) {
    Plan pl;
    pl.row_tiles = (Hq / Hkv * k + ROWS - 1) / ROWS;
    const long long units = (long long)B * Hkv * pl.row_tiles, pages = max_seq_len / PAGE;
    long long want = RESIDENT * deer_sm_count() * 9LL / 10 / units;
    if (want < 1) want = 1;
    if (want > CLUSTER_MAX) want = pages <= CLUSTER_MAX * WARPS * 6 ? CLUSTER_MAX : want / CLUSTER_MAX * CLUSTER_MAX;
    long long per = (pages + want - 1) / want;
    if (per < 2 * WARPS) per = 2 * WARPS;
    pl.chunk_pages = (int)per;
    pl.chunks = pages > per ? (int)((pages + per - 1) / per) : 1;
    pl.cluster = pl.chunks < CLUSTER_MAX ? pl.chunks : CLUSTER_MAX;
    pl.parts = (pl.chunks + pl.cluster - 1) / pl.cluster;
    return pl;
}

}  // namespace attnq

using namespace attnq;

extern "C" size_t deer_block_attn_quant_workspace_bytes(int B, int k, int Hq, int Hkv, int D, int max_seq_len) {
    if (B <= 0 || k <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || D <= 0 || max_seq_len < 0) return 0;
    // room for whichever kernel the call ends up using
    const Plan pl = plan(B, k, Hq, Hkv, max_seq_len);
    const size_t small = pl.parts == 1 ? 16 : (size_t)pl.parts * B * k * Hq * (D + 1) * sizeof(float);
    if (!use_umma(B, D, k, Hq, Hkv, max_seq_len, 1.f)) return small;
    const size_t large = umma_workspace_bytes(B, k, Hq, Hkv, max_seq_len);
    return large > small ? large : small;
}

extern "C" int deer_block_attn_quant(deer_kv* kv, const int32_t* seq_ids, const void* q, const void* k_blk, const void* v_blk, void* out,
                                     const int32_t* row_state, int B, int k, int Hq, int mask, float scale, int max_seq_len,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    DEER_CHECK_ARG(kv && seq_ids && q && k_blk && v_blk && out, DEER_ERR_INVALID_ARG, "deer_block_attn_quant: null argument");
    DEER_CHECK_ARG(kv->quant, DEER_ERR_UNSUPPORTED, "deer_block_attn_quant: the cache holds bf16 pools (deer_block_attn reads them)");
    DEER_CHECK_ARG(!row_state || mask == DEER_MASK_BIDIR, DEER_ERR_INVALID_ARG,
                   "deer_block_attn_quant: row states belong to the bidirectional mask");
    DEER_CHECK_ARG(deer_aligned16(q) && deer_aligned16(k_blk) && deer_aligned16(v_blk) && deer_aligned16(out) && deer_aligned16(workspace),
                   DEER_ERR_INVALID_ARG, "deer_block_attn_quant: pointers must be 16-byte aligned");
    DEER_CHECK_ARG(k >= 1 && k <= DEER_MAX_BLOCK, DEER_ERR_UNSUPPORTED, "deer_block_attn_quant: k must be in [1, 32]");
    DEER_CHECK_ARG(B >= 0 && B <= 65535, DEER_ERR_UNSUPPORTED, "deer_block_attn_quant: B must be in [0, 65535]");
    const int Hkv = kv->d.n_kv_heads, D = kv->d.head_dim;
    DEER_CHECK_ARG(Hq > 0 && Hq % Hkv == 0, DEER_ERR_INVALID_ARG, "deer_block_attn_quant: Hq must be a positive multiple of Hkv");
    DEER_CHECK_ARG(mask == DEER_MASK_CAUSAL || mask == DEER_MASK_BIDIR, DEER_ERR_INVALID_ARG, "deer_block_attn_quant: bad mask");
    DEER_CHECK_ARG(max_seq_len >= 0, DEER_ERR_INVALID_ARG, "deer_block_attn_quant: max_seq_len must be >= 0");
    if (B == 0) return DEER_OK;
    const size_t need = deer_block_attn_quant_workspace_bytes(B, k, Hq, Hkv, D, max_seq_len);
    DEER_CHECK_ARG(workspace && workspace_bytes >= need, DEER_ERR_WORKSPACE,
                   "deer_block_attn_quant: workspace of %zu bytes needed, %zu given", need, workspace_bytes);
    const Plan pl = plan(B, k, Hq, Hkv, max_seq_len);
    DEER_CHECK_ARG((long long)Hkv * pl.row_tiles <= 65535 && Hq <= 65535, DEER_ERR_UNSUPPORTED, "deer_block_attn_quant: too many heads");
    Params p = {};
    p.kv = kv->d;
    p.kq = kv->q;
    p.seq_ids = seq_ids;
    p.row_state = row_state;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k_blk = static_cast<const __nv_bfloat16*>(k_blk);
    p.v_blk = static_cast<const __nv_bfloat16*>(v_blk);
    p.out = static_cast<__nv_bfloat16*>(out);
    const size_t n_rows = (size_t)B * k * Hq;
    p.part_o = static_cast<float*>(workspace);
    p.part_lse = p.part_o + (size_t)pl.parts * n_rows * D;
    p.B = B;
    p.k = k;
    p.Hq = Hq;
    p.G = Hq / Hkv;
    p.mask = mask;
    p.max_seq_len = max_seq_len;
    p.scale_log2 = scale * LOG2E;
    p.row_tiles = pl.row_tiles;
    p.chunk_pages = pl.chunk_pages;
    p.cluster = pl.cluster;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (use_umma(B, D, k, Hq, Hkv, max_seq_len, scale)) return launch_umma(p, workspace, st);
    const dim3 grid((unsigned)(pl.parts * pl.cluster), (unsigned)(Hkv * pl.row_tiles), (unsigned)B);
    const auto kernel = D == 128 ? attn_quant_kernel<128> : attn_quant_kernel<64>;
    const int smem = D == 128 ? Smem<128>::BYTES : Smem<64>::BYTES;
    DEER_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    DEER_CUDA(launch_pdl_cluster(pl.cluster, kernel, grid, dim3(WARPS * 32), smem, st, p));
    if (pl.parts > 1)
        DEER_CUDA(launch_pdl(D == 128 ? attn_quant_merge_kernel<128> : attn_quant_merge_kernel<64>, dim3((unsigned)((n_rows + 7) / 8)), dim3(256), 0, st, p));
    return DEER_OK;
}
