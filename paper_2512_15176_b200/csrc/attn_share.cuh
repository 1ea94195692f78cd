// The split of a block-attention call over thread blocks: the KV tiles of all
// (sequence, KV head) units, laid end to end, are cut into one equal share per
// group of thread blocks; each (unit, block) piece of a share is a segment.
#pragma once

#include "attn.cuh"

namespace attn {

constexpr int MAX_SEGS = 48;                   // segments listed at a time; longer shares go in several rounds

struct Seg {             // one (unit, block) piece
    int b, hr;           // sequence index in the call; KV head * row_tiles + row tile
    int t_a, t_b;        // tile range within the unit; the last tile of a unit is the block rows' own K/V
    int n, s;            // committed length and cache slot of the sequence
    long long u0;        // flattened position of the unit's first tile
};

#ifdef __CUDACC__

// Share of thread block j out of nc over T tiles: [share_begin(j), share_begin(j + 1)).
__device__ __forceinline__ long long share_begin(long long T, int j, int nc) { return T * j / nc; }

// Warp-collective: lists up to MAX_SEGS segments of the flattened tile range [cursor, end) into segs[], in order.
// Returns their number; *cursor_out is where the next round starts (== end when the share is exhausted).
// tiles_of(b, &n, &s): tiles of sequence b (0: unusable), its committed length and its cache slot.
template <typename TilesOf>
__device__ int build_segments(const AttnParams& p, int HL, int rt, long long cursor, long long end, Seg* segs,
                              long long* cursor_out, int lane, TilesOf tiles_of) {
    int n_seg = 0;
    long long base = 0;                                   // flattened position of sequence b0's first tile
    long long next_cursor = end;
    bool cut = false;
    for (int b0 = 0; b0 < p.B && base < end && n_seg < MAX_SEGS; b0 += 32) {
        const int b = b0 + lane;
        int n = 0, s = 0;
        const int tiles = (b < p.B) ? tiles_of(b, &n, &s) : 0;
        const long long span = (long long)tiles * HL;     // tiles this sequence contributes to the list
        long long incl = span;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += t;
        }
        const long long my0 = base + incl - span, my1 = base + incl;
        // units of my sequence that meet [cursor, end)
        int hr_lo = 0, hr_hi = -1;
        if (tiles > 0 && my1 > cursor && my0 < end) {
            hr_lo = cursor > my0 ? (int)((cursor - my0) / tiles) : 0;
            hr_hi = (int)(((end < my1 ? end : my1) - 1 - my0) / tiles);
        }
        const int cnt = hr_hi - hr_lo + 1 > 0 ? hr_hi - hr_lo + 1 : 0;
        int cincl = cnt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, cincl, o);
            if (lane >= o) cincl += t;
        }
        const int off = n_seg + cincl - cnt;
        for (int e = 0; e < cnt; ++e) {
            const int idx = off + e;
            const int hr = hr_lo + e;
            const long long u0 = my0 + (long long)hr * tiles;
            if (idx < MAX_SEGS) {
                Seg sg;
                sg.b = b;
                sg.hr = hr * p.row_tiles + rt;
                sg.t_a = cursor > u0 ? (int)(cursor - u0) : 0;
                sg.t_b = end < u0 + tiles ? (int)(end - u0) : tiles;
                sg.n = n;
                sg.s = s;
                sg.u0 = u0;
                segs[idx] = sg;
            } else if (idx == MAX_SEGS) {
                next_cursor = u0;                          // the first segment that did not fit starts the next round
            }
        }
        const int total = __shfl_sync(0xffffffffu, cincl, 31);
        // at most one lane owns index MAX_SEGS; share its cursor
        const unsigned who = __ballot_sync(0xffffffffu, off <= MAX_SEGS && MAX_SEGS < off + cnt);
        if (who) next_cursor = __shfl_sync(0xffffffffu, next_cursor, __ffs(who) - 1);
        n_seg = n_seg + total < MAX_SEGS ? n_seg + total : MAX_SEGS;
        base += __shfl_sync(0xffffffffu, incl, 31);
        if (who) {
            cut = true;
            break;
        }
    }
    if (!cut && n_seg == MAX_SEGS) next_cursor = base < end ? base : end;   // the list filled up exactly at a sequence boundary
    *cursor_out = next_cursor;
    return n_seg;
}

#endif  // __CUDACC__

}  // namespace attn
