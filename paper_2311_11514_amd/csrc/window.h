// New rows of ragged sequences that attend a sliding window and the first positions of their contexts: what the kernels of both storage widths share.
#pragma once
#include "kernels.h"

// The tiles of 32 positions that rows at slots p_lo .. p_hi reach, by their index in a list: first the `clean` ones, which every row attends whole and the
// cache holds (positions from `held` on may not be there yet) -- first positions, then the window's inside -- and behind them those that need a mask.
struct WinTiles {
    int full, ns, w0, c0, c1, clean, nt;       // tiles [0, full) and [c0, c1) are clean, [full, ns) and [w0, p_hi / 32] otherwise are not
    __host__ __device__ __forceinline__ void set(int p_lo, int p_hi, int window, int sinks, int held) {
        const int first = p_lo - window + 1;
        w0 = first > 0 ? first >> 5 : 0;
        ns = (sinks + 31) >> 5;
        ns = ns < w0 ? ns : w0;
        full = sinks >> 5;
        full = full < ns ? full : ns;
        const int hidden = p_hi - window;      // the last row does not see this one
        c0 = hidden >= 0 ? (hidden >> 5) + 1 : 0;
        c0 = c0 > w0 ? c0 : w0;
        c1 = (p_lo < held ? p_lo + 1 : held) >> 5;
        if (c1 <= c0) c0 = c1 = w0;
        clean = full + c1 - c0;
        nt = ns + (p_hi >> 5) - w0 + 1;
    }
    __host__ __device__ __forceinline__ int at(int v) const {
        if (v < full) return v;
        if (v < clean) return v - full + c0;
        v -= c1 - c0;                          // now an index in what the clean inside of the window has been taken out of
        if (v < ns) return v;
        v += w0 - ns;
        return v < c0 ? v : v + c1 - c0;
    }
};

// bits 0 .. x - 1 of 32
__device__ __forceinline__ uint32_t win_below(int x) { return x <= 0 ? 0u : x >= 32 ? 0xffffffffu : (1u << x) - 1; }
// which of the 32 positions from p0 on the row at slot p attends
__device__ __forceinline__ uint32_t win_sees(int p0, int p, int window, int sinks) {
    return win_below(p + 1 - p0) & (~win_below(p - window + 1 - p0) | win_below(sinks - p0));
}
// do rows at slots p_lo .. p_hi attend all `width` positions from p0 on?
__device__ __forceinline__ bool win_all(int p0, int width, int p_lo, int p_hi, int window, int sinks) {
    return p0 + width - 1 <= p_lo && (p0 > p_hi - window || p0 + width <= sinks);
}
// does any of them attend one?
__device__ __forceinline__ bool win_any(int p0, int width, int p_lo, int p_hi, int window, int sinks) {
    return p0 <= p_hi && (p0 + width - 1 > p_lo - window || p0 < sinks);
}

// Which of `units` (each `per` blocks) a block belongs to, and which of its blocks it is.  Ids go round the 8 XCDs.  Many units, or a multiple of 8: a unit's
// blocks sit next to each other on one XCD and share what they read in that L2, and the units, which come in falling order of their work, are dealt there and back
// so that no XCD gets the larger one every time; a few others: block by block, so that every XCD has some.
__host__ __device__ inline bool win_grouped(int units) { return units % 8 == 0 || units >= 64; }
__host__ __device__ inline unsigned win_grid(int units, int per) { return (unsigned)per * (unsigned)(win_grouped(units) ? (units + 7) / 8 * 8 : units); }
__device__ __forceinline__ void win_place(int units, int per, int *unit, int *nth) {
    const unsigned id = blockIdx.x;
    if (win_grouped(units)) {
        *nth = (int)((id >> 3) % (unsigned)per);
        const int round = (int)((id >> 3) / (unsigned)per);
        *unit = 8 * round + (int)(round & 1 ? 7 - (id & 7) : id & 7);        // at least `units`: no work
    } else {
        *nth = (int)(id / (unsigned)units);
        *unit = (int)(id % (unsigned)units);
    }
}

// What a block works on: `rows` query rows of one (sequence, kv head) -- row r: new row r / G of the sequence, head r % G -- and a run of their
// tiles.  The last rows, which reach furthest, first; sequences in wc.order.
struct WinWork {
    int rb, split, c, seq, nth, row0, n, R, len, per, v0, v1;
    WinTiles tiles;
    __device__ __forceinline__ bool find(int hkv, int G, int nrb, int rows, const WinCall &wc, const int32_t *lens, const WinPlan &wp, bool fresh) {
        const int units = wc.batch * hkv * wp.nsplit;
        int combo;
        win_place(units, nrb, &combo, &rb);
        rb = nrb - 1 - rb;
        if (combo >= units) return false;
        split = combo % wp.nsplit;
        combo /= wp.nsplit;
        c = combo % hkv;
        nth = wc.order[combo / hkv];
        seq = wc.seq0 + nth;
        row0 = wc.cu[nth];
        len = lens[seq];
        n = min(wc.cu[nth + 1] - row0, wc.max_seq - len);     // rows that would pass the cache are left out
        R = n * G;
        if (rb * rows >= R) return false;
        const int p_lo = len + rb * rows / G, p_hi = len + min(n - 1, (rb * rows + rows - 1) / G);
        tiles.set(p_lo, p_hi, wc.window, wc.sinks, fresh ? len : p_lo + 1);
        per = max(wp.chunk, (tiles.nt + wp.nsplit - 1) / wp.nsplit);
        v0 = split * per;
        v1 = min(v0 + per, tiles.nt);
        return v0 < tiles.nt;
    }
    __device__ __forceinline__ int runs() const { return (tiles.nt + per - 1) / per; }
};
