// Attention of drafted trees over the cache, 16-bit types: appending the trees' rows, the attention itself, the move of an accepted
// path.  Compiled once per 16-bit element type (see common.h) into namespace HX_NS.
//
// The G query heads of a kv head and the n nodes of a sequence's tree make R = n G query rows (row r: node r / G, head r % G) that
// read the same K and V, so every tile of the cache serves all of them: with 8 heads and 16 nodes the attention has 128 flops
// for every byte of the cache, between the decode kernels (8) and prefill.
#include <type_traits>

#include "kernels.h"
#include "kvlayout.h"

#define NEG_INF (-INFINITY)

namespace HX_NS {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

// The stage's fused projection, raw fp32 [rows][N] -> rotary embedding at len + depth, q as plain rows, k and v into the cache.
// The projection's columns are in the order of its packed tiles: 16 columns hold elements 8 tl .. 8 tl + 7 of a head and those half a
// head further.  A thread takes four rotary pairs.  q is rounded to the element type here, once, as in the prefill path.
__global__ __launch_bounds__(256) void tree_rope_append_kernel(const float *__restrict__ qkv, int hq_l, KvGeom kg, TreeView tv,
                                                               const int32_t *__restrict__ lens, const float *__restrict__ cos_tab,
                                                               const float *__restrict__ sin_tab, h16_t *__restrict__ q, h16_t *__restrict__ q_lo,
                                                               h16_t *__restrict__ kc, h16_t *__restrict__ vc) {
    const int d = kg.d, half = d >> 1, tph = d >> 4, heads = hq_l + 2 * kg.hkv_l;
    const unsigned idx = blockIdx.x * 256u + threadIdx.x, per_row = heads * tph * 2;
    if (idx >= tv.rows * per_row) return;
    const int t = idx / per_row, rem = idx - t * per_row, head = rem / (2 * tph), tl = (rem >> 1) % tph, i0 = 8 * tl + 4 * (rem & 1);
    const TreeRow row = tv.row[t];
    const int len = lens[row.seq], slot = len + row.index;
    if (slot >= kg.smax) return;
    const float *src = qkv + (size_t)t * heads * d + (size_t)(head * tph + tl) * 16 + 4 * (rem & 1);
    floatx4 lo = *reinterpret_cast<const floatx4 *>(src), hi = *reinterpret_cast<const floatx4 *>(src + 8);
    if (head < hq_l + kg.hkv_l) {
        const size_t at = (size_t)(len + row.depth) * half + i0;
        const floatx4 c4 = *reinterpret_cast<const floatx4 *>(cos_tab + at), s4 = *reinterpret_cast<const floatx4 *>(sin_tab + at);
        const floatx4 l = lo * c4 - hi * s4;
        hi = hi * c4 + lo * s4;
        lo = l;
    }
    union { uint2 u; h16_t x[4]; } a, b, al, bl;       // the element type's parts of both halves' four elements, and what they leave
    split_pack2(lo[0], lo[1], a.u.x, al.u.x);
    split_pack2(lo[2], lo[3], a.u.y, al.u.y);
    split_pack2(hi[0], hi[1], b.u.x, bl.u.x);
    split_pack2(hi[2], hi[3], b.u.y, bl.u.y);
    if (head < hq_l) {
        const size_t at = ((size_t)t * hq_l + head) * d + i0;
        *reinterpret_cast<uint2 *>(q + at) = a.u;
        *reinterpret_cast<uint2 *>(q + at + half) = b.u;
        if (q_lo != nullptr) {
            *reinterpret_cast<uint2 *>(q_lo + at) = al.u;
            *reinterpret_cast<uint2 *>(q_lo + at + half) = bl.u;
        }
        return;
    }
    const bool key = head < hq_l + kg.hkv_l;
    const size_t slab = (size_t)row.seq * kg.seq_stride + (size_t)(head - hq_l - (key ? 0 : kg.hkv_l)) * kg.smax * d;
    if (key) {
        *reinterpret_cast<uint2 *>(kc + slab + kv_k_offset(slot, i0, d)) = a.u;
        *reinterpret_cast<uint2 *>(kc + slab + kv_k_offset(slot, half + i0, d)) = b.u;
    } else {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            vc[slab + kv_v_offset(slot, i0 + x, d)] = a.x[x];
            vc[slab + kv_v_offset(slot, half + i0 + x, d)] = b.x[x];
        }
    }
}
void launch_tree_rope_append(const float *qkv, int hq_l, KvGeom kg, const TreeView &tv, const int32_t *lens, const float *cos_tab,
                             const float *sin_tab, h16_t *q, h16_t *q_lo, h16_t *kc, h16_t *vc, hipStream_t s) {
    const unsigned n = (unsigned)tv.rows * (hq_l + 2 * kg.hkv_l) * (kg.d >> 4) * 2;
    hipLaunchKernelGGL(tree_rope_append_kernel, dim3((n + 255) / 256), dim3(256), 0, s, qkv, hq_l, kg, tv, lens, cos_tab, sin_tab, q, q_lo, kc, vc);
}

// ---- attention ----------------------------------------------------------------------------------------------------
// four consecutive elements of row t of the result, in the layout its reader takes
__device__ __forceinline__ void tree_store4(const TreeOut &out, int t, int col, const float (&x)[4]) {
    h16_t *o = static_cast<h16_t *>(out.o);
    if (out.mode == TREE_OUT_ACT) {
        uint2 a, b;
        split_pack2(x[0], x[1], a.x, b.x);
        split_pack2(x[2], x[3], a.y, b.y);
        *reinterpret_cast<uint2 *>(o + dec_act_offset(t, col, out.width >> 5, 0, out.rows)) = a;
        *reinterpret_cast<uint2 *>(o + dec_act_offset(t, col, out.width >> 5, 1, out.rows)) = b;
    } else {
        const size_t at = out.mode == TREE_OUT_FRAG ? frag_offset(t, col, out.width >> 5) : (size_t)t * out.width + col;
        *reinterpret_cast<uint2 *>(o + at) = uint2{pack_h16x2(x[0], x[1]), pack_h16x2(x[2], x[3])};
    }
}

// any of the 8 elements an infinity or a NaN
__device__ __forceinline__ bool any_odd(h16x8 v) {
#ifdef HX_ELEM_F16
    constexpr uint32_t E = 0x7c00u;
#else
    constexpr uint32_t E = 0x7f80u;
#endif
    union { h16x8 v; uint32_t u[4]; } w;
    w.v = v;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) odd = odd || (w.u[i] & E) == E || ((w.u[i] >> 16) & E) == E;
    return odd;
}

// Which of the 32 positions of tile t a node attends: bit p for position 32 t + p; the tile reaches the tree's slots (32 t + 31 >= len)
__device__ __forceinline__ uint32_t tree_sees(const uint32_t *mask, int mask_words, int t, int len) {
    const int rel = 32 * t - len;                            // index in the tree of the tile's first slot; negative: context before it
    if (rel < 0) return (mask[0] << -rel) | ((1u << -rel) - 1);
    const int w = rel >> 5, sh = rel & 31;
    const uint32_t a = w < mask_words ? mask[w] : 0u, b = w + 1 < mask_words ? mask[w + 1] : 0u;
    return sh == 0 ? a : (a >> sh) | (b << (32 - sh));
}

// The running softmax over one tile's scores (sc becomes the weights): m, l and the factor for what was summed up before
__device__ __forceinline__ float tree_softmax(floatx16 &sc, float &m, float &lsum, float scale_log2e) {
    float mx = NEG_INF;
#pragma unroll
    for (int x = 0; x < 16; ++x) mx = fmaxf(mx, sc[x]);
    const float m_new = fmaxf(m, max_halves(mx));
    const float base = m_new == NEG_INF ? 0.f : m_new;       // a row that has seen nothing yet: weights 0, no NaN
    const float alpha = __builtin_amdgcn_exp2f((m - base) * scale_log2e);
    m = m_new;
    float ps = 0.f;
#pragma unroll
    for (int x = 0; x < 16; ++x) {
        // (the difference first: scores near the type's lowest value would not cancel in a multiply-add with -base * scale)
        sc[x] = __builtin_amdgcn_exp2f((sc[x] - base) * scale_log2e);
        ps += sc[x];
    }
    lsum = lsum * alpha + ps;
    return alpha;
}
// P for k-groups hl (quads 0, 2) and 2 + hl (quads 1, 3) of the second product, in two parts like every fp32 activation of the decode kernels: one
// part alone would put a rounding of every weight on top of the result's own (a third more error), and the matrix cores have room for both.
// hi is cut off, not rounded, and lo is at least the type's smallest number (bf16: normal number) where hi is not zero: both parts of a weight are
// positive, or zero with it, so that an infinite value of the context comes out as infinite and one of a position that is not attended not at all.
union TreeP { uint32_t u[4]; h16x8 v; };
__device__ __forceinline__ void tree_pack2(float a, float b, uint32_t &hi, uint32_t &lo) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    float ah, bh;
#ifdef HX_ELEM_F16
    constexpr unsigned short LEAST = 1;
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
#else
    constexpr unsigned short LEAST = 0x80;
    hi = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
#endif
    h16x2_to_f32(hi, ah, bh);
    const u16x2 least = __builtin_elementwise_min(__builtin_bit_cast(u16x2, hi), u16x2{LEAST, LEAST});
    lo = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, pack_h16x2(a - ah, b - bh)), least));
}
__device__ __forceinline__ void tree_pack(const floatx16 &sc, TreeP (&p)[2], TreeP (&lo)[2]) {
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = 4 * g + 2 * (i & 1) + 8 * (i >> 1);
            tree_pack2(sc[x], sc[x + 1], p[g].u[i], lo[g].u[i]);
        }
}
// O^T += V^T . P^T element by element, over the positions a row attends: for tiles with values that are not finite.  vt: the tile in LDS
template <int DB>
__device__ __forceinline__ void tree_slow_tile(const h16_t *vt, const floatx16 &sc, uint32_t sees, int lane, floatx16 (&oacc)[DB]) {
    const int hl = lane >> 5;
    for (int pp = 0; pp < 32; ++pp) {
        float w = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) w = x == 4 * (pp >> 3) + (pp & 3) ? sc[x] : w;
        w = __shfl(w, (lane & 31) + 32 * ((pp >> 2) & 1), 64);
        if (!((sees >> pp) & 1u)) continue;
        const int at = (pp & 3) + 4 * (pp >> 4) + 8 * 16 * ((pp & 15) >> 2);    // kvlayout.h: position pp of element 0 of a V tile
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int dd = 32 * db + 8 * (x >> 2) + 4 * hl + (x & 3);
                oacc[db][x] = fmaf(w, h16_to_f32(vt[(dd >> 4) * 512 + (dd & 15) * 8 + at]), oacc[db][x]);
            }
    }
}

// What a block works on.  Block id = 8 slot + xcd: the row blocks of a run of tiles sit next to each other on one XCD and share the run in
// its L2; sequences in tp.order, the longest first.
struct TreeWork {
    int rb, split, c, seq, row0, n, R, len, nt, per, t0, t1;
    __device__ __forceinline__ bool find(const KvGeom &kg, int G, int nrb, int rows, const TreeView &tv, const int32_t *lens, const TreePlan &tp) {
        const int slot = blockIdx.x >> 3;
        rb = slot % nrb;
        int combo = (slot / nrb) * 8 + (blockIdx.x & 7);
        if (combo >= tv.batch * kg.hkv_l * tp.nsplit) return false;
        split = combo % tp.nsplit;
        combo /= tp.nsplit;
        c = combo % kg.hkv_l;
        const int nth = combo / kg.hkv_l;
        seq = nth < kTreeOrdered ? tp.order[nth] : nth;
        row0 = tv.cu[seq];
        n = tv.cu[seq + 1] - row0;
        R = n * G;
        if (rb * rows >= R) return false;
        len = lens[seq];
        nt = min((len + n + 31) >> 5, kg.smax >> 5);
        per = max(tp.chunk, (nt + tp.nsplit - 1) / tp.nsplit);
        t0 = split * per;
        t1 = min(t0 + per, nt);
        return t0 < nt;
    }
    __device__ __forceinline__ int runs() const { return (nt + per - 1) / per; }
};

// The rows of a drafted tree that are not in the cache yet (in.k != NULL): positions len .. len + n - 1 of a tile come from the caller's rows.  The
// 64 RW threads that share the tile put them into LDS over what the cache held there, in the cache's layout (kvlayout.h), and `append`
// blocks write them to the cache as well; other blocks of the launch may read those slots meanwhile, but put the same rows over what they got.
template <int D, int RW>
__device__ __forceinline__ void tree_patch(h16x8 (*st)[64], const TreeIn &in, int t, int len, int n, int row0, int c, int thread, bool append, h16_t *ks, h16_t *vs) {
    constexpr int KT = D / 32, P8 = D / 8, PIECES = 32 * 2 * P8 / (64 * RW), BATCH = PIECES < 8 ? PIECES : 8;      // 16-byte pieces of K and V per thread
    for (int b = 0; b < PIECES; b += BATCH) {
        uint4 r[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int idx = thread + 64 * RW * (b + i), pos = idx / (2 * P8), piece = idx % (2 * P8), e = c * D + 8 * (piece % P8);
            const int x = min(max(32 * t + pos - len, 0), n - 1);
            r[i] = piece < P8 ? *reinterpret_cast<const uint4 *>(static_cast<const h16_t *>(in.k) + (size_t)(row0 + x) * in.ldk + e)
                              : *reinterpret_cast<const uint4 *>(static_cast<const h16_t *>(in.v) + (size_t)(row0 + x) * in.ldv + e);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int idx = thread + 64 * RW * (b + i), pos = idx / (2 * P8), piece = idx % (2 * P8), dd = 8 * (piece % P8);
            const int x = 32 * t + pos - len;
            if (x < 0 || x >= n) continue;
            // an offset in a tile pair's K (V) fragments is the same in LDS and, from the pair's first tile on, in the cache
            if (piece < P8) {
                const size_t at = kv_k_offset(pos, dd, D);
                *reinterpret_cast<uint4 *>(reinterpret_cast<h16_t *>(st) + at) = r[i];
                if (append) *reinterpret_cast<uint4 *>(ks + (size_t)t * 32 * D + at) = r[i];
            } else {
                union { uint4 u; h16_t e[8]; } w;
                w.u = r[i];
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const size_t at = kv_v_offset(pos, dd + y, D);
                    reinterpret_cast<h16_t *>(st + 2 * KT)[at] = w.e[y];
                    if (append) vs[(size_t)t * 32 * D + at] = w.e[y];
                }
            }
        }
    }
}

// Many rows: a block of four waves takes 32 RW query rows of one (sequence, kv head) and a run of 32-position tiles; RW groups of 32 rows times
// CW = 4 / RW neighbouring tiles a step.  The tiles go from HBM to LDS directly, S steps in flight, and S^T = K . Q^T,
// O^T = V^T . P^T run on the 32 x 32 x 16 MFMA as in the prefill attention: a lane owns one query row, P stays in its
// registers and goes into the second product in two parts (tree_pack2; with one part, which leaves results a fifth to a third less exact, the times
// below were 127, 354 and 182).
// Tiles that lie in the context need no mask; of a tile that reaches the tree's slots a lane takes 32 bits of its node's ancestors.
// A weight of zero times an infinity would be a NaN, so a masked tile with a value that is not finite is multiplied out element
// by element over what each row attends.
// Contexts are cut into runs of tp.chunk tiles (tp.nsplit at most), whose (m, l, o) tree_merge_kernel joins: a launch of its own, since joining
// 128 rows of a run moves 64 KB, which one last block would take longer over.
// Bound by HBM with few nodes, by each wave's chain of LDS reads, products and softmax with many (matrix cores 44 % busy, vector units 53 %): d 128, 64 query and 8 kv heads, 32
// sequences of 4000: 16 nodes 139 us (3.8 TB/s), 64 nodes 447 (600 TFLOP/s); contexts of 240 .. 4027 and 8 .. 64 nodes 209 (383 TFLOP/s: a quarter of
// the blocks' rows do not exist, and the long contexts end late).
// QLO: the query rows come in two parts.
template <int D, int RW, int S, bool QLO>
__global__ __launch_bounds__(256, RW == 4 ? 3 : 2) void tree_attn_kernel(const h16_t *__restrict__ q, const h16_t *__restrict__ q_lo, int64_t ldq, TreeIn in, h16_t *kc, h16_t *vc, KvGeom kg, int hq_l, int G, int nrb,
                                                           TreeView tv, const int32_t *__restrict__ lens, TreePlan tp, TreeOut out, float scale_log2e) {
    constexpr int CW = 4 / RW, ROWS = 32 * RW;
    constexpr int KT = D / 32, DT = D / 16, DB = D / 32, TILES = 2 * KT + DT;
    constexpr int LPT = TILES / RW;                       // 1 KB loads per wave and step: RW waves share a tile position
    constexpr int OS = D + 4;                             // floats between rows of the merge buffer: eight rows on distinct banks
    constexpr int STAGE = S * CW * TILES * 1024, MERGE = CW > 1 ? 4 * 32 * OS * 4 : 0;
    __shared__ __align__(16) unsigned char smem[STAGE > MERGE ? STAGE : MERGE];
    __shared__ float s_m[4][32], s_l[4][32];
    h16x8(*stage)[CW][TILES][64] = reinterpret_cast<h16x8(*)[CW][TILES][64]>(smem);
    TreeWork wk;
    if (!wk.find(kg, G, nrb, ROWS, tv, lens, tp)) return;
    const int len = wk.len, t0 = wk.t0, t1 = wk.t1, R = wk.R, row0 = wk.row0, steps = (t1 - t0 + CW - 1) / CW;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int rw = wave % RW, cw = wave / RW, hl = lane >> 5;
    const int r = wk.rb * ROWS + rw * 32 + (lane & 31);
    const bool idle = wk.rb * ROWS + rw * 32 >= R;        // the wave has no row: it feeds the others
    const int rr = min(r, R - 1), node = rr / G, head = wk.c * G + (rr - node * G);    // rows past the last repeat it and are not stored
    const uint32_t *mask = tv.mask + (size_t)(row0 + node) * tv.mask_words;

    h16x8 qf[2 * KT], ql[QLO ? 2 * KT : 1];
#pragma unroll
    for (int kk = 0; kk < 2 * KT; ++kk) {
        const size_t at = (size_t)(row0 + node) * ldq + (size_t)head * D + 16 * kk + 8 * hl;
        qf[kk] = *reinterpret_cast<const h16x8 *>(q + at);
        if constexpr (QLO) ql[kk] = *reinterpret_cast<const h16x8 *>(q_lo + at);
    }
    floatx16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) oacc[db][x] = 0.f;
    float m = NEG_INF, lsum = 0.f;

    const size_t slab = (size_t)wk.seq * kg.seq_stride + (size_t)wk.c * kg.smax * D;
    h16_t *kslab = kc + slab, *vslab = vc + slab;
    const h16x8 *ks = reinterpret_cast<const h16x8 *>(kslab), *vs = reinterpret_cast<const h16x8 *>(vslab);
    const unsigned lane_bytes = (unsigned)lane * 16u;
    auto issue = [&](int step) {
        const int t = min(t0 + step * CW + cw, t1 - 1);
#pragma unroll
        for (int x = 0; x < LPT; ++x) {
            const int tile = rw + RW * x;
            const h16x8 *src = tile < 2 * KT ? ks + (size_t)(2 * t * KT + tile) * 64 : vs + (size_t)(t * DT + tile - 2 * KT) * 64;
            hx_load_lds16(hx_lds_addr(&stage[step % S][cw][tile][0]), lane_bytes, src);
        }
    };
    const int sub = (lane & 31) >> 4, fl = (lane & 15) + 16 * hl;
    HX_WAIT_VM(0);            // the query rows have landed before the first load that the compiler does not see
#pragma unroll
    for (int x = 0; x < S - 1; ++x)
        if (x < steps) issue(x);
    // a step whose tiles all lie in the context (TAIL false), or one that may reach the tree's slots
    auto walk = [&](int step, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        // steps step + 1 .. step + S - 2 may stay in flight
        if (S > 2 && step + 1 < steps) HX_WAIT_VM(LPT);
        else HX_WAIT_VM(0);
        HX_LDS_BARRIER();
        const int t = t0 + step * CW + cw;
        const bool masked = TAIL && 32 * t + 31 >= len;
        if constexpr (TAIL) {
            if (in.k != nullptr) {                            // the same in every wave
                if (t < t1 && masked) tree_patch<D, RW>(stage[step % S][cw], in, t, len, wk.n, row0, wk.c, rw * 64 + lane, wk.rb == 0, kslab, vslab);
                __syncthreads();
            }
        }
        if (step + S - 1 < steps) issue(step + S - 1);       // into the buffer that every wave has left
        if (t >= t1 || idle) return;
        const h16x8(*st)[64] = stage[step % S][cw];
        floatx16 sc;
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 2 * KT; ++kk) {
            const h16x8 k = st[sub * KT + (kk >> 1)][fl + 32 * (kk & 1)];
            if constexpr (QLO) sc = hx_mfma32(k, ql[kk], sc);
            sc = hx_mfma32(k, qf[kk], sc);
        }
        uint32_t sees = 0xffffffffu;
        if (masked) {
            sees = tree_sees(mask, tv.mask_words, t, len);
#pragma unroll
            for (int x = 0; x < 16; ++x) sc[x] = (sees >> (8 * (x >> 2) + 4 * hl + (x & 3))) & 1u ? sc[x] : NEG_INF;
        }
        const float alpha = tree_softmax(sc, m, lsum, scale_log2e);
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int x = 0; x < 16; ++x) oacc[db][x] *= alpha;
        }
        if constexpr (TAIL) {
            bool odd = false;
            if (masked) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) odd = odd || any_odd(st[2 * KT + dt][lane]);
            }
            if (__builtin_amdgcn_ballot_w64(odd) != 0) {
                tree_slow_tile<DB>(reinterpret_cast<const h16_t *>(st[2 * KT]), sc, sees, lane, oacc);
                return;
            }
        }
        TreeP p[2], lo[2];
        tree_pack(sc, p, lo);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const h16x8 v = st[2 * KT + 2 * db + sub][fl + 32 * g];
                oacc[db] = hx_mfma32(v, lo[g].v, oacc[db]);
                oacc[db] = hx_mfma32(v, p[g].v, oacc[db]);
            }
    };
    const int clean = min(max(((len >> 5) - t0) / CW, 0), steps);
    for (int step = 0; step < clean; ++step) walk(step, std::false_type{});
    for (int step = clean; step < steps; ++step) walk(step, std::true_type{});
    lsum = sum_halves(lsum);
    const int nb = wk.runs();
    const size_t part_row = (size_t)tv.rows * hq_l;
    auto finish = [&](int t, int hd, int dd, const float (&o)[4], float M, float L) {
        if (nb == 1) {
            const float inv = 1.0f / L, x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
            tree_store4(out, t, hd * D + dd, x);
            return;
        }
        const size_t e = wk.split * part_row + (size_t)t * hq_l + hd;
        *reinterpret_cast<floatx4 *>(tp.part_o + e * D + dd) = floatx4{o[0], o[1], o[2], o[3]};
        if (dd == 0) *reinterpret_cast<float2 *>(tp.part_ml + 2 * e) = float2{M, L};
    };
    if constexpr (CW == 1) {
        if (r >= R) return;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int qd = 0; qd < 4; ++qd) {
                const float x[4] = {oacc[db][4 * qd], oacc[db][4 * qd + 1], oacc[db][4 * qd + 2], oacc[db][4 * qd + 3]};
                finish(row0 + node, head, 32 * db + 8 * qd + 4 * hl, x, m, lsum);
            }
    } else {
        // the waves that shared a row group meet in LDS, in the order of their tiles
        float *s_o = reinterpret_cast<float *>(smem);
        __syncthreads();
        if (hl == 0) { s_m[wave][lane] = m; s_l[wave][lane] = lsum; }
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int qd = 0; qd < 4; ++qd)
                *reinterpret_cast<floatx4 *>(s_o + (wave * 32 + (lane & 31)) * OS + 32 * db + 8 * qd + 4 * hl) =
                    floatx4{oacc[db][4 * qd], oacc[db][4 * qd + 1], oacc[db][4 * qd + 2], oacc[db][4 * qd + 3]};
        __syncthreads();
        for (int idx = threadIdx.x; idx < ROWS * (D / 4); idx += 256) {
            const int row = idx / (D / 4), dd = 4 * (idx - row * (D / 4)), grp = row >> 5, i = row & 31, at = wk.rb * ROWS + row;
            if (at >= R) break;
            float M = NEG_INF, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < CW; ++w) M = fmaxf(M, s_m[w * RW + grp][i]);
            const float b = M == NEG_INF ? 0.f : M;
#pragma unroll
            for (int w = 0; w < CW; ++w) {
                const int wv = w * RW + grp;
                const float wt = __builtin_amdgcn_exp2f((s_m[wv][i] - b) * scale_log2e);
                const floatx4 v = *reinterpret_cast<const floatx4 *>(s_o + (wv * 32 + i) * OS + dd);
                L += s_l[wv][i] * wt;
#pragma unroll
                for (int x = 0; x < 4; ++x) o[x] += v[x] * wt;
            }
            finish(row0 + at / G, wk.c * G + at % G, dd, o, M, L);
        }
    }
}

// Joins the runs of every (row, head): D / 4 threads each, runs in the order of the context, four requested at a time.
template <int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(KvGeom kg, int hq_l, TreeView tv, const int32_t *__restrict__ lens, TreePlan tp, TreeOut out, float scale_log2e) {
    constexpr int TP = D / 4;
    const int e = blockIdx.x * (256 / TP) + threadIdx.x / TP, dd = 4 * (threadIdx.x % TP);
    if (e >= tv.rows * hq_l) return;
    const int t = e / hq_l, seq = tv.row[t].seq, n = tv.cu[seq + 1] - tv.cu[seq];
    const int nt = min((lens[seq] + n + 31) >> 5, kg.smax >> 5), per = max(tp.chunk, (nt + tp.nsplit - 1) / tp.nsplit), nb = (nt + per - 1) / per;
    if (nb <= 1) return;
    const size_t part_row = (size_t)tv.rows * hq_l;
    float M = NEG_INF, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int u0 = 0; u0 < nb; u0 += 4) {
        float2 ml[4];
        floatx4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const size_t at = min(u0 + u, nb - 1) * part_row + e;
            ml[u] = *reinterpret_cast<const float2 *>(tp.part_ml + 2 * at);
            v[u] = *reinterpret_cast<const floatx4 *>(tp.part_o + at * D + dd);
        }
        float M4 = M;
#pragma unroll
        for (int u = 0; u < 4; ++u) M4 = fmaxf(M4, ml[u].x);
        const float b = M4 == NEG_INF ? 0.f : M4, alpha = __builtin_amdgcn_exp2f((M - b) * scale_log2e);
        M = M4;
        L *= alpha;
#pragma unroll
        for (int x = 0; x < 4; ++x) o[x] *= alpha;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u0 + u >= nb) break;
            const float wt = __builtin_amdgcn_exp2f((ml[u].x - b) * scale_log2e);
            L += ml[u].y * wt;
#pragma unroll
            for (int x = 0; x < 4; ++x) o[x] += v[u][x] * wt;
        }
    }
    const float inv = 1.0f / L, x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    tree_store4(out, t, (e - t * hq_l) * D + dd, x);
}

// Few rows, or little work in all: a block of eight waves takes 32 query rows and the waves take the run's tiles in turn.  No tile serves two
// waves, so K and V go straight to registers in the operands' layout (the next tile's K is requested before this tile's softmax); the query rows, the
// same for all waves, wait in LDS (in registers they would make this kernel spill), and there the waves meet at the end.  Bound by latency, or by HBM where there are
// many sequences: d 128, one kv head of eight, one sequence of 2048 with 26 nodes 13.6 us, sixteen with 8 nodes 15.7 (1.1 TB/s), a context of a
// tile or two 8.5; eight kv heads, one sequence of 4000 with 16 nodes 17.3.  The arithmetic is that of the kernel above.
// Runs leave (m, l, o) with device-scope stores and count themselves; whoever is last joins them in the order of the context, so that the
// result does not depend on who that was, and resets the counter.  Nobody waits for anybody.
template <int D, bool QLO>
__global__ __launch_bounds__(512, 2) void tree_few_kernel(const h16_t *__restrict__ q, const h16_t *__restrict__ q_lo, int64_t ldq, TreeIn in, h16_t *kc, h16_t *vc, KvGeom kg, int hq_l, int G, int nrb,
                                                          TreeView tv, const int32_t *__restrict__ lens, TreePlan tp, TreeOut out, float scale_log2e) {
    constexpr int W = 8, KT = D / 32, DT = D / 16, DB = D / 32, OS = D + 4;
    __shared__ __align__(16) float s_o[W][32 * OS];
    __shared__ h16x8 s_q[QLO ? 2 : 1][2 * KT][64];
    __shared__ float s_m[W][32], s_l[W][32];
    __shared__ int s_last;
    TreeWork wk;
    if (!wk.find(kg, G, nrb, 32, tv, lens, tp)) return;
    const int len = wk.len, R = wk.R, row0 = wk.row0;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hl = lane >> 5, i32 = lane & 31;
    const int sub = i32 >> 4, fl = (lane & 15) + 16 * hl;
    const int rr = min(wk.rb * 32 + i32, R - 1), node = rr / G, head = wk.c * G + (rr - node * G);    // rows past the last repeat it and are not stored
    const uint32_t *mask = tv.mask + (size_t)(row0 + node) * tv.mask_words;
    const size_t slab = (size_t)wk.seq * kg.seq_stride + (size_t)wk.c * kg.smax * D;
    h16_t *kslab = kc + slab, *vslab = vc + slab;
    const bool fresh = in.k != nullptr;                       // the tree's rows are the caller's, not in the cache yet

    h16x8 kf[2 * KT], vf[2 * DB];
    const int clean = min(wk.t1, len >> 5);                   // tiles before it lie in the context
    // K: lane l takes position l % 32, elements 16 kk + 8 (l / 32) ..; a slot of the tree comes from its row
    auto load_k = [&](int t, auto tail) {
        const h16_t *src = kslab + ((size_t)(2 * t + sub) * KT * 64 + fl) * 8;
        const int x = 32 * t + i32 - len;
        if (decltype(tail)::value && fresh && x >= 0 && x < wk.n) {
            const h16_t *row = static_cast<const h16_t *>(in.k) + (size_t)(row0 + x) * in.ldk + wk.c * D + 8 * hl;
#pragma unroll
            for (int kk = 0; kk < 2 * KT; ++kk) kf[kk] = *reinterpret_cast<const h16x8 *>(row + 16 * kk);
        } else {
#pragma unroll
            for (int kk = 0; kk < 2 * KT; ++kk) kf[kk] = *reinterpret_cast<const h16x8 *>(src + ((kk >> 1) * 64 + 32 * (kk & 1)) * 8);
        }
    };
    static_assert(2 * KT <= W, "a piece of the query rows per wave");
    h16x8 qf, ql;
    const size_t q_at = (size_t)(row0 + node) * ldq + (size_t)head * D + 16 * wave + 8 * hl;
    if (wave < 2 * KT) {
        qf = *reinterpret_cast<const h16x8 *>(q + q_at);
        if constexpr (QLO) ql = *reinterpret_cast<const h16x8 *>(q_lo + q_at);
    }
    const int tw = wk.t0 + wave;
    if (tw < clean) load_k(tw, std::false_type{});
    if (wave < 2 * KT) {
        s_q[0][wave][lane] = qf;
        if constexpr (QLO) s_q[1][wave][lane] = ql;
    }
    HX_LDS_BARRIER();
    floatx16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) oacc[db][x] = 0.f;
    float m = NEG_INF, lsum = 0.f;
    // a tile in the context (TAIL false), or one that reaches the tree's slots
    auto walk = [&](int t, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if constexpr (TAIL) load_k(t, tail);
        // V^T: lane l takes element 32 db + l % 32 and k-group 2 h + l / 32 (kvlayout.h)
        const h16_t *vsrc = vslab + ((size_t)(t * DT + sub) * 64 + fl) * 8;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) vf[2 * db + h] = *reinterpret_cast<const h16x8 *>(vsrc + (2 * db * 64 + 32 * h) * 8);
        // the tree's values among them, element by element from the rows (slots of others take some row of the tree, not used), all requested at once:
        // one after the other they were most of a short call
        union Piece { h16x8 v; h16_t e[8]; uint32_t u[4]; } own[TAIL ? 2 * DB : 1];
        uint32_t sees = 0xffffffffu;
        if constexpr (TAIL) {
            if (fresh) {
                const h16_t *rows = static_cast<const h16_t *>(in.v) + (size_t)row0 * in.ldv + wk.c * D + i32;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int x = 32 * t + (j & 3) + 4 * (2 * h + hl) + 16 * (j >> 2) - len;
                        const h16_t *row = rows + min(max(x, 0), wk.n - 1) * in.ldv;
#pragma unroll
                        for (int db = 0; db < DB; ++db) own[2 * db + h].e[j] = row[32 * db];
                    }
            }
            sees = tree_sees(mask, tv.mask_words, t, len);
        }
        floatx16 sc;
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
        for (int part = QLO ? 1 : 0; part >= 0; --part) {
#pragma unroll
            for (int kk = 0; kk < 2 * KT; ++kk) sc = hx_mfma32(kf[kk], s_q[part][kk][lane], sc);
            if (part > 0) __builtin_amdgcn_sched_barrier(0);      // one part's pieces at a time in registers
        }
        if constexpr (TAIL) {
            if (fresh) {
                // over what the cache held there; the first block of rows appends what it has put together
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int x = 32 * t + 2 * (i & 1) + 4 * (2 * h + hl) + 16 * (i >> 1) - len;     // of elements 2 i and 2 i + 1
                        const uint32_t take = (x >= 0 && x < wk.n ? 0xffffu : 0u) | (x >= -1 && x < wk.n - 1 ? 0xffff0000u : 0u);
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            Piece w;
                            w.v = vf[2 * db + h];
                            w.u[i] = (own[2 * db + h].u[i] & take) | (w.u[i] & ~take);
                            vf[2 * db + h] = w.v;
                        }
                    }
                if (wk.rb == 0) {
                    const int x = 32 * t + i32 - len;
                    h16_t *dst = kslab + ((size_t)(2 * t + sub) * KT * 64 + fl) * 8;
                    if (x >= 0 && x < wk.n) {
#pragma unroll
                        for (int kk = 0; kk < 2 * KT; ++kk) *reinterpret_cast<h16x8 *>(dst + ((kk >> 1) * 64 + 32 * (kk & 1)) * 8) = kf[kk];
                    }
                    h16_t *vdst = vslab + ((size_t)(t * DT + sub) * 64 + fl) * 8;      // whole pieces: slots that are not the tree's keep their values
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int h = 0; h < 2; ++h) *reinterpret_cast<h16x8 *>(vdst + (2 * db * 64 + 32 * h) * 8) = vf[2 * db + h];
                }
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) sc[x] = (sees >> (8 * (x >> 2) + 4 * hl + (x & 3))) & 1u ? sc[x] : NEG_INF;
        }
        if (!TAIL && t + W < clean) load_k(t + W, std::false_type{});
        const float alpha = tree_softmax(sc, m, lsum, scale_log2e);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int x = 0; x < 16; ++x) oacc[db][x] *= alpha;
        if constexpr (TAIL) {
            bool odd = false;
#pragma unroll
            for (int x = 0; x < 2 * DB; ++x) odd = odd || any_odd(vf[x]);
            if (__builtin_amdgcn_ballot_w64(odd) != 0) {
                h16x8 *vt = reinterpret_cast<h16x8 *>(s_o[wave]);      // the wave's own part of the merge buffer, not in use yet
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int h = 0; h < 2; ++h) vt[(2 * db + sub) * 64 + fl + 32 * h] = vf[2 * db + h];
                tree_slow_tile<DB>(reinterpret_cast<const h16_t *>(vt), sc, sees, lane, oacc);
                return;
            }
        }
        TreeP p[2], lo[2];
        tree_pack(sc, p, lo);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                oacc[db] = hx_mfma32(vf[2 * db + g], lo[g].v, oacc[db]);
                oacc[db] = hx_mfma32(vf[2 * db + g], p[g].v, oacc[db]);
            }
    };
    int tile = tw;
    for (; tile < clean; tile += W) walk(tile, std::false_type{});
    for (; tile < wk.t1; tile += W) walk(tile, std::true_type{});
    const int live = min(W, wk.t1 - wk.t0);                   // waves that had a tile
    if (wave < live) {
        lsum = sum_halves(lsum);
        if (hl == 0) { s_m[wave][i32] = m; s_l[wave][i32] = lsum; }
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int qd = 0; qd < 4; ++qd)
                *reinterpret_cast<floatx4 *>(&s_o[wave][i32 * OS + 32 * db + 8 * qd + 4 * hl]) =
                    floatx4{oacc[db][4 * qd], oacc[db][4 * qd + 1], oacc[db][4 * qd + 2], oacc[db][4 * qd + 3]};
    }
    __syncthreads();
    const int nb = wk.runs(), rows = min(32, R - wk.rb * 32);
    const size_t part_row = (size_t)tv.rows * hq_l;
    constexpr int TP = D / 4, QUADS = 32 * TP / 512;              // threads of a row, and quads of a thread: rows threadIdx.x / TP + i 512 / TP
    const int dd = 4 * (threadIdx.x % TP);
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int row = threadIdx.x / TP + i * (512 / TP), at = wk.rb * 32 + row;
        if (row >= rows) break;
        float M = NEG_INF, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, s_m[min(w, live - 1)][row]);
        const float b = M == NEG_INF ? 0.f : M;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w >= live) break;
            const float wt = __builtin_amdgcn_exp2f((s_m[w][row] - b) * scale_log2e);
            const floatx4 v = *reinterpret_cast<const floatx4 *>(&s_o[w][row * OS + dd]);
            L += s_l[w][row] * wt;
#pragma unroll
            for (int x = 0; x < 4; ++x) o[x] += v[x] * wt;
        }
        const int t = row0 + at / G, hd = wk.c * G + at % G;
        if (nb == 1) {
            const float inv = 1.0f / L, x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
            tree_store4(out, t, hd * D + dd, x);
        } else {
            const size_t e = wk.split * part_row + (size_t)t * hq_l + hd;
            dev_store2(tp.part_o + e * D + dd, o[0], o[1]);
            dev_store2(tp.part_o + e * D + dd + 2, o[2], o[3]);
            if (dd == 0) dev_store2(tp.part_ml + 2 * e, M, L);
        }
    }
    if (nb == 1) return;
    if (!tree_arrive(tp.arrived + ((size_t)wk.seq * kg.hkv_l + wk.c) * nrb + wk.rb, nb, &s_last)) return;
    // the last block: a thread requests the (m, l) and sums of its quads of eight runs at once
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int row = threadIdx.x / TP + i * (512 / TP), at = wk.rb * 32 + row;
        if (row >= rows) break;
        const int t = row0 + at / G, hd = wk.c * G + at % G;
        const size_t e = (size_t)t * hq_l + hd;
        float M = NEG_INF, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (int u0 = 0; u0 < nb; u0 += 8) {
            float2 ml[8], a[8], b[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const size_t at_u = min(u0 + u, nb - 1) * part_row + e;
                ml[u] = dev_load2(tp.part_ml + 2 * at_u);
                a[u] = dev_load2(tp.part_o + at_u * D + dd);
                b[u] = dev_load2(tp.part_o + at_u * D + dd + 2);
            }
            float M8 = M;
#pragma unroll
            for (int u = 0; u < 8; ++u) M8 = fmaxf(M8, ml[u].x);
            const float base = M8 == NEG_INF ? 0.f : M8, alpha = __builtin_amdgcn_exp2f((M - base) * scale_log2e);
            M = M8;
            L *= alpha;
#pragma unroll
            for (int x = 0; x < 4; ++x) o[x] *= alpha;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (u0 + u >= nb) break;
                const float wt = __builtin_amdgcn_exp2f((ml[u].x - base) * scale_log2e);
                L += ml[u].y * wt;
                o[0] += a[u].x * wt; o[1] += a[u].y * wt; o[2] += b[u].x * wt; o[3] += b[u].y * wt;
            }
        }
        const float inv = 1.0f / L, x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        tree_store4(out, t, hd * D + dd, x);
    }
}

void launch_tree_attn(const h16_t *q, const h16_t *q_lo, int64_t ldq, const TreeIn &in, h16_t *kc, h16_t *vc, KvGeom kg, int hq_l, const TreeView &tv,
                      const int32_t *lens, const TreePlan &tp, const TreeOut &out, hipStream_t s) {
    const int G = hq_l / kg.hkv_l, nrb = tree_row_blocks(tv.max_n, G, 32 * tp.row_groups);
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)kg.d);
    const dim3 grid((unsigned)nrb * (unsigned)((tv.batch * kg.hkv_l * tp.nsplit + 7) / 8 * 8));
#define HX_TREE(KERNEL, THREADS) hipLaunchKernelGGL((KERNEL), grid, dim3(THREADS), 0, s, q, q_lo, ldq, in, kc, vc, kg, hq_l, G, nrb, tv, lens, tp, out, scale_log2e)
#define HX_TREE_D(DD)                                                                                                                              \
    do {                                                                                                                                           \
        if (tp.row_groups == 1) { if (q_lo != nullptr) HX_TREE((tree_few_kernel<DD, true>), 512); else HX_TREE((tree_few_kernel<DD, false>), 512); } \
        else if (tp.row_groups == 2) { if (q_lo != nullptr) HX_TREE((tree_attn_kernel<DD, 2, 2, true>), 256); else HX_TREE((tree_attn_kernel<DD, 2, 2, false>), 256); } \
        else HX_TREE((tree_attn_kernel<DD, 4, 3, false>), 256);                                                                                    \
        if (tp.row_groups > 1 && tp.nsplit > 1)                                                                                                    \
            hipLaunchKernelGGL(tree_merge_kernel<DD>, dim3((tv.rows * hq_l + 1024 / DD - 1) / (1024 / DD)), dim3(256), 0, s, kg, hq_l, tv, lens, tp, out, scale_log2e); \
    } while (0)
    if (kg.d == 128) HX_TREE_D(128);
    else HX_TREE_D(64);
#undef HX_TREE
#undef HX_TREE_D
}

// ---- keeping an accepted path -------------------------------------------------------------------------------------
// Slot len + path[j] -> len + j, in every layer.  A thread moves one element of K and of V along the whole path, eight nodes
// read before eight are written: a path only grows, so that a slot is written (j) after it was read (path[i] = j has i <= j).
__global__ __launch_bounds__(256) void tree_keep_kernel(h16_t *__restrict__ kc, h16_t *__restrict__ vc, int64_t layer_stride, KvGeom kg,
                                                        const int32_t *__restrict__ lens, const int32_t *__restrict__ cu,
                                                        const int32_t *__restrict__ kept, const int32_t *__restrict__ path) {
    const int seq = blockIdx.y, dd = (blockIdx.x * 256 + threadIdx.x) % kg.d, c = (blockIdx.x * 256 + threadIdx.x) / kg.d;
    const int n = kept[seq], len = lens[seq], row0 = cu[seq];
    if (c >= kg.hkv_l || len + n > kg.smax) return;
    const size_t slab = (size_t)blockIdx.z * layer_stride + (size_t)seq * kg.seq_stride + (size_t)c * kg.smax * kg.d;
    h16_t *ks = kc + slab, *vs = vc + slab;
    for (int j0 = 1; j0 < n; j0 += 8) {
        h16_t a[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int src = len + path[row0 + min(j0 + i, n - 1)];
            a[i] = ks[kv_k_offset(src, dd, kg.d)];
            b[i] = vs[kv_v_offset(src, dd, kg.d)];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j0 + i < n) {
                ks[kv_k_offset(len + j0 + i, dd, kg.d)] = a[i];
                vs[kv_v_offset(len + j0 + i, dd, kg.d)] = b[i];
            }
    }
}
void launch_tree_keep(h16_t *kc, h16_t *vc, int64_t layer_stride, int layers, KvGeom kg, int batch, const int32_t *lens, const int32_t *cu,
                      const int32_t *kept, const int32_t *path, hipStream_t s) {
    for (int l0 = 0; l0 < layers; l0 += 65535) {
        const dim3 grid((kg.hkv_l * kg.d + 255) / 256, batch, layers - l0 < 65535 ? layers - l0 : 65535);
        hipLaunchKernelGGL(tree_keep_kernel, grid, dim3(256), 0, s, kc + l0 * layer_stride, vc + l0 * layer_stride, layer_stride, kg, lens, cu, kept, path);
    }
}

}  // namespace HX_NS
