// Attention of drafted trees over the cache, 16-bit types: appending the trees' rows, the attention itself, the move of an accepted
// path.  Compiled once per 16-bit element type (see common.h) into namespace HX_NS.
//
// The G query heads of a kv head and the n nodes of a sequence's tree make R = n G query rows (row r: node r / G, head r % G) that
// read the same K and V, so every tile of the cache serves all of them: with 8 heads and 16 nodes the attention has 128 flops
// for every byte of the cache, between the decode kernels (8) and prefill.
#include "kernels.h"
#include "kvlayout.h"

#define NEG_INF (-INFINITY)

namespace HX_NS {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

// ---- appending ----------------------------------------------------------------------------------------------------
// rows of a user's projection -> cache slots len + index; a thread takes 8 elements of one head of K and of V
__global__ __launch_bounds__(256) void tree_append_kernel(const h16_t *__restrict__ k, int64_t ldk, const h16_t *__restrict__ v, int64_t ldv,
                                                          h16_t *__restrict__ kc, h16_t *__restrict__ vc, KvGeom kg, TreeView tv,
                                                          const int32_t *__restrict__ lens) {
    const int per_row = kg.hkv_l * kg.d / 8, idx = blockIdx.x * 256 + threadIdx.x;
    if (idx >= tv.rows * per_row) return;
    const int t = idx / per_row, e = (idx - t * per_row) * 8, c = e / kg.d, dd = e - c * kg.d;
    const TreeRow row = tv.row[t];
    const int slot = lens[row.seq] + row.index;
    if (slot >= kg.smax) return;
    const size_t slab = (size_t)row.seq * kg.seq_stride + (size_t)c * kg.smax * kg.d;
    *reinterpret_cast<uint4 *>(kc + slab + kv_k_offset(slot, dd, kg.d)) = *reinterpret_cast<const uint4 *>(k + (size_t)t * ldk + e);
    union { uint4 u; h16_t x[8]; } w;
    w.u = *reinterpret_cast<const uint4 *>(v + (size_t)t * ldv + e);
#pragma unroll
    for (int i = 0; i < 8; ++i) vc[slab + kv_v_offset(slot, dd + i, kg.d)] = w.x[i];
}
void launch_tree_append(const h16_t *k, int64_t ldk, const h16_t *v, int64_t ldv, h16_t *kc, h16_t *vc, KvGeom kg, const TreeView &tv,
                        const int32_t *lens, hipStream_t s) {
    const int n = tv.rows * (kg.hkv_l * kg.d / 8);
    hipLaunchKernelGGL(tree_append_kernel, dim3((n + 255) / 256), dim3(256), 0, s, k, ldk, v, ldv, kc, vc, kg, tv, lens);
}

// The stage's fused projection, raw fp32 [rows][N] -> rotary embedding at len + depth, q as plain rows, k and v into the cache.
// The projection's columns are in the order of its packed tiles: 16 columns hold elements 8 tl .. 8 tl + 7 of a head and those half a
// head further.  A thread takes four rotary pairs.  q is rounded to the element type here, once, as in the prefill path.
__global__ __launch_bounds__(256) void tree_rope_append_kernel(const float *__restrict__ qkv, int hq_l, KvGeom kg, TreeView tv,
                                                               const int32_t *__restrict__ lens, const float *__restrict__ cos_tab,
                                                               const float *__restrict__ sin_tab, h16_t *__restrict__ q,
                                                               h16_t *__restrict__ kc, h16_t *__restrict__ vc) {
    const int d = kg.d, half = d >> 1, tph = d >> 4, heads = hq_l + 2 * kg.hkv_l, per_row = heads * tph * 2;
    const int idx = blockIdx.x * 256 + threadIdx.x;
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
    union { uint2 u; h16_t x[4]; } a, b;
    a.u = uint2{pack_h16x2(lo[0], lo[1]), pack_h16x2(lo[2], lo[3])};
    b.u = uint2{pack_h16x2(hi[0], hi[1]), pack_h16x2(hi[2], hi[3])};
    if (head < hq_l) {
        h16_t *dst = q + ((size_t)t * hq_l + head) * d;
        *reinterpret_cast<uint2 *>(dst + i0) = a.u;
        *reinterpret_cast<uint2 *>(dst + half + i0) = b.u;
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
                             const float *sin_tab, h16_t *q, h16_t *kc, h16_t *vc, hipStream_t s) {
    const int n = tv.rows * (hq_l + 2 * kg.hkv_l) * (kg.d >> 4) * 2;
    hipLaunchKernelGGL(tree_rope_append_kernel, dim3((n + 255) / 256), dim3(256), 0, s, qkv, hq_l, kg, tv, lens, cos_tab, sin_tab, q, kc, vc);
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

// A block of four waves takes 32 RW query rows of one (sequence, kv head) and a run of 32-position tiles; RW groups of 32 rows times
// CW = 4 / RW neighbouring tiles a step.  The tiles go from HBM to LDS directly, S steps in flight, and S^T = K . Q^T,
// O^T = V^T . P^T run on the 32 x 32 x 16 MFMA exactly as in the prefill attention: a lane owns one query row, P stays in its
// registers and is rounded to the element type for the second product (2^-9 per weight for bf16, against 2^-9 of the rounded result;
// the weights' sum takes them unrounded).
// Tiles that lie in the context need no mask; of a tile that reaches the tree's slots a lane takes 32 bits of its node's ancestors.
// A weight of zero times an infinity would be a NaN, so a masked tile with a value that is not finite is multiplied out element
// by element over what each row attends.
// A long context is cut into runs of sp.chunk tiles (sp.nsplit at most), whose (m, l, o) tree_merge_kernel joins in their order.
template <int D, int RW, int S>
__global__ __launch_bounds__(256, RW == 1 ? 1 : 2) void tree_attn_kernel(const h16_t *__restrict__ q, int64_t ldq, const h16_t *__restrict__ kc,
                                                                         const h16_t *__restrict__ vc, KvGeom kg, int hq_l, int G, int nrb,
                                                                         TreeView tv, const int32_t *__restrict__ lens, TreeSplit sp,
                                                                         TreeOut out, float scale_log2e) {
    constexpr int CW = 4 / RW, ROWS = 32 * RW;
    constexpr int KT = D / 32, DT = D / 16, DB = D / 32, TILES = 2 * KT + DT;
    constexpr int LPT = TILES / RW;                       // 1 KB loads per wave and step: RW waves share a tile position
    constexpr int OS = D + 4;                             // floats between rows of the merge buffer: eight rows on distinct banks
    constexpr int STAGE = S * CW * TILES * 1024, MERGE = CW > 1 ? 4 * 32 * OS * 4 : 0;
    __shared__ __align__(16) unsigned char smem[STAGE > MERGE ? STAGE : MERGE];
    __shared__ float s_m[4][32], s_l[4][32];
    h16x8(*stage)[CW][TILES][64] = reinterpret_cast<h16x8(*)[CW][TILES][64]>(smem);
    // block id = 8 slot + xcd: the row blocks of a run of tiles sit next to each other on one XCD and share the run in its L2
    const int slot = blockIdx.x >> 3, rb = slot % nrb;
    int combo = (slot / nrb) * 8 + (blockIdx.x & 7);
    if (combo >= tv.batch * kg.hkv_l * sp.nsplit) return;
    const int split = combo % sp.nsplit;
    combo /= sp.nsplit;
    const int c = combo % kg.hkv_l, seq = combo / kg.hkv_l;
    const int row0 = tv.cu[seq], n = tv.cu[seq + 1] - row0, R = n * G;
    if (rb * ROWS >= R) return;
    const int len = lens[seq], nt = min((len + n + 31) >> 5, kg.smax >> 5);
    const int per = max(sp.chunk, (nt + sp.nsplit - 1) / sp.nsplit), t0 = split * per;
    if (t0 >= nt) return;
    const int t1 = min(t0 + per, nt), steps = (t1 - t0 + CW - 1) / CW;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int rw = wave % RW, cw = wave / RW, hl = lane >> 5;
    const int r = rb * ROWS + rw * 32 + (lane & 31);
    const int rr = min(r, R - 1), node = rr / G, head = c * G + (rr - node * G);    // rows past the last repeat it and are not stored
    const uint32_t *mask = tv.mask + (size_t)(row0 + node) * tv.mask_words;

    h16x8 qf[2 * KT];
#pragma unroll
    for (int kk = 0; kk < 2 * KT; ++kk)
        qf[kk] = *reinterpret_cast<const h16x8 *>(q + (size_t)(row0 + node) * ldq + (size_t)head * D + 16 * kk + 8 * hl);
    floatx16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) oacc[db][x] = 0.f;
    float m = NEG_INF, lsum = 0.f;

    const size_t slab = (size_t)seq * kg.seq_stride + (size_t)c * kg.smax * D;
    const h16x8 *ks = reinterpret_cast<const h16x8 *>(kc + slab), *vs = reinterpret_cast<const h16x8 *>(vc + slab);
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
    for (int step = 0; step < steps; ++step) {
        // steps step + 1 .. step + S - 2 may stay in flight
        if (S > 2 && step + 1 < steps) HX_WAIT_VM(LPT);
        else HX_WAIT_VM(0);
        HX_LDS_BARRIER();
        if (step + S - 1 < steps) issue(step + S - 1);       // into the buffer that every wave has left
        const int t = t0 + step * CW + cw;
        if (t >= t1) continue;
        const h16x8(*st)[64] = stage[step % S][cw];
        floatx16 sc;
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 2 * KT; ++kk) sc = hx_mfma32(st[sub * KT + (kk >> 1)][fl + 32 * (kk & 1)], qf[kk], sc);
        const bool masked = 32 * t + 31 >= len;
        uint32_t sees = 0xffffffffu;
        if (masked) {
            const int rel = 32 * t - len;                    // index in the tree of the tile's first slot; negative: context before it
            if (rel < 0) {
                sees = (mask[0] << -rel) | ((1u << -rel) - 1);
            } else {
                const int w = rel >> 5, sh = rel & 31;
                const uint32_t a = w < tv.mask_words ? mask[w] : 0u, b = w + 1 < tv.mask_words ? mask[w + 1] : 0u;
                sees = sh == 0 ? a : (a >> sh) | (b << (32 - sh));
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) sc[x] = (sees >> (8 * (x >> 2) + 4 * hl + (x & 3))) & 1u ? sc[x] : NEG_INF;
        }
        float mx = NEG_INF;
#pragma unroll
        for (int x = 0; x < 16; ++x) mx = fmaxf(mx, sc[x]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx);
        const float base = m_new == NEG_INF ? 0.f : m_new;   // a row that has seen nothing yet: weights 0, no NaN
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
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int x = 0; x < 16; ++x) oacc[db][x] *= alpha;
        }
        bool odd = false;
        if (masked) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) odd = odd || any_odd(st[2 * KT + dt][lane]);
        }
        if (__builtin_amdgcn_ballot_w64(odd) == 0) {
            union { uint32_t u[4]; h16x8 v; } p0, p1;        // P for k-groups hl (quads 0, 2) and 2 + hl (quads 1, 3)
            p0.u[0] = pack_h16x2(sc[0], sc[1]);   p0.u[1] = pack_h16x2(sc[2], sc[3]);
            p0.u[2] = pack_h16x2(sc[8], sc[9]);   p0.u[3] = pack_h16x2(sc[10], sc[11]);
            p1.u[0] = pack_h16x2(sc[4], sc[5]);   p1.u[1] = pack_h16x2(sc[6], sc[7]);
            p1.u[2] = pack_h16x2(sc[12], sc[13]); p1.u[3] = pack_h16x2(sc[14], sc[15]);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                oacc[db] = hx_mfma32(st[2 * KT + 2 * db + sub][fl], p0.v, oacc[db]);
                oacc[db] = hx_mfma32(st[2 * KT + 2 * db + sub][fl + 32], p1.v, oacc[db]);
            }
        } else {
            const h16_t *vt = reinterpret_cast<const h16_t *>(st[2 * KT]);
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
    }
    lsum += __shfl_xor(lsum, 32, 64);
    const int nb = (nt + per - 1) / per;
    const size_t part_row = (size_t)tv.rows * hq_l;
    auto finish = [&](int t, int hd, int dd, const float (&o)[4], float M, float L) {
        if (nb == 1) {
            const float inv = 1.0f / L, x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
            tree_store4(out, t, hd * D + dd, x);
            return;
        }
        const size_t e = split * part_row + (size_t)t * hq_l + hd;
        *reinterpret_cast<floatx4 *>(sp.part_o + e * D + dd) = floatx4{o[0], o[1], o[2], o[3]};
        if (dd == 0) *reinterpret_cast<float2 *>(sp.part_ml + 2 * e) = float2{M, L};
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
            const int row = idx / (D / 4), dd = 4 * (idx - row * (D / 4)), grp = row >> 5, i = row & 31, at = rb * ROWS + row;
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
            finish(row0 + at / G, c * G + at % G, dd, o, M, L);
        }
    }
}

// Joins the runs of every (row, head): D / 4 threads each, runs in the order of the context.
template <int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(KvGeom kg, int hq_l, TreeView tv, const int32_t *__restrict__ lens, TreeSplit sp,
                                                         TreeOut out, float scale_log2e) {
    constexpr int TP = D / 4;
    const int e = blockIdx.x * (256 / TP) + threadIdx.x / TP, dd = 4 * (threadIdx.x % TP);
    if (e >= tv.rows * hq_l) return;
    const int t = e / hq_l, seq = tv.row[t].seq, n = tv.cu[seq + 1] - tv.cu[seq];
    const int nt = min((lens[seq] + n + 31) >> 5, kg.smax >> 5), per = max(sp.chunk, (nt + sp.nsplit - 1) / sp.nsplit), nb = (nt + per - 1) / per;
    if (nb <= 1) return;
    const size_t part_row = (size_t)tv.rows * hq_l;
    float M = NEG_INF;
    for (int u = 0; u < nb; ++u) M = fmaxf(M, sp.part_ml[2 * (u * part_row + e)]);
    const float b = M == NEG_INF ? 0.f : M;
    float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int u = 0; u < nb; ++u) {
        const float2 ml = *reinterpret_cast<const float2 *>(sp.part_ml + 2 * (u * part_row + e));
        const float wt = __builtin_amdgcn_exp2f((ml.x - b) * scale_log2e);
        const floatx4 v = *reinterpret_cast<const floatx4 *>(sp.part_o + (u * part_row + e) * D + dd);
        L += ml.y * wt;
#pragma unroll
        for (int x = 0; x < 4; ++x) o[x] += v[x] * wt;
    }
    const float inv = 1.0f / L, x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    tree_store4(out, t, (e - t * hq_l) * D + dd, x);
}

void launch_tree_attn(const h16_t *q, int64_t ldq, const h16_t *kc, const h16_t *vc, KvGeom kg, int hq_l, const TreeView &tv,
                      const int32_t *lens, const TreeSplit &sp, const TreeOut &out, hipStream_t s) {
    const int G = hq_l / kg.hkv_l, groups = tree_row_groups(tv.max_n, G), nrb = (tv.max_n * G + 32 * groups - 1) / (32 * groups);
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)kg.d);
    const dim3 grid((unsigned)nrb * (unsigned)((tv.batch * kg.hkv_l * sp.nsplit + 7) / 8 * 8));
#define HX_TREE(DD, RW, S) hipLaunchKernelGGL((tree_attn_kernel<DD, RW, S>), grid, dim3(256), 0, s, q, ldq, kc, vc, kg, hq_l, G, nrb, tv, lens, sp, out, scale_log2e)
    if (kg.d == 128) {
        if (groups == 1) HX_TREE(128, 1, 2);
        else if (groups == 2) HX_TREE(128, 2, 2);
        else HX_TREE(128, 4, 3);
    } else {
        if (groups == 1) HX_TREE(64, 1, 2);
        else if (groups == 2) HX_TREE(64, 2, 2);
        else HX_TREE(64, 4, 3);
    }
#undef HX_TREE
    if (sp.nsplit <= 1) return;
    if (kg.d == 128) hipLaunchKernelGGL(tree_merge_kernel<128>, dim3((tv.rows * hq_l + 7) / 8), dim3(256), 0, s, kg, hq_l, tv, lens, sp, out, scale_log2e);
    else hipLaunchKernelGGL(tree_merge_kernel<64>, dim3((tv.rows * hq_l + 15) / 16), dim3(256), 0, s, kg, hq_l, tv, lens, sp, out, scale_log2e);
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
