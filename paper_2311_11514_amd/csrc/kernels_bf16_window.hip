// Attention of new rows over the cache with a sliding window and first positions that stay visible, 16-bit types: appending the rows, the attention, the
// sums of its weights, and the move of what an eviction keeps.  Compiled once per 16-bit element type (see common.h) into namespace HX_NS.
//
// The G query heads of a kv head and the n new rows of a sequence make R = n G query rows (row r: new row r / G, head r % G) that share the tiles of the
// cache, as the nodes of a drafted tree do; here a row attends slots j <= p with p - j < window or j < sinks, so that blocks of rows have tile lists
// of their own (WinTiles), most of them without a mask.
#include <algorithm>
#include <type_traits>

#include "attn_rows.h"
#include "window.h"

namespace HX_NS {

// ---- appending ------------------------------------------------------------------------------------------------------
// The stage's fused projection, raw fp32 [rows][N], columns in the order of its packed tiles -> rotary embedding at len + row, q as plain rows (in two parts
// where q_lo is given), k and v into the cache.  A thread takes four rotary pairs.
__global__ __launch_bounds__(256) void win_rope_append_kernel(const float *__restrict__ qkv, int hq_l, KvGeom kg, WinCall wc, const int32_t *__restrict__ lens,
                                                              const float *__restrict__ cos_tab, const float *__restrict__ sin_tab, h16_t *__restrict__ q,
                                                              h16_t *__restrict__ q_lo, h16_t *__restrict__ kc, h16_t *__restrict__ vc) {
    const int d = kg.d, half = d >> 1, tph = d >> 4, heads = hq_l + 2 * kg.hkv_l;
    const unsigned idx = blockIdx.x * 256u + threadIdx.x, per_row = heads * tph * 2;
    const int first = wc.cu[0], t = first + (int)(idx / per_row), rem = idx % per_row, head = rem / (2 * tph), tl = (rem >> 1) % tph, i0 = 8 * tl + 4 * (rem & 1);
    if (t >= wc.cu[wc.batch]) return;
    int lo_seq = 0, hi_seq = wc.batch;                        // the last sequence whose first row is not behind t
    while (hi_seq - lo_seq > 1) {
        const int mid = (lo_seq + hi_seq) >> 1;
        if (wc.cu[mid] <= t) lo_seq = mid;
        else hi_seq = mid;
    }
    const int seq = wc.seq0 + lo_seq, slot = lens[seq] + t - wc.cu[lo_seq];
    if (slot >= wc.max_seq) return;
    const float *src = qkv + (size_t)t * heads * d + (size_t)(head * tph + tl) * 16 + 4 * (rem & 1);
    floatx4 lo = *reinterpret_cast<const floatx4 *>(src), hi = *reinterpret_cast<const floatx4 *>(src + 8);
    if (head < hq_l + kg.hkv_l) {
        const size_t at = (size_t)slot * half + i0;
        const floatx4 c4 = *reinterpret_cast<const floatx4 *>(cos_tab + at), s4 = *reinterpret_cast<const floatx4 *>(sin_tab + at);
        const floatx4 l = lo * c4 - hi * s4;
        hi = hi * c4 + lo * s4;
        lo = l;
    }
    union { uint2 u; h16_t x[4]; } a, b, al, bl;             // the element type's parts of both halves' four elements, and what they leave
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
    const size_t slab = (size_t)seq * kg.seq_stride + (size_t)(head - hq_l - (key ? 0 : kg.hkv_l)) * kg.smax * d;
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
void launch_win_rope_append(const float *qkv, int hq_l, KvGeom kg, const WinCall &wc, const int32_t *lens, const float *cos_tab, const float *sin_tab,
                            h16_t *q, h16_t *q_lo, h16_t *kc, h16_t *vc, hipStream_t s) {
    const unsigned n = (unsigned)(wc.cu[wc.batch] - wc.cu[0]) * (hq_l + 2 * kg.hkv_l) * (kg.d >> 4) * 2;
    hipLaunchKernelGGL(win_rope_append_kernel, dim3((n + 255) / 256), dim3(256), 0, s, qkv, hq_l, kg, wc, lens, cos_tab, sin_tab, q, q_lo, kc, vc);
}

// Plain rows into the cache, a block per tile of 32 slots: K in pieces of 16 bytes, V through LDS, so that the tile's transposed pieces are written whole.
// Bound by HBM: 4096 rows of 8 kv heads, d 128, 8.9 us (3.8 TB/s read and written).
template <int D>
__global__ __launch_bounds__(256) void win_append_kernel(TreeIn in, h16_t *__restrict__ kc, h16_t *__restrict__ vc, KvGeom kg, WinCall wc, const int32_t *__restrict__ lens) {
    constexpr int P8 = D / 8, PIECES = 32 * P8 / 256;
    __shared__ __align__(16) h16_t s_v[32][D + 8];
    const int nth = blockIdx.z, seq = wc.seq0 + nth, c = blockIdx.y, row0 = wc.cu[nth], len = lens[seq];
    const int n = min(wc.cu[nth + 1] - row0, wc.max_seq - len), t = (len >> 5) + blockIdx.x;
    if (32 * t >= len + n || n <= 0) return;
    const size_t slab = (size_t)seq * kg.seq_stride + (size_t)c * kg.smax * D;
    uint4 k[PIECES], v[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int idx = threadIdx.x + 256 * i, e = c * D + 8 * (idx % P8), x = min(max(32 * t + idx / P8 - len, 0), n - 1);
        k[i] = *reinterpret_cast<const uint4 *>(static_cast<const h16_t *>(in.k) + (size_t)(row0 + x) * in.ldk + e);
        v[i] = *reinterpret_cast<const uint4 *>(static_cast<const h16_t *>(in.v) + (size_t)(row0 + x) * in.ldv + e);
    }
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int idx = threadIdx.x + 256 * i, pos = idx / P8, dd = 8 * (idx % P8), x = 32 * t + pos - len;
        *reinterpret_cast<uint4 *>(&s_v[pos][dd]) = v[i];
        if (x >= 0 && x < n) *reinterpret_cast<uint4 *>(kc + slab + kv_k_offset(32 * t + pos, dd, D)) = k[i];
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 4 * D; idx += 256) {
        const int dd = idx % D, g = idx / D;                  // kvlayout.h: positions 4 g .. 4 g + 3 and 16 + 4 g .. + 3 of element dd are 16 bytes
        union { uint4 u; h16_t e[8]; } w;
        bool whole = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int pos = 4 * g + (j & 3) + 16 * (j >> 2), x = 32 * t + pos - len;
            w.e[j] = s_v[pos][dd];
            whole = whole && x >= 0 && x < n;
        }
        h16_t *dst = vc + slab + kv_v_offset(32 * t + 4 * g, dd, D);
        if (whole) {
            *reinterpret_cast<uint4 *>(dst) = w.u;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int x = 32 * t + 4 * g + (j & 3) + 16 * (j >> 2) - len;
                if (x >= 0 && x < n) dst[j] = w.e[j];
            }
        }
    }
}
void launch_win_append(const TreeIn &in, h16_t *kc, h16_t *vc, KvGeom kg, const WinCall &wc, const int32_t *lens, hipStream_t s) {
    const dim3 grid(wc.max_n / 32 + 2, kg.hkv_l, wc.batch);  // a sequence's rows may begin and end inside a tile
    if (kg.d == 128) hipLaunchKernelGGL(win_append_kernel<128>, grid, dim3(256), 0, s, in, kc, vc, kg, wc, lens);
    else hipLaunchKernelGGL(win_append_kernel<64>, grid, dim3(256), 0, s, in, kc, vc, kg, wc, lens);
}

// ---- statistics -------------------------------------------------------------------------------------------------------
// What a row's softmax is relative to.  In blocks that share tiles its weights are exp2(s c - base), c = log2(e) / sqrt(d), one multiply-add a score, with base = the
// rounded product of c and a score near the largest: the same number in the sum, in what is rescaled and in the weights' sums later, so that its rounding
// cancels.  From 2^20 on, where it would not (a product's last bit is 1/8 there, and from 2^31 on an exponent could overflow), and in blocks of few rows the
// difference of the scores is taken first.  Statistics say which: 1 / sum with its sign changed stands beside a base that is a score.
constexpr float kWinFarBase = 1048576.0f;
__device__ __forceinline__ float2 win_stat(float base, float inv, bool score) { return float2{base, score ? -inv : inv}; }
// a weight from a score: exp2((s - a) c - b) / sum
struct WinBase {
    float a, b, inv;
    __device__ __forceinline__ WinBase(float base, float given) : a(given < 0.f ? base : 0.f), b(given < 0.f ? 0.f : base), inv(fabsf(given)) {}
    __device__ __forceinline__ float exp(float s, float scale_log2e) const { return __builtin_amdgcn_exp2f(fmaf(s - a, scale_log2e, -b)); }
    // its sum is an infinity or a NaN: what the row does not attend (a score of -infinity) must not take part, not even as zero times that
    __device__ __forceinline__ bool odd() const { return !(inv < INFINITY); }
    __device__ __forceinline__ float add(float sum, float s, float scale_log2e, bool careful) const {
        const float e = exp(s, scale_log2e);
        return !careful ? fmaf(e, inv, sum) : s == NEG_INF ? sum : sum + e * inv;
    }
};

// ---- attention, few rows ----------------------------------------------------------------------------------------------
// A block of eight waves takes 32 query rows and a run of their tiles, which the waves take in turn, K and V straight to registers in the operands'
// layout (the next unmasked tile's K is requested before this tile's softmax); the waves meet in LDS.  S^T = K . Q^T and O^T = V^T . P^T with P in
// two parts (tree_pack2).  Rows that are not in the cache yet (in.k != NULL: a sequence's rows are one block's then) are put over the tile and appended by
// the run that holds their tile.  Runs leave (m, l, o) with device-scope stores; the last to arrive joins them in the order of the context.
// A weight of zero times an infinity would be a NaN: a masked tile with a value that is not finite is multiplied out over what each row attends.
// Unmasked tiles come first (WinTiles), in a loop of their own: with masked and unmasked ones in one the compiler spilled 126 registers.
// Bound by HBM where there are many sequences, by the chain launch, rows, tiles, joining where there are few: d 128, one row each, 8 heads a kv head: 32 contexts of
// 240 .. 4027 under a window of 2048, 8 kv heads, 38.6 us (5.5 TB/s), 43.2 with the scores for the weights' sums (14 MB); one sequence, one kv head, window 1024 10.8;
// sixteen of 2048, one kv head, 10.9.
template <int D, bool QLO>
__global__ __launch_bounds__(512, 2) void win_few_kernel(const h16_t *__restrict__ q, const h16_t *__restrict__ q_lo, int64_t ldq, TreeIn in, h16_t *kc, h16_t *vc,
                                                         KvGeom kg, int hq_l, int G, int nrb, WinCall wc, const int32_t *__restrict__ lens, WinPlan wp, TreeOut out,
                                                         float scale_log2e) {
    constexpr int W = 8, KT = D / 32, DT = D / 16, DB = D / 32, OS = D + 4;
    __shared__ __align__(16) float s_o[W][32 * OS];
    __shared__ h16x8 s_q[QLO ? 2 : 1][2 * KT][64];
    __shared__ float s_m[W][32], s_l[W][32];
    __shared__ int s_last;
    WinWork wk;
    const bool fresh = in.k != nullptr;
    if (!wk.find(kg.hkv_l, G, nrb, 32, wc, lens, wp, fresh)) return;
    const int len = wk.len, R = wk.R, row0 = wk.row0;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hl = lane >> 5, i32 = lane & 31;
    const int sub = i32 >> 4, fl = (lane & 15) + 16 * hl;
    const int rr = min(wk.rb * 32 + i32, R - 1), node = rr / G, head = wk.c * G + (rr - node * G);    // rows past the last repeat it and are not stored
    const int qpos = len + node;
    const size_t slab = (size_t)wk.seq * kg.seq_stride + (size_t)wk.c * kg.smax * D;
    h16_t *kslab = kc + slab, *vslab = vc + slab;
    h16x8 kf[2 * KT], vf[2 * DB];
    const int clean = min(wk.v1, wk.tiles.clean);
    // K: lane l takes position l % 32, elements 16 kk + 8 (l / 32) ..; a new row's slot comes from the row
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
    int v = wk.v0 + wave;
    if (v < clean) load_k(wk.tiles.at(v), std::false_type{});
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
    // a tile that every row attends and the cache holds (TAIL false), or one that needs a mask or new rows
    auto walk = [&](int t, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if constexpr (TAIL) load_k(t, tail);
        const bool patch = TAIL && fresh && 32 * t + 31 >= len;     // the same in every lane
        // V^T: lane l takes element 32 db + l % 32 and k-group 2 h + l / 32 (kvlayout.h)
        const h16_t *vsrc = vslab + ((size_t)(t * DT + sub) * 64 + fl) * 8;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int h = 0; h < 2; ++h) vf[2 * db + h] = *reinterpret_cast<const h16x8 *>(vsrc + (2 * db * 64 + 32 * h) * 8);
        // the new rows' values among them, all requested at once (slots of others take some row, not used)
        union Piece { h16x8 v; h16_t e[8]; uint32_t u[4]; } own[TAIL ? 2 * DB : 1];
        uint32_t sees = 0xffffffffu;
        if constexpr (TAIL) {
            if (patch) {
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
            sees = win_sees(32 * t, qpos, wc.window, wc.sinks);
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
            if (patch) {
                // over what the cache held there, which gets what has been put together
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
                const int x = 32 * t + i32 - len;
                h16_t *dst = kslab + ((size_t)(2 * t + sub) * KT * 64 + fl) * 8;
                if (x >= 0 && x < wk.n) {
#pragma unroll
                    for (int kk = 0; kk < 2 * KT; ++kk) *reinterpret_cast<h16x8 *>(dst + ((kk >> 1) * 64 + 32 * (kk & 1)) * 8) = kf[kk];
                }
                h16_t *vdst = vslab + ((size_t)(t * DT + sub) * 64 + fl) * 8;      // whole pieces: slots that are not the rows' keep their values
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int h = 0; h < 2; ++h) *reinterpret_cast<h16x8 *>(vdst + (2 * db * 64 + 32 * h) * 8) = vf[2 * db + h];
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) sc[x] = (sees >> (8 * (x >> 2) + 4 * hl + (x & 3))) & 1u ? sc[x] : NEG_INF;
        }
        if (!TAIL && v + W < clean) load_k(wk.tiles.at(v + W), std::false_type{});
        if (wp.scores != nullptr && wk.rb * 32 + i32 < R) {   // for the weights' sums: four positions of the lane's row a store
            float *dst = wp.scores + ((size_t)(row0 + node) * hq_l + head) * 32 * wp.score_tiles + 32 * v + 4 * hl;
#pragma unroll
            for (int qd = 0; qd < 4; ++qd) *reinterpret_cast<floatx4 *>(dst + 8 * qd) = floatx4{sc[4 * qd], sc[4 * qd + 1], sc[4 * qd + 2], sc[4 * qd + 3]};
        }
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
    for (; v < clean; v += W) walk(wk.tiles.at(v), std::false_type{});
    for (; v < wk.v1; v += W) walk(wk.tiles.at(v), std::true_type{});
    const int live = min(W, wk.v1 - wk.v0);                   // waves that had a tile
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
    const size_t part_row = (size_t)wc.rows * hq_l;
    constexpr int TP = D / 4, QUADS = 32 * TP / 512;              // threads of a row, and quads of a thread: rows threadIdx.x / TP + i 512 / TP
    const int dd = 4 * (threadIdx.x % TP);
    auto finish = [&](int t, int hd, const float (&o)[4], float M, float L) {
        const float inv = 1.0f / L, x[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
        tree_store4(out, t, hd * D + dd, x);
        if (wp.stat != nullptr && dd == 0) *reinterpret_cast<float2 *>(wp.stat + 2 * ((size_t)t * hq_l + hd)) = win_stat(M, inv * kWeightUnit, true);
    };
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
            const floatx4 x4 = *reinterpret_cast<const floatx4 *>(&s_o[w][row * OS + dd]);
            L += s_l[w][row] * wt;
#pragma unroll
            for (int x = 0; x < 4; ++x) o[x] += x4[x] * wt;
        }
        const int t = row0 + at / G, hd = wk.c * G + at % G;
        if (nb == 1) {
            finish(t, hd, o, M, L);
        } else {
            const size_t e = wk.split * part_row + (size_t)t * hq_l + hd;
            dev_store2(wp.part_o + e * D + dd, o[0], o[1]);
            dev_store2(wp.part_o + e * D + dd + 2, o[2], o[3]);
            if (dd == 0) dev_store2(wp.part_ml + 2 * e, M, L);
        }
    }
    if (nb == 1) return;
    if (!tree_arrive(wp.arrived + ((size_t)wk.nth * kg.hkv_l + wk.c) * nrb + wk.rb, nb, &s_last)) return;
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
                ml[u] = dev_load2(wp.part_ml + 2 * at_u);
                a[u] = dev_load2(wp.part_o + at_u * D + dd);
                b[u] = dev_load2(wp.part_o + at_u * D + dd + 2);
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
        finish(t, hd, o, M, L);
    }
}

// ---- attention, many rows ---------------------------------------------------------------------------------------------
// A block of four waves takes 128 query rows, 32 a wave; their tiles go from HBM to LDS directly, four buffers deep, and are shared.  The rows are in the cache
// already.  S^T = K . Q^T, O^T = V^T . P^T on the 32 x 32 x 16 MFMA, P in registers, in two parts as in blocks of few rows, so that a row is as exact whatever rows its
// call has besides.  (Rounded once, as in the prefill attention, results are a third less exact, RMS against 64 bits 2.1e-3 instead of 1.6e-3 in bf16, and a call of 4096 rows
// under a window of 1024 takes 166 us instead of 211, one of 8 x 512 rows that gathers weights 360 instead of 425.)
// While the vector unit works on a tile's weights the matrix cores have the next tile's scores.  Bound by each wave's chain of LDS reads, products and softmax, 1.7 waves
// a SIMD (240 registers): matrix cores 42 % busy, vector units 47 %.  A wave's second product beside the packing of its other half, by order or by scheduling groups, is no faster.
// d 128, 64 query and 8 kv heads, 4096 rows under a window of 1024: of launches on their own, as a profiler has them, 237 us, the smallest 217 (556 TFLOP/s over the pairs that are
// attended; calls one behind another 211 with the append); 8 x 512 rows at 1000 .. 3500, 32 / 4 heads, 284 and 268 (647).
template <int D>
__global__ __launch_bounds__(256, 2) void win_attn_kernel(const h16_t *__restrict__ q, int64_t ldq, const h16_t *__restrict__ kc, const h16_t *__restrict__ vc, KvGeom kg,
                                                          int hq_l, int G, int nrb, WinCall wc, const int32_t *__restrict__ lens, WinPlan wp, TreeOut out,
                                                          float scale_log2e) {
    constexpr int RW = 4, S = 4, ROWS = 32 * RW;
    constexpr int KT = D / 32, DT = D / 16, DB = D / 32, TILES = 2 * KT + DT;
    constexpr int LPT = TILES / RW;                       // 1 KB loads per wave and step
    __shared__ h16x8 stage[S][TILES][64];
    WinWork wk;
    if (!wk.find(kg.hkv_l, G, nrb, ROWS, wc, lens, wp, false)) return;
    const int len = wk.len, R = wk.R, row0 = wk.row0, steps = wk.tiles.nt;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hl = lane >> 5;
    const int r = wk.rb * ROWS + wave * 32 + (lane & 31);
    const int rr = min(r, R - 1), node = rr / G, head = wk.c * G + (rr - node * G);    // rows past the last repeat it and are not stored
    const int qpos = len + node;
    const int r0w = wk.rb * ROWS + wave * 32;             // the wave's slots; none if it has no row: it feeds the others
    const bool idle = r0w >= R;

    h16x8 qf[2 * KT];
#pragma unroll
    for (int kk = 0; kk < 2 * KT; ++kk) qf[kk] = *reinterpret_cast<const h16x8 *>(q + (size_t)(row0 + node) * ldq + (size_t)head * D + 16 * kk + 8 * hl);
    floatx16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 16; ++x) oacc[db][x] = 0.f;
    float m = NEG_INF, base = 0.f, lsum = 0.f;            // the score that the base was taken from, and the base (win_stat)
    bool far = false;                                     // of some row of the wave: the base is that score itself
    // Weights are carried times 2^SHIFT (kWeightShift), up to 2^SLACK of that above the base: fp16's largest number is just below 2^16
    constexpr float SHIFT = kWeightShift > 0.f ? kWeightShift - 1.f : 0.f, UNIT = kWeightShift > 0.f ? 0.5f * kWeightUnit : 1.f, SLACK = kWeightShift > 0.f ? 2.f : 8.f;
    const float slack = SLACK / scale_log2e;

    const size_t slab = (size_t)wk.seq * kg.seq_stride + (size_t)wk.c * kg.smax * D;
    const h16x8 *ks = reinterpret_cast<const h16x8 *>(kc + slab), *vs = reinterpret_cast<const h16x8 *>(vc + slab);
    const unsigned lane_bytes = (unsigned)lane * 16u;
    auto issue = [&](int step) {
        const int t = wk.tiles.at(step);
#pragma unroll
        for (int x = 0; x < LPT; ++x) {
            const int tile = wave + RW * x;
            const h16x8 *src = tile < 2 * KT ? ks + (size_t)(2 * t * KT + tile) * 64 : vs + (size_t)(t * DT + tile - 2 * KT) * 64;
            hx_load_lds16(hx_lds_addr(&stage[step % S][tile][0]), lane_bytes, src);
        }
    };
    const int sub = (lane & 31) >> 4, fl = (lane & 15) + 16 * hl;
    HX_WAIT_VM(0);            // the query rows have landed before the first load that the compiler does not see
    issue(0);
    if (steps > 1) issue(1);
    if (steps > 2) issue(2);
    auto scores = [&](int step, floatx16 &sc) {
        const h16x8(*st)[64] = stage[step % S];
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = 0.f;
#pragma unroll
        for (int kk = 0; kk < 2 * KT; ++kk) sc = hx_mfma32(st[sub * KT + (kk >> 1)][fl + 32 * (kk & 1)], qf[kk], sc);
    };
    if (steps > 2) HX_WAIT_VM(2 * LPT);
    else if (steps > 1) HX_WAIT_VM(LPT);
    else HX_WAIT_VM(0);
    HX_LDS_BARRIER();
    floatx16 sc;
    scores(0, sc);
    // a step whose tile every row of the block attends (TAIL false), or one that needs a mask; sc holds its scores
    auto walk = [&](int step, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if (step + 2 < steps) HX_WAIT_VM(LPT);            // step + 2 may stay in flight
        else HX_WAIT_VM(0);
        HX_LDS_BARRIER();
        if (step + 3 < steps) issue(step + 3);            // into the buffer that every wave has left
        if (idle) return;
        const int t = wk.tiles.at(step);
        const h16x8(*st)[64] = stage[step % S];
        uint32_t sees = 0xffffffffu;
        if constexpr (TAIL) {
            sees = win_sees(32 * t, qpos, wc.window, wc.sinks);
#pragma unroll
            for (int x = 0; x < 16; ++x) sc[x] = (sees >> (8 * (x >> 2) + 4 * hl + (x & 3))) & 1u ? sc[x] : NEG_INF;
        }
        float mx = NEG_INF;
#pragma unroll
        for (int x = 0; x < 16; ++x) mx = fmaxf(mx, sc[x]);
        mx = max_halves(mx);
        // A larger score moves the base only if its weight would pass 2^SLACK: what has been summed up is rescaled for the first tiles of a row and hardly again.
        // (Any base is right: numerator and sum are relative to the same one, in floating point.)
        if (__builtin_amdgcn_ballot_w64(mx > m + slack) != 0) {
            const float m_new = fmaxf(m, mx), to = m_new == NEG_INF ? 0.f : m_new;       // a row that has seen nothing yet: weights 0, no NaN
            const bool was = far;
            far = far || __builtin_amdgcn_ballot_w64(fabsf(to * scale_log2e) >= kWinFarBase) != 0;
            const float from = was ? base : m, next = far ? to : to * scale_log2e - SHIFT;
            // (nothing summed up yet: 0, whatever base a row without a score stands at)
            const float alpha = __builtin_amdgcn_exp2f(m == NEG_INF ? NEG_INF : far ? (from - to) * scale_log2e : base - next);
            m = m_new;
            base = next;
            lsum *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int x = 0; x < 16; ++x) oacc[db][x] *= alpha;
        }
        // the next tile's scores on the matrix cores while this one's weights are on the vector unit
        floatx16 ahead;
        float ps = 0.f;
        if (far) {
            scores(min(step + 1, steps - 1), ahead);
#pragma unroll
            for (int x = 0; x < 16; ++x) { sc[x] = __builtin_amdgcn_exp2f(fmaf(sc[x] - base, scale_log2e, SHIFT)); ps += sc[x]; }
        } else {
            scores(min(step + 1, steps - 1), ahead);
#pragma unroll
            for (int x = 0; x < 16; ++x) { sc[x] = __builtin_amdgcn_exp2f(fmaf(sc[x], scale_log2e, -base)); ps += sc[x]; }
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);          // reads of LDS; then a matrix instruction, a read, and what the vector unit does meanwhile
#pragma unroll
            for (int x = 0; x < 2 * KT; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
            }
        }
        lsum += ps;
        if constexpr (TAIL) {
            bool odd = false;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) odd = odd || any_odd(st[2 * KT + dt][lane]);
            if (__builtin_amdgcn_ballot_w64(odd) != 0) {
                tree_slow_tile<DB>(reinterpret_cast<const h16_t *>(st[2 * KT]), sc, sees, lane, oacc);
                sc = ahead;
                return;
            }
        }
        TreeP p[2], lo[2];
        tree_pack(sc, p, lo);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const h16x8 v = st[2 * KT + 2 * db + sub][fl + 32 * g];
                oacc[db] = hx_mfma32(v, lo[g].v, oacc[db]);
                oacc[db] = hx_mfma32(v, p[g].v, oacc[db]);
            }
        sc = ahead;
    };
    int step = 0;
    for (; step < wk.tiles.clean; ++step) walk(step, std::false_type{});
    for (; step < steps; ++step) walk(step, std::true_type{});
    lsum = sum_halves(lsum);
    if (r >= R) return;
    const float inv = 1.0f / lsum;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
            const float x[4] = {oacc[db][4 * qd] * inv, oacc[db][4 * qd + 1] * inv, oacc[db][4 * qd + 2] * inv, oacc[db][4 * qd + 3] * inv};
            tree_store4(out, row0 + node, head * D + 32 * db + 8 * qd + 4 * hl, x);
        }
    if (wp.stat != nullptr && hl == 0) *reinterpret_cast<float2 *>(wp.stat + 2 * ((size_t)(row0 + node) * hq_l + head)) = win_stat(base, far ? inv * UNIT : inv, far);
}

void launch_win_attn(const h16_t *q, const h16_t *q_lo, int64_t ldq, const TreeIn &in, h16_t *kc, h16_t *vc, KvGeom kg, int hq_l, const WinCall &wc,
                     const int32_t *lens, const WinPlan &wp, const TreeOut &out, hipStream_t s) {
    const int G = hq_l / kg.hkv_l, nrb = win_row_blocks(wc.max_n, G, wp.shared ? 128 : 32);
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)kg.d);
    const dim3 grid(win_grid(wc.batch * kg.hkv_l * wp.nsplit, nrb));
#define HX_WIN_D(DD)                                                                                                                                               \
    do {                                                                                                                                                           \
        if (wp.shared) hipLaunchKernelGGL((win_attn_kernel<DD>), grid, dim3(256), 0, s, q, ldq, kc, vc, kg, hq_l, G, nrb, wc, lens, wp, out, scale_log2e);          \
        else if (q_lo != nullptr) hipLaunchKernelGGL((win_few_kernel<DD, true>), grid, dim3(512), 0, s, q, q_lo, ldq, in, kc, vc, kg, hq_l, G, nrb, wc, lens, wp, out, scale_log2e); \
        else hipLaunchKernelGGL((win_few_kernel<DD, false>), grid, dim3(512), 0, s, q, q_lo, ldq, in, kc, vc, kg, hq_l, G, nrb, wc, lens, wp, out, scale_log2e);    \
    } while (0)
    if (kg.d == 128) HX_WIN_D(128);
    else HX_WIN_D(64);
#undef HX_WIN_D
}

// ---- the weights' sums ------------------------------------------------------------------------------------------------
// weights[j] += sum over the call's rows and a kv head's query heads of exp(s_rj - m_r) / l_r, once every row's maximum and sum are known.  Every position belongs to
// one wave, or its partial sums are joined in one order; nothing is added atomically, so that the same call gives the same bits.
// Here: the scores once more.  A wave keeps the keys of one tile in registers and goes through the rows that attend it in groups of 32; the sums stay in its
// lanes (lane: a column of every group) and meet at the end.  For 33 to 64 rows a kv head, and for fewer where the scores have no room.
// Bound by each wave's chain of row loads and products: sixteen sequences of five rows at 2000, eight kv heads of eight, 26 us for 66 MB of keys (2.5 TB/s).
template <int D, bool QLO>
__global__ __launch_bounds__(256, 4) void win_weights_kernel(const h16_t *__restrict__ q, const h16_t *__restrict__ q_lo, int64_t ldq, const h16_t *__restrict__ kc, KvGeom kg,
                                                             int hq_l, int G, int tile_blocks, WinCall wc, const int32_t *__restrict__ lens, const float *__restrict__ stat,
                                                             float *__restrict__ weights, float scale_log2e) {
    constexpr int KT = D / 32;
    const int tb = blockIdx.x % tile_blocks, c = (blockIdx.x / tile_blocks) % kg.hkv_l, nth = blockIdx.x / tile_blocks / kg.hkv_l;
    const int seq = wc.seq0 + nth, row0 = wc.cu[nth], len = lens[seq], n = min(wc.cu[nth + 1] - row0, wc.max_seq - len), R = n * G;
    if (n <= 0) return;
    WinTiles tiles;
    tiles.set(len, len + n - 1, wc.window, wc.sinks, 0);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hl = lane >> 5, i32 = lane & 31;
    const int sub = i32 >> 4, fl = (lane & 15) + 16 * hl;
    for (int v = 4 * tb + wave; v < tiles.nt; v += 4 * tile_blocks) {
        const int t = tiles.at(v), p0 = 32 * t;
        const h16_t *src = kc + (size_t)seq * kg.seq_stride + (size_t)c * kg.smax * D + ((size_t)(2 * t + sub) * KT * 64 + fl) * 8;
        h16x8 kf[2 * KT];
#pragma unroll
        for (int kk = 0; kk < 2 * KT; ++kk) kf[kk] = *reinterpret_cast<const h16x8 *>(src + ((kk >> 1) * 64 + 32 * (kk & 1)) * 8);
        // new rows that attend one of its positions: from the first at or behind the tile to the last whose window reaches it
        const int x_lo = max(0, p0 - len), x_hi = p0 < wc.sinks ? n - 1 : min(n - 1, p0 + 31 + wc.window - 1 - len);
        floatx16 acc;
#pragma unroll
        for (int x = 0; x < 16; ++x) acc[x] = 0.f;
        for (int g = x_lo * G / 32; g <= (x_hi * G + G - 1) / 32; ++g) {
            const int r = 32 * g + i32, rr = min(r, R - 1), node = rr / G, head = c * G + (rr - node * G);
            const size_t at = (size_t)(row0 + node) * ldq + (size_t)head * D + 8 * hl;
            const float2 ml = *reinterpret_cast<const float2 *>(stat + 2 * ((size_t)(row0 + node) * hq_l + head));
            floatx16 sc;
#pragma unroll
            for (int x = 0; x < 16; ++x) sc[x] = 0.f;
            if constexpr (QLO) {
#pragma unroll
                for (int kk = 0; kk < 2 * KT; ++kk) sc = hx_mfma32(kf[kk], *reinterpret_cast<const h16x8 *>(q_lo + at + 16 * kk), sc);
            }
#pragma unroll
            for (int kk = 0; kk < 2 * KT; ++kk) sc = hx_mfma32(kf[kk], *reinterpret_cast<const h16x8 *>(q + at + 16 * kk), sc);
            const WinBase base(ml.x, ml.y);
            const bool careful = __builtin_amdgcn_ballot_w64(base.odd()) != 0;
            const int first = len + 32 * g / G, last = len + min(32 * g + 31, R - 1) / G;
            if (32 * g + 31 >= R || !win_all(p0, 32, first, last, wc.window, wc.sinks)) {
                const uint32_t sees = r < R ? win_sees(p0, len + node, wc.window, wc.sinks) : 0u;
#pragma unroll
                for (int x = 0; x < 16; ++x) sc[x] = (sees >> (8 * (x >> 2) + 4 * hl + (x & 3))) & 1u ? sc[x] : NEG_INF;
            }
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[x] = base.add(acc[x], sc[x], scale_log2e, careful);
        }
        float mine = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            float a = acc[x];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) a += __shfl_xor(a, o, 64);
            mine = i32 == x ? a : mine;
        }
        const int pos = p0 + 8 * ((i32 & 15) >> 2) + 4 * hl + (i32 & 3);
        if (i32 < 16 && pos < len + n) {
            float *dst = weights + ((size_t)seq * kg.hkv_l + c) * wc.max_seq + pos;
            *dst += mine;
        }
    }
}
// The same for up to 32 rows a kv head from the scores that the attention has left (WinPlan), a thread per position: 32 ragged contexts, 8 heads a kv head, 6.2 us
// where the keys once more took 23 to 28
__global__ __launch_bounds__(256) void win_gather_kernel(KvGeom kg, int hq_l, int G, int tile_blocks, bool fresh, WinCall wc, const int32_t *__restrict__ lens, WinPlan wp,
                                                         float *__restrict__ weights, float scale_log2e) {
    const int tb = blockIdx.x % tile_blocks, c = (blockIdx.x / tile_blocks) % kg.hkv_l, nth = blockIdx.x / tile_blocks / kg.hkv_l;
    const int seq = wc.seq0 + nth, row0 = wc.cu[nth], len = lens[seq], n = min(wc.cu[nth + 1] - row0, wc.max_seq - len);
    if (n <= 0) return;
    WinTiles tiles;                                           // as the attention had them: one block of rows
    tiles.set(len, len + n - 1, wc.window, wc.sinks, fresh ? len : len + 1);
    const size_t row_floats = (size_t)32 * wp.score_tiles;
    for (int v = 8 * tb + threadIdx.x / 32; v < tiles.nt; v += 8 * tile_blocks) {
        const int pos = 32 * tiles.at(v) + threadIdx.x % 32;
        if (pos >= len + n) continue;
        float sum = 0.f;
        for (int x = 0; x < n; ++x) {
            const size_t e = (size_t)(row0 + x) * hq_l + c * G;
            const float *scores = wp.scores + e * row_floats + 32 * v + threadIdx.x % 32, *stat = wp.stat + 2 * e;
#pragma unroll 8
            for (int h = 0; h < G; ++h) {
                const WinBase base(stat[2 * h], stat[2 * h + 1]);
                sum = base.add(sum, scores[h * row_floats], scale_log2e, true);
            }
        }
        weights[((size_t)seq * kg.hkv_l + c) * wc.max_seq + pos] += sum;
    }
}

// groups of eight tiles in a cache's positions, each with a counter and a place for its sums
__host__ __device__ inline int win_units(int smax) { return (smax / 32 + 7) / 8; }
// The same for calls of many rows: a wave keeps the keys of two tiles, and the block's four waves share the rows, which go from memory to LDS directly, two
// groups ahead, together with each row's statistics.  Where tiles are few the groups are dealt to `splits` blocks; their sums meet in the order of the
// rows, added up by the last block to arrive.
template <int D, bool QLO>
__global__ __launch_bounds__(256, 2) void win_weights_shared_kernel(const h16_t *__restrict__ q, const h16_t *__restrict__ q_lo, int64_t ldq, const h16_t *__restrict__ kc,
                                                                    KvGeom kg, int hq_l, int G, int tile_blocks, int splits, WinCall wc, const int32_t *__restrict__ lens,
                                                                    const float *__restrict__ stat, float *__restrict__ weights, float *part, unsigned *arrived,
                                                                    float scale_log2e) {
    constexpr int KT = D / 32, W = 4, TW = 2, S = 3, PIECES = 2 * KT * (QLO ? 2 : 1), LPT = PIECES / W;      // 1 KB pieces of a group of 32 rows
    __shared__ h16x8 s_q[S][PIECES][64];
    __shared__ float s_stat[S][W][64];                        // largest score and 1 / sum of the group's rows, a copy for every wave
    __shared__ int s_last;
    int pair, id;
    win_place(wc.batch * kg.hkv_l, tile_blocks * splits, &pair, &id);
    if (pair >= wc.batch * kg.hkv_l) return;
    const int split = id % splits, tb = id / splits, c = pair % kg.hkv_l, nth = wc.order[pair / kg.hkv_l];
    const int seq = wc.seq0 + nth, row0 = wc.cu[nth], len = lens[seq], n = min(wc.cu[nth + 1] - row0, wc.max_seq - len);
    if (n <= 0) return;
    WinTiles tiles;
    tiles.set(len, len + n - 1, wc.window, wc.sinks, 0);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hl = lane >> 5, i32 = lane & 31;
    const int sub = i32 >> 4, fl = (lane & 15) + 16 * hl;
    const h16_t *slab = kc + (size_t)seq * kg.seq_stride + (size_t)c * kg.smax * D;
    const int per32 = 32 / G, rem32 = 32 % G;                 // what 32 rows on is in new rows and heads
    for (int v0 = W * TW * tb; v0 < tiles.nt; v0 += W * TW * tile_blocks) {
        // new rows that attend a position of the block's tiles: from the first at or behind them to the last whose window reaches them
        const int t_first = tiles.at(v0), t_last = tiles.at(min(v0 + W * TW, tiles.nt) - 1);
        const int x_lo = max(0, 32 * t_first - len), x_hi = 32 * t_first < wc.sinks ? n - 1 : min(n - 1, 32 * t_last + 31 + wc.window - 1 - len);
        int g0 = x_lo * G / 32, g1 = (x_hi * G + G - 1) / 32 + 1;
        const int share = (g1 - g0 + splits - 1) / splits;
        g0 += split * share;
        g1 = min(g1, g0 + share);
        int p0[TW];
        bool live[TW];
        h16x8 kf[TW][2 * KT];
        floatx16 acc[TW];
#pragma unroll
        for (int w = 0; w < TW; ++w) {
            const int v = v0 + TW * wave + w, t = tiles.at(min(v, tiles.nt - 1));
            p0[w] = 32 * t;                                   // past the last tile it once more, not stored
            live[w] = v < tiles.nt;
            const h16_t *src = slab + ((size_t)(2 * t + sub) * KT * 64 + fl) * 8;
#pragma unroll
            for (int kk = 0; kk < 2 * KT; ++kk) kf[w][kk] = *reinterpret_cast<const h16x8 *>(src + ((kk >> 1) * 64 + 32 * (kk & 1)) * 8);
#pragma unroll
            for (int x = 0; x < 16; ++x) acc[w][x] = 0.f;
        }
        // row r of a lane's next group to request, and of the statistics: new row and head
        int nq = (32 * g0 + i32) / G, hq = (32 * g0 + i32) - nq * G, ns = (32 * g0 + (lane >> 1)) / G, hs = (32 * g0 + (lane >> 1)) - ns * G;
        auto issue = [&](int g) {
            const int base = __builtin_amdgcn_readfirstlane(min(nq, n - 1));
            const bool past = nq >= n;                        // rows past the last repeat it
            const unsigned row = (unsigned)((past ? n - 1 : nq) - base) * (unsigned)ldq + (unsigned)((past ? G - 1 : hq) * D + 8 * hl);
            const size_t first = (size_t)(row0 + base) * ldq + (size_t)c * G * D;
#pragma unroll
            for (int x = 0; x < LPT; ++x) {
                const int piece = wave * LPT + x, kk = piece % (2 * KT);
                const h16_t *src = (piece < 2 * KT ? q : q_lo) + first;
                hx_load_lds16(hx_lds_addr(&s_q[g % S][piece][0]), 2u * (row + 16u * kk), src);
            }
            const bool gone = ns >= n;
            const int at = ((gone ? n - 1 : ns) - base) * hq_l + (gone ? G - 1 : hs);
            hx_load_lds4(hx_lds_addr(&s_stat[g % S][wave][0]), (unsigned)(8 * at + 4 * (lane & 1)), stat + 2 * ((size_t)(row0 + base) * hq_l + (size_t)c * G));
            nq += per32; hq += rem32; ns += per32; hs += rem32;
            if (hq >= G) { hq -= G; ++nq; }
            if (hs >= G) { hs -= G; ++ns; }
        };
        int node = nq, head = hq;                             // of this lane's row of the group that is worked on
        __syncthreads();                                      // every wave has left the buffers of the tiles before
        HX_WAIT_VM(0);
        if (g0 < g1) issue(g0);
        if (g0 + 1 < g1) issue(g0 + 1);
        for (int g = g0; g < g1; ++g) {
            if (g + 1 < g1) HX_WAIT_VM(LPT + 1);              // the next group may stay in flight
            else HX_WAIT_VM(0);
            HX_LDS_BARRIER();
            if (g + 2 < g1) issue(g + 2);                     // into the buffer that every wave has left
            const WinBase base(s_stat[g % S][wave][2 * i32], s_stat[g % S][wave][2 * i32 + 1]);
            const bool careful = __builtin_amdgcn_ballot_w64(base.odd()) != 0;
            const int first = len + __builtin_amdgcn_readfirstlane(node), last = len + __builtin_amdgcn_readlane(node, 31);
            h16x8 rows[PIECES];
#pragma unroll
            for (int x = 0; x < PIECES; ++x) rows[x] = s_q[g % S][x][lane];
            floatx16 sc[TW];
            auto scores = [&](int w) {
#pragma unroll
                for (int x = 0; x < 16; ++x) sc[w][x] = 0.f;
#pragma unroll
                for (int x = PIECES - 1; x >= 0; --x) sc[w] = hx_mfma32(kf[w][x % (2 * KT)], rows[x], sc[w]);
            };
            auto mask = [&](int w) {
                if (last < len + n && win_all(p0[w], 32, first, last, wc.window, wc.sinks)) return;
                const uint32_t sees = node < n ? win_sees(p0[w], len + node, wc.window, wc.sinks) : 0u;
#pragma unroll
                for (int x = 0; x < 16; ++x) sc[w][x] = (sees >> (8 * (x >> 2) + 4 * hl + (x & 3))) & 1u ? sc[w][x] : NEG_INF;
            };
            auto add = [&](int w) {
                if (careful) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) acc[w][x] = base.add(acc[w][x], sc[w][x], scale_log2e, true);
                } else {
#pragma unroll
                    for (int x = 0; x < 16; ++x) acc[w][x] = base.add(acc[w][x], sc[w][x], scale_log2e, false);
                }
            };
            static_assert(TW == 2, "the second tile's scores on the matrix cores while the first one's weights are on the vector unit");
            scores(0);
            mask(0);
            scores(1);
            add(0);
#pragma unroll
            for (int x = 0; x < PIECES; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);      // a matrix instruction, then what the vector unit does meanwhile
                __builtin_amdgcn_sched_group_barrier(0x002, 64 / PIECES, 0);
            }
            mask(1);
            add(1);
            node += per32; head += rem32;
            if (head >= G) { head -= G; ++node; }
        }
        const size_t unit = (size_t)(nth * kg.hkv_l + c) * win_units(kg.smax) + v0 / (W * TW);
#pragma unroll
        for (int w = 0; w < TW; ++w) {
            float mine = 0.f;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                float a = acc[w][x];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) a += __shfl_xor(a, o, 64);
                mine = i32 == x ? a : mine;
            }
            const int pos = 8 * ((i32 & 15) >> 2) + 4 * hl + (i32 & 3);
            if (i32 >= 16) continue;
            if (splits > 1) dev_store(part + ((unit * splits + split) * W + wave) * TW * 32 + 32 * w + pos, mine);
            else if (live[w] && p0[w] + pos < len + n) weights[((size_t)seq * kg.hkv_l + c) * wc.max_seq + p0[w] + pos] += mine;
        }
        if (splits > 1 && tree_arrive(arrived + unit, splits, &s_last)) {
            const int x = threadIdx.x, v = v0 + x / 32;       // one of the block's positions per thread
            if (v < tiles.nt) {
                const int pos = 32 * tiles.at(v) + x % 32;
                float sum = 0.f;
                for (int u = 0; u < splits; ++u) sum += dev_load(part + (unit * splits + u) * W * TW * 32 + x);
                if (pos < len + n) weights[((size_t)seq * kg.hkv_l + c) * wc.max_seq + pos] += sum;
            }
        }
    }
}

void launch_win_weights(const h16_t *q, const h16_t *q_lo, int64_t ldq, const h16_t *kc, KvGeom kg, int hq_l, const WinCall &wc, const int32_t *lens,
                        const WinPlan &wp, bool fresh, float *weights, const WinReach &reach, hipStream_t s) {
    const int G = hq_l / kg.hkv_l;
    const float scale_log2e = 1.4426950408889634f / sqrtf((float)kg.d);
    if (wp.scores != nullptr) {
        const int tile_blocks = (reach.most + 7) / 8;
        hipLaunchKernelGGL(win_gather_kernel, dim3((unsigned)tile_blocks * kg.hkv_l * wc.batch), dim3(256), 0, s, kg, hq_l, G, tile_blocks, fresh, wc, lens, wp, weights, scale_log2e);
        return;
    }
    // shared from 65 rows on (a whole call at 2000 positions, eight kv heads of eight, us, tiles alone / shared: one sequence of 8 rows 28.3 / 29.2, of 16 32.1 / 31.9, of
    // 64 58.6 / 40.7; sixteen of 5 rows 62.3 / 61.5, of 8 66.0 / 62.6, of 16 104 / 90)
    const bool shared = (int64_t)wc.max_n * G > 64;
    const int tile_blocks = (reach.most + (shared ? 7 : 3)) / (shared ? 8 : 4);
    const int64_t blocks = (int64_t)tile_blocks * kg.hkv_l * wc.batch, groups = ((int64_t)wc.max_n * G + 31) / 32;
    int splits = 1;
    const int64_t units = (int64_t)wc.batch * kg.hkv_l * win_units(kg.smax);        // a length on the device may be beyond what the host knows
    // Two blocks a CU: so many rounds of 512, each of a block's share of the groups and of what it costs besides (keys, the first rows' way, its sums: as
    // much as six groups)
    if (shared && units <= kWinUnits) {
        int64_t least = INT64_MAX;
        for (int64_t x = 1; x <= std::min<int64_t>({16, (groups + 7) / 8, (int64_t)kWinPartFloats / (256 * units)}); ++x) {
            const int64_t cost = (reach.groups * kg.hkv_l * x + 511) / 512 * ((groups + x - 1) / x + 6);
            if (cost < least) { least = cost; splits = (int)x; }
        }
    }
    const dim3 grid(shared ? win_grid(kg.hkv_l * wc.batch, tile_blocks * splits) : (unsigned)blocks);
#define HX_WIN_W(DD, LO)                                                                                                                                                   \
    do {                                                                                                                                                                   \
        if (shared)                                                                                                                                                        \
            hipLaunchKernelGGL((win_weights_shared_kernel<DD, LO>), grid, dim3(256), 0, s, q, q_lo, ldq, kc, kg, hq_l, G, tile_blocks, splits, wc, lens, wp.stat, weights, \
                               wp.part_o, wp.arrived, scale_log2e);                                                                                                        \
        else                                                                                                                                                               \
            hipLaunchKernelGGL((win_weights_kernel<DD, LO>), grid, dim3(256), 0, s, q, q_lo, ldq, kc, kg, hq_l, G, tile_blocks, wc, lens, wp.stat, weights, scale_log2e);  \
    } while (0)
    if (kg.d == 128) { if (q_lo != nullptr) HX_WIN_W(128, true); else HX_WIN_W(128, false); }
    else { if (q_lo != nullptr) HX_WIN_W(64, true); else HX_WIN_W(64, false); }
#undef HX_WIN_W
}

// ---- eviction: the move ------------------------------------------------------------------------------------------------
// The kept rows of one (layer, sequence, kv head): row slots[j] of the source becomes row j.  A group of 256 threads takes chunks of 32 destination rows and
// reads a chunk whole before it writes it.  In place there is one block for all of them, four chunks at a time, in order: rows only move to the front
// (slots[j] >= j, both growing), so that what is written has been read.  K moves in pieces of 16 bytes, V, which lies transposed, through LDS.
// Keys that are rotated back by their distance are rotated in fp32 and rounded to the element type once more.
// Bound by HBM: where slots stay here and there, nearly every 64 bytes of the context hold one of them (K four, V eight positions each), so that a fetch takes most of it:
// 2 layers x 8 x 8 heads, 1500 .. 4000 to 1024 slots by weight 50 us (134 MB of rows moved, 230 MB over HBM at 4.6 TB/s); 2 x 16 x 1 heads, 2048 newest of 4000, rotated 22 us (67 MB).
template <int D, bool ROT, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS) void evict_move_kernel(EvictCall ec, EvictMove mv, int blocks) {
    constexpr int KT = D / 32, PIECES = ROT ? 2 : 2 * KT / 4, HALF = D / 2;
    __shared__ h16_t s_rows[GROUPS][32][D + 2];
    __shared__ int s_slots[GROUPS][32];
    const int group = threadIdx.x / 256, thread = threadIdx.x % 256, wave = thread >> 6, lane = thread & 63;
    h16_t(*s_v)[D + 2] = s_rows[group];
    int *s_slot = s_slots[group];
    const unsigned unit = blockIdx.x / (unsigned)blocks;
    const int chunk = (int)(blockIdx.x % (unsigned)blocks), c = unit % ec.hkv, b = (unit / ec.hkv) % ec.batch, layer = unit / ec.hkv / ec.batch;
    const int32_t *slots = ec.slots + (size_t)unit * ec.dst_seq;
    const size_t src = (size_t)layer * mv.src_layer + (size_t)b * mv.src.seq_stride + (size_t)c * mv.src.smax * D;
    const size_t dst = (size_t)layer * mv.dst_layer + (size_t)b * mv.dst.seq_stride + (size_t)c * mv.dst.smax * D;
    const h16_t *ks = static_cast<const h16_t *>(mv.ks) + src, *vs = static_cast<const h16_t *>(mv.vs) + src;
    h16_t *kd = static_cast<h16_t *>(mv.kd) + dst, *vd = static_cast<h16_t *>(mv.vd) + dst;
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < mv.dst_batch; i += 256 * GROUPS) mv.dst_lens[i] = i < ec.batch ? min(min(mv.lens[i], ec.max_seq), ec.keep) : 0;
    const int most = min(ec.keep, ec.dst_seq);
    for (int first = 32 * GROUPS * chunk; first < most; first += 32 * GROUPS * blocks) {
        const int j0 = first + 32 * group;
        __syncthreads();
        if (thread < 32) s_slot[thread] = j0 + thread < most ? slots[j0 + thread] : -1;
        __syncthreads();
        // nothing to move: the kept ones come first; or in place, and every row is where it belongs
        const bool moves = s_slot[0] >= 0 && !(mv.ks == mv.kd && s_slot[31] == j0 + 31);
        // a wave's piece i: one fragment tile, 16 rows x 32 elements, as it lies in the destination (rotated: and the one half a head further); rows that are not
        // there read slot 0
        typedef uint32_t piece __attribute__((ext_vector_type(4)));
        piece k[PIECES];
        constexpr int ACROSS = ROT ? KT / 2 : KT;
        const bool has = !ROT || wave < KT;                     // a rotated head of 64 is two waves' work
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int tile = wave + (ROT ? 0 : 4 * i), row = 16 * (tile / ACROSS) + (lane & 15), dd = 32 * (tile % ACROSS) + 8 * (lane >> 4) + (ROT ? HALF * i : 0);
            k[i] = *reinterpret_cast<const piece *>(ks + kv_k_offset(has ? max(s_slot[row], 0) : 0, dd, D));
        }
        if constexpr (ROT) {
            const int row = 16 * (wave / ACROSS) + (lane & 15), dd = 32 * (wave % ACROSS) + 8 * (lane >> 4);
            const int moved = has ? max(s_slot[row] - (j0 + row), 0) : 0;
            if (moved != 0) {
                const floatx4 *cs = reinterpret_cast<const floatx4 *>(mv.cos_tab + (size_t)moved * HALF + dd), *sn = reinterpret_cast<const floatx4 *>(mv.sin_tab + (size_t)moved * HALF + dd);
                piece &lo = k[0], &hi = k[PIECES - 1];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const floatx4 c4 = cs[h], s4 = sn[h];
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        float a0, a1, b0, b1;
                        h16x2_to_f32(lo[2 * h + p], a0, a1);
                        h16x2_to_f32(hi[2 * h + p], b0, b1);
                        lo[2 * h + p] = pack_h16x2(a0 * c4[2 * p] + b0 * s4[2 * p], a1 * c4[2 * p + 1] + b1 * s4[2 * p + 1]);
                        hi[2 * h + p] = pack_h16x2(b0 * c4[2 * p] - a0 * s4[2 * p], b1 * c4[2 * p + 1] - a1 * s4[2 * p + 1]);
                    }
                }
            }
        }
        for (int idx = moves ? thread : 32 * D; idx < 32 * D; idx += 256) {
            const int row = idx / D, dd = idx % D;             // a wave: 64 elements of one row, two bytes of every 16 (kvlayout.h)
            s_v[row][dd] = vs[kv_v_offset(max(s_slot[row], 0), dd, D)];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int tile = wave + (ROT ? 0 : 4 * i), row = 16 * (tile / ACROSS) + (lane & 15), dd = 32 * (tile % ACROSS) + 8 * (lane >> 4) + (ROT ? HALF * i : 0);
            if (has && moves && s_slot[row] >= 0) *reinterpret_cast<piece *>(kd + kv_k_offset(j0 + row, dd, D)) = k[i];
        }
        for (int idx = moves ? thread : 4 * D; idx < 4 * D; idx += 256) {
            const int dd = (idx & 15) + 16 * (idx >> 6), g = (idx >> 4) & 3;    // 16-byte pieces in the order in which they lie (kvlayout.h)
            union { uint4 u; h16_t e[8]; } w;
#pragma unroll
            for (int j = 0; j < 8; ++j) w.e[j] = s_v[4 * g + (j & 3) + 16 * (j >> 2)][dd];
            h16_t *at = vd + kv_v_offset(j0 + 4 * g, dd, D);
            if (s_slot[31] >= 0) {
                *reinterpret_cast<uint4 *>(at) = w.u;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (s_slot[4 * g + (j & 3) + 16 * (j >> 2)] >= 0) at[j] = w.e[j];
            }
        }
    }
}
void launch_evict_move(const EvictCall &ec, const EvictMove &mv, hipStream_t s) {
    const int blocks = evict_blocks(ec, mv);
    const dim3 grid((unsigned)blocks * ec.layers * ec.batch * ec.hkv);
#define HX_MOVE(DD, R)                                                                                                                     \
    do {                                                                                                                                   \
        if (mv.ks == mv.kd) hipLaunchKernelGGL((evict_move_kernel<DD, R, 4>), grid, dim3(1024), 0, s, ec, mv, blocks);                      \
        else hipLaunchKernelGGL((evict_move_kernel<DD, R, 1>), grid, dim3(256), 0, s, ec, mv, blocks);                                      \
    } while (0)
    if (mv.src.d == 128) { if (mv.cos_tab != nullptr) HX_MOVE(128, true); else HX_MOVE(128, false); }
    else { if (mv.cos_tab != nullptr) HX_MOVE(64, true); else HX_MOVE(64, false); }
#undef HX_MOVE
}

}  // namespace HX_NS
