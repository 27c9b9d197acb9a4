// Windowed rows over the cache and eviction, fp32 stages (cache [seq][kv head][smax][d]), and what does not depend on the type: the choice of slots.
#include <algorithm>

#include "window.h"

#define NEG_INF (-INFINITY)

namespace {

__device__ __forceinline__ floatx4 mfma_f32(float a, float b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// raw projection [rows][(hq + 2 hkv) d] -> rotary embedding at len + row, q as plain rows, k and v into the cache; a rotary pair per thread
__global__ __launch_bounds__(256) void f32_win_rope_append_kernel(const float *__restrict__ qkv, int hq_l, KvGeom kg, WinCall wc, const int32_t *__restrict__ lens,
                                                                  const float *__restrict__ cos_tab, const float *__restrict__ sin_tab, float *__restrict__ q,
                                                                  float *__restrict__ kc, float *__restrict__ vc) {
    const int d = kg.d, half = d >> 1, heads = hq_l + 2 * kg.hkv_l;
    const unsigned idx = blockIdx.x * 256u + threadIdx.x, per_row = heads * half;
    const int t = wc.cu[0] + (int)(idx / per_row), rem = idx % per_row, head = rem / half, i = rem - head * half;
    if (t >= wc.cu[wc.batch]) return;
    int lo_seq = 0, hi_seq = wc.batch;                        // the last sequence whose first row is not behind t
    while (hi_seq - lo_seq > 1) {
        const int mid = (lo_seq + hi_seq) >> 1;
        if (wc.cu[mid] <= t) lo_seq = mid;
        else hi_seq = mid;
    }
    const int seq = wc.seq0 + lo_seq, slot = lens[seq] + t - wc.cu[lo_seq];
    if (slot >= wc.max_seq) return;
    const float *src = qkv + (size_t)t * heads * d + (size_t)head * d + i;
    float lo = src[0], hi = src[half];
    if (head < hq_l + kg.hkv_l) {
        const size_t at = (size_t)slot * half + i;
        const float c = cos_tab[at], sn = sin_tab[at], l = lo * c - hi * sn;
        hi = hi * c + lo * sn;
        lo = l;
    }
    const size_t slab = (size_t)seq * kg.seq_stride;
    float *dst = head < hq_l ? q + ((size_t)t * hq_l + head) * d
                 : head < hq_l + kg.hkv_l ? kc + slab + ((size_t)(head - hq_l) * kg.smax + slot) * d
                                          : vc + slab + ((size_t)(head - hq_l - kg.hkv_l) * kg.smax + slot) * d;
    dst[i] = lo;
    dst[half + i] = hi;
}

// plain rows into the cache, 16 bytes of K and of V per thread
__global__ __launch_bounds__(256) void f32_win_append_kernel(TreeIn in, float *__restrict__ kc, float *__restrict__ vc, KvGeom kg, WinCall wc, const int32_t *__restrict__ lens) {
    const int nth = blockIdx.z, seq = wc.seq0 + nth, row0 = wc.cu[nth], len = lens[seq], n = min(wc.cu[nth + 1] - row0, wc.max_seq - len);
    const int q4 = kg.d >> 2, width = kg.hkv_l * q4;
    for (unsigned idx = blockIdx.x * 256u + threadIdx.x; (int)(idx / width) < n; idx += gridDim.x * 256u) {
        const int x = idx / width, e = idx % width, c = e / q4, dd = 4 * (e % q4);
        const size_t at = (size_t)seq * kg.seq_stride + ((size_t)c * kg.smax + len + x) * kg.d + dd;
        *reinterpret_cast<floatx4 *>(kc + at) = *reinterpret_cast<const floatx4 *>(static_cast<const float *>(in.k) + (size_t)(row0 + x) * in.ldk + c * kg.d + dd);
        *reinterpret_cast<floatx4 *>(vc + at) = *reinterpret_cast<const floatx4 *>(static_cast<const float *>(in.v) + (size_t)(row0 + x) * in.ldv + c * kg.d + dd);
    }
}

// A block takes 16 query columns of one (sequence, kv head) -- column j: new row j / G, head j % G -- and a run of their tiles, over whose halves of 16 positions
// its W waves interleave; products and register layouts are those of the stage's fp32 attention (v_mfma_f32_16x16x4_f32, a lane owns column l % 16
// and positions 4 (l / 16) + r, P stays in registers).  Rows that are not in the cache yet (in.k != NULL: a sequence's rows are one block's columns then) are
// read from the caller's and appended by the run that holds their tile.  Three waves a SIMD instead of two: 30.7 -> 25.8 us.
// Bound by each wave's chain of loads and fp32 matrix instructions (32 cycles each, 64 for 16 positions): d 128, 16 / 4 heads, three prompts of 90 .. 301 rows under a window
// of 128 25.8 us; one row at 40 positions, d 64, 5.3, half of that the launch.
template <int D, int W>
__global__ __launch_bounds__(64 * W, 3) void f32_win_attn_kernel(const float *__restrict__ q, int64_t ldq, TreeIn in, float *kc, float *vc, KvGeom kg, int hq_l, int G, int nrb,
                                                              WinCall wc, const int32_t *__restrict__ lens, WinPlan wp, float *__restrict__ o) {
    constexpr int KT = D / 16, VH = D / 64;
    __shared__ float s_m[W][16], s_l[W][16];
    __shared__ __align__(16) float s_o[W][16][D];
    __shared__ int s_last;
    WinWork wk;
    const bool fresh = in.k != nullptr;
    if (!wk.find(kg.hkv_l, G, nrb, 16, wc, lens, wp, fresh)) return;
    const int len = wk.len, R = wk.R, row0 = wk.row0, rb = wk.rb, c = wk.c, seen = len + wk.n - 1;    // the last slot that is anybody's
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int rr = min(rb * 16 + i, R - 1), node = rr / G, head = c * G + (rr - node * G), qpos = len + node;
    const int p_lo = len + rb * 16 / G, p_hi = len + min(wk.n - 1, (rb * 16 + 15) / G);
    const size_t slab = (size_t)wk.seq * kg.seq_stride + (size_t)c * kg.smax * D;
    float *K = kc + slab, *V = vc + slab;
    const float *nk = fresh ? static_cast<const float *>(in.k) + (size_t)row0 * in.ldk + c * D : nullptr;
    const float *nv = fresh ? static_cast<const float *>(in.v) + (size_t)row0 * in.ldv + c * D : nullptr;
    // position p of the keys and values: the cache's, or the new row that will be there
    auto key_at = [&](int p) { return fresh && p >= len ? nk + (size_t)(p - len) * in.ldk : K + (size_t)p * D; };
    auto value_at = [&](int p) { return fresh && p >= len ? nv + (size_t)(p - len) * in.ldv : V + (size_t)p * D; };
    floatx4 qf[KT];
#pragma unroll
    for (int k = 0; k < KT; ++k) qf[k] = *reinterpret_cast<const floatx4 *>(q + (size_t)(row0 + node) * ldq + (size_t)head * D + 16 * k + 4 * g);
    const float scale = 1.0f / sqrtf((float)D);
    floatx4 oacc[VH][4];
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) oacc[h][e] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m = NEG_INF, lsum = 0.f;
    for (int u = 2 * wk.v0 + wave; u < 2 * wk.v1; u += W) {
        const int p0 = 32 * wk.tiles.at(u >> 1) + 16 * (u & 1);
        if (!win_any(p0, 16, p_lo, p_hi, wc.window, wc.sinks)) continue;
        floatx4 kf[KT], vf[4][VH];
        const float *kp = key_at(min(p0 + i, seen)) + 4 * g;
#pragma unroll
        for (int k = 0; k < KT; ++k) kf[k] = *reinterpret_cast<const floatx4 *>(kp + 16 * k);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float *vp = value_at(min(p0 + 4 * g + x, seen)) + 4 * i;
#pragma unroll
            for (int h = 0; h < VH; ++h) vf[x][h] = *reinterpret_cast<const floatx4 *>(vp + 64 * h);
        }
        if (fresh && p0 + 15 >= len) {                         // append; nobody else reads these slots in this launch
            const int p = p0 + i;
            if (p >= len && p <= seen) {
#pragma unroll
                for (int k = 0; k < KT; ++k) *reinterpret_cast<floatx4 *>(K + (size_t)p * D + 16 * k + 4 * g) = kf[k];
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int pv = p0 + 4 * g + x;
                if (pv < len || pv > seen) continue;
#pragma unroll
                for (int h = 0; h < VH; ++h) *reinterpret_cast<floatx4 *>(V + (size_t)pv * D + 64 * h + 4 * i) = vf[x][h];
            }
        }
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int x = 0; x < 4; ++x) s = mfma_f32(kf[k][x], qf[k][x], s);
        const bool masked = !win_all(p0, 16, p_lo, p_hi, wc.window, wc.sinks);
        const uint32_t sees = masked ? win_sees(p0, qpos, wc.window, wc.sinks) : 0xffffu;
        float mx = NEG_INF;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            s[r] = (sees >> (4 * g + r)) & 1u ? s[r] * scale : NEG_INF;
            mx = fmaxf(mx, s[r]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx), base = m_new == NEG_INF ? 0.f : m_new, alpha = expf(m - base);
        m = m_new;
        float ps = 0.f, pr[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            pr[r] = expf(s[r] - base);
            ps += pr[r];
        }
        lsum = lsum * alpha + ps;
#pragma unroll
        for (int h = 0; h < VH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) oacc[h][e] *= alpha;
        bool odd = false;
        if (masked) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int h = 0; h < VH; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd = odd || !(fabsf(vf[x][h][e]) < INFINITY);
        }
        if (__builtin_amdgcn_ballot_w64(odd) == 0) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int h = 0; h < VH; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) oacc[h][e] = mfma_f32(vf[x][h][e], pr[x], oacc[h][e]);
        } else {
            // a weight of zero times an infinity would be a NaN: element by element over what each column attends
            for (int pp = 0; pp < 16; ++pp) {
                const int src = i + 16 * (pp >> 2);
                const float w0 = __shfl(pr[0], src, 64), w1 = __shfl(pr[1], src, 64), w2 = __shfl(pr[2], src, 64), w3 = __shfl(pr[3], src, 64);
                const float w = (pp & 3) == 0 ? w0 : (pp & 3) == 1 ? w1 : (pp & 3) == 2 ? w2 : w3;
                if (!((sees >> pp) & 1u)) continue;
                const float *vp = value_at(min(p0 + pp, seen));
#pragma unroll
                for (int h = 0; h < VH; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int r = 0; r < 4; ++r) oacc[h][e][r] = fmaf(w, vp[64 * h + 4 * (4 * g + r) + e], oacc[h][e][r]);
            }
        }
    }
    lsum += __shfl_xor(lsum, 16, 64);
    lsum += __shfl_xor(lsum, 32, 64);
    if (g == 0) { s_m[wave][i] = m; s_l[wave][i] = lsum; }
    // register r of oacc[h][e]: head element 64 h + 4 (4 g + r) + e of column i
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            *reinterpret_cast<floatx4 *>(&s_o[wave][i][64 * h + 16 * g + 4 * r]) = floatx4{oacc[h][0][r], oacc[h][1][r], oacc[h][2][r], oacc[h][3][r]};
    __syncthreads();
    const int nb = wk.runs();
    const size_t part_row = (size_t)wc.rows * hq_l;
    auto finish = [&](size_t e, int dd, const floatx4 &acc, float M, float L) {
        *reinterpret_cast<floatx4 *>(o + e * D + dd) = acc / L;
        if (wp.stat != nullptr && dd == 0) *reinterpret_cast<float2 *>(wp.stat + 2 * e) = float2{M, 1.0f / L};
    };
    for (int idx = threadIdx.x * 4; idx < 16 * D; idx += 64 * W * 4) {
        const int j = idx / D, dd = idx % D, at = rb * 16 + j;
        if (at >= R) break;
        float M = NEG_INF, L = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, s_m[w][j]);
        const float b = M == NEG_INF ? 0.f : M;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float wt = expf(s_m[w][j] - b);
            L += s_l[w][j] * wt;
            acc += *reinterpret_cast<const floatx4 *>(&s_o[w][j][dd]) * wt;
        }
        const size_t e = (size_t)(row0 + at / G) * hq_l + c * G + at % G;
        if (nb == 1) {
            finish(e, dd, acc, M, L);
        } else {
            float *po = wp.part_o + (wk.split * part_row + e) * D + dd;
            dev_store2(po, acc[0], acc[1]);
            dev_store2(po + 2, acc[2], acc[3]);
            if (dd == 0) dev_store2(wp.part_ml + 2 * (wk.split * part_row + e), M, L);
        }
    }
    if (nb == 1) return;
    if (!tree_arrive(wp.arrived + ((size_t)wk.nth * kg.hkv_l + c) * nrb + rb, nb, &s_last)) return;
    // the last block joins the runs in the order of the list; their maxima are requested all at once
    float(*s_max)[kWinMaxSplit] = reinterpret_cast<float(*)[kWinMaxSplit]>(s_o);
    for (int idx = threadIdx.x; idx < 16 * nb; idx += 64 * W) {
        const int j = idx / nb, u = idx - j * nb, at = min(rb * 16 + j, R - 1);
        s_max[j][u] = dev_load(wp.part_ml + 2 * (u * part_row + (size_t)(row0 + at / G) * hq_l + c * G + at % G));
    }
    __syncthreads();
    for (int idx = threadIdx.x * 4; idx < 16 * D; idx += 64 * W * 4) {
        const int j = idx / D, dd = idx % D, at = rb * 16 + j;
        if (at >= R) break;
        const size_t e = (size_t)(row0 + at / G) * hq_l + c * G + at % G;
        float M = NEG_INF, L = 0.f;
        for (int u = 0; u < nb; ++u) M = fmaxf(M, s_max[j][u]);
        const float b = M == NEG_INF ? 0.f : M;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int u0 = 0; u0 < nb; u0 += 4) {
            float2 ml[4], a[4], c2[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const size_t at_u = min(u0 + u, nb - 1) * part_row + e;
                ml[u] = dev_load2(wp.part_ml + 2 * at_u);
                a[u] = dev_load2(wp.part_o + at_u * D + dd);
                c2[u] = dev_load2(wp.part_o + at_u * D + dd + 2);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (u0 + u >= nb) break;
                const float wt = expf(ml[u].x - b);
                L += ml[u].y * wt;
                acc += floatx4{a[u].x, a[u].y, c2[u].x, c2[u].y} * wt;
            }
        }
        finish(e, dd, acc, M, L);
    }
}

// weights[j] += sum over rows and heads of exp(s_rj - m_r) / l_r, as in the 16-bit kernels: a block takes 16 positions, whose keys all of its waves hold; the waves
// take the rows that attend them in turn, 16 columns at a time, the next ones' requested ahead, and meet in LDS in the order of the waves.  Three prompts as above 21.5 us
// (one wave a tile of all rows 91, eight waves a block 23): the first positions, which every row attends, are the longest chain.
template <int D, int W>
__global__ __launch_bounds__(64 * W) void f32_win_weights_kernel(const float *__restrict__ q, int64_t ldq, const float *__restrict__ kc, KvGeom kg, int hq_l, int G, int tile_blocks,
                                                                 WinCall wc, const int32_t *__restrict__ lens, const float *__restrict__ stat, float *__restrict__ weights) {
    constexpr int KT = D / 16;
    __shared__ float s_sum[W][16];
    const int tb = blockIdx.x % tile_blocks, c = (blockIdx.x / tile_blocks) % kg.hkv_l, nth = blockIdx.x / tile_blocks / kg.hkv_l;
    const int seq = wc.seq0 + nth, row0 = wc.cu[nth], len = lens[seq], n = min(wc.cu[nth + 1] - row0, wc.max_seq - len), R = n * G;
    if (n <= 0) return;
    WinTiles tiles;
    tiles.set(len, len + n - 1, wc.window, wc.sinks, 0);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, i = lane & 15, g4 = lane >> 4;
    const int seen = len + n - 1;
    const float scale = 1.0f / sqrtf((float)D);
    for (int u = tb; u < 2 * tiles.nt; u += tile_blocks) {
        const int p0 = 32 * tiles.at(u >> 1) + 16 * (u & 1);
        if (p0 > seen) continue;                              // the same in every wave
        const float *kp = kc + (size_t)seq * kg.seq_stride + ((size_t)c * kg.smax + min(p0 + i, seen)) * D + 4 * g4;
        const int x_lo = max(0, p0 - len), x_hi = p0 < wc.sinks ? n - 1 : min(n - 1, p0 + 15 + wc.window - 1 - len);
        const int last = (x_hi * G + G - 1) / 16;
        floatx4 kf[KT], qf[KT];
        float2 ml;
        auto load_q = [&](int g) {
            const int rr = min(16 * g + i, R - 1), node = rr / G, head = c * G + (rr - node * G);
            const float *qp = q + (size_t)(row0 + node) * ldq + (size_t)head * D + 4 * g4;
#pragma unroll
            for (int k = 0; k < KT; ++k) qf[k] = *reinterpret_cast<const floatx4 *>(qp + 16 * k);
            ml = *reinterpret_cast<const float2 *>(stat + 2 * ((size_t)(row0 + node) * hq_l + head));
        };
        int g = x_lo * G / 16 + wave;
        if (g <= last) load_q(g);
#pragma unroll
        for (int k = 0; k < KT; ++k) kf[k] = *reinterpret_cast<const floatx4 *>(kp + 16 * k);
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        for (; g <= last; g += W) {
            // two chains of sums: an fp32 matrix instruction waits for the one before it
            floatx4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KT; ++k) {
#pragma unroll
                for (int x = 0; x < 4; x += 2) {
                    s0 = mfma_f32(kf[k][x], qf[k][x], s0);
                    s1 = mfma_f32(kf[k][x + 1], qf[k][x + 1], s1);
                }
            }
            const float2 now = ml;
            const int r = 16 * g + i, node = min(r, R - 1) / G;
            if (g + W <= last) load_q(g + W);
            const uint32_t sees = r < R ? win_sees(p0, len + node, wc.window, wc.sinks) : 0u;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float w = expf((s0[x] + s1[x]) * scale - now.x) * now.y;
                acc[x] += (sees >> (4 * g4 + x)) & 1u ? w : 0.f;
            }
        }
        float mine = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            float a = acc[x];
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) a += __shfl_xor(a, o, 64);
            mine = i == x ? a : mine;
        }
        __syncthreads();                                      // the sums of the positions before have been read
        if (i < 4) s_sum[wave][4 * g4 + i] = mine;
        __syncthreads();
        if (threadIdx.x < 16 && p0 + (int)threadIdx.x <= seen) {
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) sum += s_sum[w][threadIdx.x];
            weights[((size_t)seq * kg.hkv_l + c) * wc.max_seq + p0 + threadIdx.x] += sum;
        }
    }
}

__global__ void win_advance_kernel(int32_t *__restrict__ lens, WinCall wc) {
    const int i = threadIdx.x;
    if (i < wc.batch) lens[wc.seq0 + i] = min(lens[wc.seq0 + i] + wc.cu[i + 1] - wc.cu[i], wc.max_seq);
}

// ---- eviction ----------------------------------------------------------------------------------------------------------
// a weight's order as an unsigned number: NaN below everything, both zeros alike
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = __float_as_uint(w + 0.0f);
    return w != w ? 0u : u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A block per (layer, sequence, kv head) finds the smallest weight that stays by its digits, eight bits at a time from the top -- how many of the weights with the digits
// found so far have each value of the next one --, then goes through the slots once in order: what is first, recent, heavier than that one, or equal to it
// and among the first such as are still wanted.  The counts are integers: the result does not depend on the order of the LDS atomics.
// Bound by latency: four digits of three barriers each.  A thread has up to PER slots next to each other, so many that all threads have some; contexts of up to T PER slots are read once and stay in registers.
template <int T>
__global__ __launch_bounds__(T) void evict_select_kernel(EvictCall ec, const int32_t *__restrict__ lens) {
    constexpr int WAVES = T / 64, PER = 8;
    __shared__ unsigned s_hist[256];
    __shared__ unsigned s_prefix, s_want;
    __shared__ int s_eq[WAVES], s_take[WAVES];
    const unsigned unit = blockIdx.x;
    const int seq = (unit / ec.hkv) % ec.batch, thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    const int n = min(lens[seq], ec.max_seq), kept = min(n, ec.keep);
    const float *w = ec.w != nullptr ? ec.w + (size_t)unit * ec.max_seq : nullptr;
    float *w_out = w != nullptr ? ec.w_out + (size_t)unit * ec.dst_seq : nullptr;
    int32_t *slots = ec.slots + (size_t)unit * ec.dst_seq;
    if (w == nullptr || n <= ec.keep) {                       // by position alone
        for (int j = thread; j < ec.dst_seq; j += T) {
            slots[j] = j >= kept ? -1 : n <= ec.keep || j < ec.sinks ? j : n - ec.keep + j;
            if (w != nullptr) w_out[j] = j < kept ? w[j] : 0.f;
        }
        return;
    }
    const int c0 = ec.sinks, c1 = n - ec.recent, want = ec.keep - ec.sinks - ec.recent;       // the slots that are chosen from, and how many
    const int per = min((n + T - 1) / T, PER), pass = T * per;
    const bool once = n <= pass;
    float x[PER];
    auto load = [&](int i0) {
#pragma unroll
        for (int j = 0; j < PER; ++j) x[j] = w[min(i0 + per * thread + j, n - 1)];
    };
    if (once) load(0);
    uint32_t prefix = 0u;
    unsigned left = want;                                     // of those with the digits found so far: wanted
    if (want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = thread; i < 256; i += T) s_hist[i] = 0u;
            __syncthreads();
            const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int i0 = 0; i0 < n; i0 += pass) {
                if (!once) load(i0);
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    if (j >= per) break;
                    const int i = i0 + per * thread + j;
                    const uint32_t key = weight_key(x[j]);
                    const bool mine = i >= c0 && i < c1 && (key & mask) == prefix;
                    const unsigned digit = (key >> shift) & 255u;
                    // weights of one scale share their first digits: what has the same as the first of the wave is counted at once
                    const unsigned long long some = __builtin_amdgcn_ballot_w64(mine);
                    if (some == 0) continue;
                    const int leader = __builtin_ctzll(some);
                    const unsigned common = __builtin_amdgcn_readlane(digit, leader);
                    const unsigned long long same = __builtin_amdgcn_ballot_w64(mine && digit == common);
                    if (lane == leader) atomicAdd(&s_hist[common], (unsigned)__builtin_popcountll(same));
                    if (mine && digit != common) atomicAdd(&s_hist[digit], 1u);
                }
            }
            __syncthreads();
            if (wave == 0) {
                // lane l: digits 255 - 4 l down to 252 - 4 l; before: how many have larger digits
                unsigned h[4], sum = 0u;
#pragma unroll
                for (int d = 0; d < 4; ++d) { h[d] = s_hist[255 - 4 * lane - d]; sum += h[d]; }
                unsigned before = sum;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const unsigned up = __shfl_up(before, o, 64);
                    before += lane >= o ? up : 0u;
                }
                before -= sum;
                if (before < left && before + sum >= left) {
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        if (before < left && before + h[d] >= left) {
                            s_prefix = prefix | (unsigned)(255 - 4 * lane - d) << shift;
                            s_want = left - before;
                            before = left;                    // found
                        } else {
                            before += h[d];
                        }
                    }
                }
            }
            __syncthreads();
            prefix = s_prefix;
            left = s_want;
        }
    }
    const int limit = (int)left;                              // of the weights equal to the last one that stays
    int eq_before = 0, out_before = 0;
    for (int i0 = 0; i0 < n; i0 += pass) {
        const int first = i0 + per * thread;
        if (!once) load(i0);
        bool eq[PER], take[PER];
        int eqs = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = first + j;
            const bool there = j < per && i < n, open = there && i >= c0 && i < c1 && want > 0;
            const uint32_t key = weight_key(x[j]);
            eq[j] = open && key == prefix;
            take[j] = there && (i < c0 || i >= c1 || (open && key > prefix));
            eqs += eq[j];
        }
        int eq_rank = eqs;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(eq_rank, o, 64);
            eq_rank += lane >= o ? up : 0;
        }
        if (lane == 63) s_eq[wave] = eq_rank;
        __syncthreads();
        eq_rank += eq_before - eqs;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            eq_rank += v < wave ? s_eq[v] : 0;
            eq_before += s_eq[v];
        }
        int takes = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (eq[j]) take[j] = eq_rank++ < limit;
            takes += take[j];
        }
        int rank = takes;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(rank, o, 64);
            rank += lane >= o ? up : 0;
        }
        if (lane == 63) s_take[wave] = rank;
        __syncthreads();                                      // every weight of the pass has been read: those in front may be written
        rank += out_before - takes;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) {
            rank += v < wave ? s_take[v] : 0;
            out_before += s_take[v];
        }
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (take[j]) {
                slots[rank] = first + j;
                w_out[rank] = x[j];
                ++rank;
            }
    }
    __syncthreads();
    for (int j = kept + thread; j < ec.dst_seq; j += T) {
        slots[j] = -1;
        w_out[j] = 0.f;
    }
}

// The kept rows, as in the 16-bit kernel: chunks of 32 rows, read whole before they are written; one block for all chunks in place, four at a time
template <int D, bool ROT, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS) void f32_evict_move_kernel(EvictCall ec, EvictMove mv, int blocks) {
    constexpr int P4 = D / 4, PIECES = 32 * P4 / 256, HALF = D / 2;
    __shared__ int s_slots[GROUPS][32];
    const int group = threadIdx.x / 256, thread = threadIdx.x % 256;
    int *s_slot = s_slots[group];
    const unsigned unit = blockIdx.x / (unsigned)blocks;
    const int chunk = (int)(blockIdx.x % (unsigned)blocks), c = unit % ec.hkv, b = (unit / ec.hkv) % ec.batch, layer = unit / ec.hkv / ec.batch;
    const int32_t *slots = ec.slots + (size_t)unit * ec.dst_seq;
    const size_t src = (size_t)layer * mv.src_layer + (size_t)b * mv.src.seq_stride + (size_t)c * mv.src.smax * D;
    const size_t dst = (size_t)layer * mv.dst_layer + (size_t)b * mv.dst.seq_stride + (size_t)c * mv.dst.smax * D;
    const float *ks = static_cast<const float *>(mv.ks) + src, *vs = static_cast<const float *>(mv.vs) + src;
    float *kd = static_cast<float *>(mv.kd) + dst, *vd = static_cast<float *>(mv.vd) + dst;
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < mv.dst_batch; i += 256 * GROUPS) mv.dst_lens[i] = i < ec.batch ? min(min(mv.lens[i], ec.max_seq), ec.keep) : 0;
    const int most = min(ec.keep, ec.dst_seq);
    for (int first = 32 * GROUPS * chunk; first < most; first += 32 * GROUPS * blocks) {
        const int j0 = first + 32 * group;
        __syncthreads();
        if (thread < 32) s_slot[thread] = j0 + thread < most ? slots[j0 + thread] : -1;
        __syncthreads();
        const bool moves = s_slot[0] >= 0 && !(mv.ks == mv.kd && s_slot[31] == j0 + 31);
        floatx4 k[PIECES], v[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int idx = thread + 256 * i, at = max(s_slot[idx / P4], 0), dd = 4 * (idx % P4);
            k[i] = *reinterpret_cast<const floatx4 *>(ks + (size_t)at * D + dd);
            v[i] = *reinterpret_cast<const floatx4 *>(vs + (size_t)at * D + dd);
            if constexpr (ROT) {
                const floatx4 o = *reinterpret_cast<const floatx4 *>(ks + (size_t)at * D + (dd < HALF ? dd + HALF : dd - HALF));
                const int moved = max(at - (j0 + idx / P4), 0), i0 = dd < HALF ? dd : dd - HALF;
                const floatx4 cs = *reinterpret_cast<const floatx4 *>(mv.cos_tab + (size_t)moved * HALF + i0);
                const floatx4 sn = *reinterpret_cast<const floatx4 *>(mv.sin_tab + (size_t)moved * HALF + i0);
                if (moved != 0) k[i] = dd < HALF ? k[i] * cs + o * sn : k[i] * cs - o * sn;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int idx = thread + 256 * i, row = idx / P4, dd = 4 * (idx % P4);
            if (!moves || s_slot[row] < 0) continue;
            *reinterpret_cast<floatx4 *>(kd + (size_t)(j0 + row) * D + dd) = k[i];
            *reinterpret_cast<floatx4 *>(vd + (size_t)(j0 + row) * D + dd) = v[i];
        }
    }
}

}  // namespace

void f32_launch_win_rope_append(const float *qkv, int hq_l, KvGeom kg, const WinCall &wc, const int32_t *lens, const float *cos_tab, const float *sin_tab,
                                float *q, float *kc, float *vc, hipStream_t s) {
    const unsigned n = (unsigned)(wc.cu[wc.batch] - wc.cu[0]) * (hq_l + 2 * kg.hkv_l) * (kg.d / 2);
    hipLaunchKernelGGL(f32_win_rope_append_kernel, dim3((n + 255) / 256), dim3(256), 0, s, qkv, hq_l, kg, wc, lens, cos_tab, sin_tab, q, kc, vc);
}
void f32_launch_win_append(const TreeIn &in, float *kc, float *vc, KvGeom kg, const WinCall &wc, const int32_t *lens, hipStream_t s) {
    const int64_t pieces = (int64_t)wc.max_n * kg.hkv_l * (kg.d / 4);
    const dim3 grid((unsigned)std::min<int64_t>((pieces + 255) / 256, 1 << 16), 1, wc.batch);
    hipLaunchKernelGGL(f32_win_append_kernel, grid, dim3(256), 0, s, in, kc, vc, kg, wc, lens);
}
void f32_launch_win_attn(const float *q, int64_t ldq, const TreeIn &in, float *kc, float *vc, KvGeom kg, int hq_l, const WinCall &wc, const int32_t *lens,
                         const WinPlan &wp, float *o, hipStream_t s) {
    const int G = hq_l / kg.hkv_l, nrb = win_row_blocks(wc.max_n, G, 16);
    const dim3 grid(win_grid(wc.batch * kg.hkv_l * wp.nsplit, nrb));
    if (kg.d == 128) hipLaunchKernelGGL((f32_win_attn_kernel<128, 4>), grid, dim3(256), 0, s, q, ldq, in, kc, vc, kg, hq_l, G, nrb, wc, lens, wp, o);
    else hipLaunchKernelGGL((f32_win_attn_kernel<64, 4>), grid, dim3(256), 0, s, q, ldq, in, kc, vc, kg, hq_l, G, nrb, wc, lens, wp, o);
}
void f32_launch_win_weights(const float *q, int64_t ldq, const float *kc, KvGeom kg, int hq_l, const WinCall &wc, const int32_t *lens, const float *stat,
                            float *weights, const WinReach &reach, hipStream_t s) {
    const int G = hq_l / kg.hkv_l, tile_blocks = 2 * reach.most;
    const dim3 grid((unsigned)tile_blocks * kg.hkv_l * wc.batch);
    if (kg.d == 128) hipLaunchKernelGGL((f32_win_weights_kernel<128, 4>), grid, dim3(256), 0, s, q, ldq, kc, kg, hq_l, G, tile_blocks, wc, lens, stat, weights);
    else hipLaunchKernelGGL((f32_win_weights_kernel<64, 4>), grid, dim3(256), 0, s, q, ldq, kc, kg, hq_l, G, tile_blocks, wc, lens, stat, weights);
}
void launch_win_advance(int32_t *lens, const WinCall &wc, hipStream_t s) {
    hipLaunchKernelGGL(win_advance_kernel, dim3(1), dim3(kWinSeqs), 0, s, lens, wc);
}
// Small contexts in four waves, whose barriers cost less than more lanes gain: 333 slots 8.8 us in 256 threads, in 1024 10.6; 4000 slots 13.5 us in
// 1024 and 15 in 512
void launch_evict_select(const EvictCall &ec, int longest, const int32_t *lens, hipStream_t s) {
    const dim3 grid((unsigned)ec.layers * ec.batch * ec.hkv);
    if (longest <= 1024) hipLaunchKernelGGL(evict_select_kernel<256>, grid, dim3(256), 0, s, ec, lens);
    else hipLaunchKernelGGL(evict_select_kernel<1024>, grid, dim3(1024), 0, s, ec, lens);
}
void f32_launch_evict_move(const EvictCall &ec, const EvictMove &mv, hipStream_t s) {
    const int blocks = evict_blocks(ec, mv);
    const dim3 grid((unsigned)blocks * ec.layers * ec.batch * ec.hkv);
#define HX_MOVE(DD, R)                                                                                                                     \
    do {                                                                                                                                   \
        if (mv.ks == mv.kd) hipLaunchKernelGGL((f32_evict_move_kernel<DD, R, 4>), grid, dim3(1024), 0, s, ec, mv, blocks);                  \
        else hipLaunchKernelGGL((f32_evict_move_kernel<DD, R, 1>), grid, dim3(256), 0, s, ec, mv, blocks);                                  \
    } while (0)
    if (mv.src.d == 128) { if (mv.cos_tab != nullptr) HX_MOVE(128, true); else HX_MOVE(128, false); }
    else { if (mv.cos_tab != nullptr) HX_MOVE(64, true); else HX_MOVE(64, false); }
#undef HX_MOVE
}
