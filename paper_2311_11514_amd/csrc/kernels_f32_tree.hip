// Attention of drafted trees over the cache, fp32 stages (cache [seq][kv head][smax][d]), and what does not depend on the type: acceptance.
#include "kernels.h"

#define NEG_INF (-INFINITY)

namespace {

__device__ __forceinline__ floatx4 mfma_f32(float a, float b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// raw projection [rows][(hq + 2 hkv) d] -> rotary embedding at len + depth, q as plain rows, k and v into the cache; a rotary pair per thread
__global__ __launch_bounds__(256) void f32_tree_rope_append_kernel(const float *__restrict__ qkv, int hq_l, KvGeom kg, TreeView tv,
                                                                   const int32_t *__restrict__ lens, const float *__restrict__ cos_tab,
                                                                   const float *__restrict__ sin_tab, float *__restrict__ q,
                                                                   float *__restrict__ kc, float *__restrict__ vc) {
    const int d = kg.d, half = d >> 1, heads = hq_l + 2 * kg.hkv_l;
    const unsigned idx = blockIdx.x * 256u + threadIdx.x, per_row = heads * half;
    if (idx >= tv.rows * per_row) return;
    const int t = idx / per_row, rem = idx - t * per_row, head = rem / half, i = rem - head * half;
    const TreeRow row = tv.row[t];
    const int len = lens[row.seq], slot = len + row.index;
    if (slot >= kg.smax) return;
    const float *src = qkv + (size_t)t * heads * d + (size_t)head * d + i;
    float lo = src[0], hi = src[half];
    if (head < hq_l + kg.hkv_l) {
        const size_t at = (size_t)(len + row.depth) * half + i;
        const float c = cos_tab[at], sn = sin_tab[at], l = lo * c - hi * sn;
        hi = hi * c + lo * sn;
        lo = l;
    }
    const size_t slab = (size_t)row.seq * kg.seq_stride;
    float *dst = head < hq_l ? q + ((size_t)t * hq_l + head) * d
                 : head < hq_l + kg.hkv_l ? kc + slab + ((size_t)(head - hq_l) * kg.smax + slot) * d
                                          : vc + slab + ((size_t)(head - hq_l - kg.hkv_l) * kg.smax + slot) * d;
    dst[i] = lo;
    dst[half + i] = hi;
}

// A block takes 16 query columns of one (sequence, kv head) -- column j: node j / G, head j % G -- and a run of 16-position tiles, over
// which its W waves interleave; the products and register layouts are those of the stage's fp32 attention (v_mfma_f32_16x16x4_f32, a
// lane owns column l % 16 and positions 4 (l / 16) + r, P stays in registers).  Rows that are not in the cache yet (in.k != NULL) are read from the
// caller's and appended by the first block of columns.  Masks, runs and the way of values that are not finite as in the 16-bit kernel.
// Bound by the fp32 matrix instructions, 32 cycles for 4 KB of K or V, and by the one round trip per tile and wave: d 128, 16 query and 4 kv heads, four
// sequences of 2048 with 8 nodes 22.5 us, eight of 600, one kv head 15.3; d 64, a context of 40 with five nodes 5.7, half of that the launch.
template <int D, int W>
__global__ __launch_bounds__(64 * W) void f32_tree_attn_kernel(const float *__restrict__ q, int64_t ldq, TreeIn in, float *kc, float *vc, KvGeom kg, int hq_l, int G, int nrb,
                                                               TreeView tv, const int32_t *__restrict__ lens, TreePlan tp, float *__restrict__ o) {
    constexpr int KT = D / 16, VH = D / 64;
    __shared__ float s_m[W][16], s_l[W][16];
    __shared__ __align__(16) float s_o[W][16][D];
    __shared__ int s_last;
    const int slot = blockIdx.x >> 3, rb = slot % nrb;
    int combo = (slot / nrb) * 8 + (blockIdx.x & 7);
    if (combo >= tv.batch * kg.hkv_l * tp.nsplit) return;
    const int split = combo % tp.nsplit;
    combo /= tp.nsplit;
    const int c = combo % kg.hkv_l, nth = combo / kg.hkv_l, seq = nth < kTreeOrdered ? tp.order[nth] : nth;
    const int row0 = tv.cu[seq], n = tv.cu[seq + 1] - row0, R = n * G;
    if (rb * 16 >= R) return;
    const int len = lens[seq], last = min(len + n, kg.smax) - 1, nt = (last + 32) >> 5;      // runs count 32 positions, as for 16 bits
    const int per = max(tp.chunk, (nt + tp.nsplit - 1) / tp.nsplit), t0 = split * per;
    if (t0 >= nt) return;
    const int t1 = min(2 * (t0 + per), (last >> 4) + 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int rr = min(rb * 16 + i, R - 1), node = rr / G, head = c * G + (rr - node * G);
    const uint32_t *mask = tv.mask + (size_t)(row0 + node) * tv.mask_words;
    const size_t slab = (size_t)seq * kg.seq_stride + (size_t)c * kg.smax * D;
    float *K = kc + slab, *V = vc + slab;
    const float *nk = in.k != nullptr ? static_cast<const float *>(in.k) + (size_t)row0 * in.ldk + c * D : nullptr;
    const float *nv = in.k != nullptr ? static_cast<const float *>(in.v) + (size_t)row0 * in.ldv + c * D : nullptr;
    // position p of the keys and values: the cache's, or the tree's row that will be there
    auto key_at = [&](int p) { return nk != nullptr && p >= len ? nk + (size_t)(p - len) * in.ldk : K + (size_t)p * D; };
    auto value_at = [&](int p) { return nv != nullptr && p >= len ? nv + (size_t)(p - len) * in.ldv : V + (size_t)p * D; };
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
    for (int t = 2 * t0 + wave; t < t1; t += W) {
        floatx4 kf[KT], vf[4][VH];
        const float *kp = key_at(min(16 * t + i, last)) + 4 * g;
#pragma unroll
        for (int k = 0; k < KT; ++k) kf[k] = *reinterpret_cast<const floatx4 *>(kp + 16 * k);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float *vp = value_at(min(16 * t + 4 * g + x, last)) + 4 * i;
#pragma unroll
            for (int h = 0; h < VH; ++h) vf[x][h] = *reinterpret_cast<const floatx4 *>(vp + 64 * h);
        }
        const bool masked = 16 * t + 15 >= len;
        if (masked && nk != nullptr && rb == 0) {              // append; nobody reads these slots in this launch
            const int p = 16 * t + i;
            if (p >= len && p <= last) {
#pragma unroll
                for (int k = 0; k < KT; ++k) *reinterpret_cast<floatx4 *>(K + (size_t)p * D + 16 * k + 4 * g) = kf[k];
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int pv = 16 * t + 4 * g + x;
                if (pv < len || pv > last) continue;
#pragma unroll
                for (int h = 0; h < VH; ++h) *reinterpret_cast<floatx4 *>(V + (size_t)pv * D + 64 * h + 4 * i) = vf[x][h];
            }
        }
        floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int x = 0; x < 4; ++x) s = mfma_f32(kf[k][x], qf[k][x], s);
        uint32_t sees = 0xffffu;                              // of the tile's 16 positions
        if (masked) {
            const int rel = 16 * t - len;
            if (rel < 0) {
                sees = (mask[0] << -rel) | ((1u << -rel) - 1);
            } else {
                const int w = rel >> 5, sh = rel & 31;
                const uint32_t a = w < tv.mask_words ? mask[w] : 0u, b = w + 1 < tv.mask_words ? mask[w + 1] : 0u;
                sees = sh == 0 ? a : (a >> sh) | (b << (32 - sh));
            }
        }
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
            for (int pp = 0; pp < 16; ++pp) {
                const int src = i + 16 * (pp >> 2);
                const float w0 = __shfl(pr[0], src, 64), w1 = __shfl(pr[1], src, 64), w2 = __shfl(pr[2], src, 64), w3 = __shfl(pr[3], src, 64);
                const float w = (pp & 3) == 0 ? w0 : (pp & 3) == 1 ? w1 : (pp & 3) == 2 ? w2 : w3;
                if (!((sees >> pp) & 1u)) continue;
                const float *vp = value_at(min(16 * t + pp, last));
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
    const int nb = (nt + per - 1) / per;
    const size_t part_row = (size_t)tv.rows * hq_l;
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
            *reinterpret_cast<floatx4 *>(o + e * D + dd) = acc / L;
        } else {
            float *po = tp.part_o + (split * part_row + e) * D + dd;
            dev_store2(po, acc[0], acc[1]);
            dev_store2(po + 2, acc[2], acc[3]);
            if (dd == 0) dev_store2(tp.part_ml + 2 * (split * part_row + e), M, L);
        }
    }
    if (nb == 1) return;
    if (!tree_arrive(tp.arrived + ((size_t)seq * kg.hkv_l + c) * nrb + rb, nb, &s_last)) return;
    // the last block joins the runs in the order of the context; their maxima are requested all at once
    float(*s_max)[kTreeMaxSplit] = reinterpret_cast<float(*)[kTreeMaxSplit]>(s_o);
    for (int idx = threadIdx.x; idx < 16 * nb; idx += 64 * W) {
        const int j = idx / nb, u = idx - j * nb, at = min(rb * 16 + j, R - 1);
        s_max[j][u] = dev_load(tp.part_ml + 2 * (u * part_row + (size_t)(row0 + at / G) * hq_l + c * G + at % G));
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
                ml[u] = dev_load2(tp.part_ml + 2 * at_u);
                a[u] = dev_load2(tp.part_o + at_u * D + dd);
                c2[u] = dev_load2(tp.part_o + at_u * D + dd + 2);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (u0 + u >= nb) break;
                const float wt = expf(ml[u].x - b);
                L += ml[u].y * wt;
                acc += floatx4{a[u].x, a[u].y, c2[u].x, c2[u].y} * wt;
            }
        }
        *reinterpret_cast<floatx4 *>(o + e * D + dd) = acc / L;
    }
}

// slot len + path[j] -> len + j in every layer, one element of K and V per thread (see the 16-bit kernel for the order)
__global__ __launch_bounds__(256) void f32_tree_keep_kernel(float *__restrict__ kc, float *__restrict__ vc, int64_t layer_stride, KvGeom kg,
                                                            const int32_t *__restrict__ lens, const int32_t *__restrict__ cu,
                                                            const int32_t *__restrict__ kept, const int32_t *__restrict__ path) {
    const int seq = blockIdx.y, dd = (blockIdx.x * 256 + threadIdx.x) % kg.d, c = (blockIdx.x * 256 + threadIdx.x) / kg.d;
    const int n = kept[seq], len = lens[seq], row0 = cu[seq];
    if (c >= kg.hkv_l || len + n > kg.smax) return;
    const size_t slab = (size_t)blockIdx.z * layer_stride + (size_t)seq * kg.seq_stride + (size_t)c * kg.smax * kg.d + dd;
    float *ks = kc + slab, *vs = vc + slab;
    for (int j0 = 1; j0 < n; j0 += 8) {
        float a[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const size_t src = (size_t)(len + path[row0 + min(j0 + i, n - 1)]) * kg.d;
            a[i] = ks[src];
            b[i] = vs[src];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j0 + i < n) {
                ks[(size_t)(len + j0 + i) * kg.d] = a[i];
                vs[(size_t)(len + j0 + i) * kg.d] = b[i];
            }
    }
}

// a path that would pass the cache (replayed steps have taken its length beyond what the host knows) has not been moved and is not counted either
__global__ void tree_advance_kernel(int32_t *__restrict__ lens, const int32_t *__restrict__ kept, int batch, int smax) {
    const int i = blockIdx.x * 64 + threadIdx.x;
    if (i < batch && lens[i] + kept[i] <= smax) lens[i] += kept[i];
}

// One wave per sequence walks its tree: the 64 lanes look at four nodes each for the first child of the current node whose drafted
// token is the chosen one.  Bound by latency: a step is a ballot and two reads of LDS (one tree of 26 nodes 1.9 us, 64 of 4 .. 64 nodes 3.0).
__global__ __launch_bounds__(64) void tree_accept_kernel(TreeView tv, const int32_t *__restrict__ draft, const int32_t *__restrict__ chosen,
                                                         int32_t *__restrict__ kept, int32_t *__restrict__ path, int32_t *__restrict__ tokens) {
    constexpr int PL = kTreeMaxNodes / 64;
    __shared__ int32_t s_chosen[kTreeMaxNodes];
    const int seq = blockIdx.x, lane = threadIdx.x, row0 = tv.cu[seq], n = tv.cu[seq + 1] - row0;
    int parent[PL], token[PL];
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        const int x = 64 * i + lane;
        parent[i] = -2;                                       // no node: nobody's child
        token[i] = 0;
        if (x < n) {
            parent[i] = tv.row[row0 + x].parent;
            token[i] = draft[row0 + x];
            s_chosen[x] = chosen[row0 + x];
        }
    }
    __syncthreads();
    int count = 0, at = n > 0 ? 0 : -1;
    while (at >= 0) {
        const int want = s_chosen[at];
        if (lane == 0) { path[row0 + count] = at; tokens[row0 + count] = want; }
        ++count;
        int next = -1;
#pragma unroll
        for (int i = 0; i < PL; ++i) {
            if (64 * i >= n) break;
            const unsigned long long hit = __builtin_amdgcn_ballot_w64(parent[i] == at && token[i] == want);
            if (next < 0 && hit != 0) next = 64 * i + __builtin_ctzll(hit);
        }
        at = next;                                            // children have larger indexes than their parents: the walk ends
    }
    for (int x = count + lane; x < n; x += 64) { path[row0 + x] = -1; tokens[row0 + x] = -1; }
    if (lane == 0) kept[seq] = count;
}

}  // namespace

void launch_tree_accept(const TreeView &tv, const int32_t *draft, const int32_t *chosen, int32_t *kept, int32_t *path, int32_t *tokens, hipStream_t s) {
    hipLaunchKernelGGL(tree_accept_kernel, dim3(tv.batch), dim3(64), 0, s, tv, draft, chosen, kept, path, tokens);
}
void launch_tree_advance(int32_t *lens, const int32_t *kept, int batch, int smax, hipStream_t s) {
    hipLaunchKernelGGL(tree_advance_kernel, dim3((batch + 63) / 64), dim3(64), 0, s, lens, kept, batch, smax);
}
void f32_launch_tree_rope_append(const float *qkv, int hq_l, KvGeom kg, const TreeView &tv, const int32_t *lens, const float *cos_tab,
                                 const float *sin_tab, float *q, float *kc, float *vc, hipStream_t s) {
    const unsigned n = (unsigned)tv.rows * (hq_l + 2 * kg.hkv_l) * (kg.d / 2);
    hipLaunchKernelGGL(f32_tree_rope_append_kernel, dim3((n + 255) / 256), dim3(256), 0, s, qkv, hq_l, kg, tv, lens, cos_tab, sin_tab, q, kc, vc);
}
void f32_launch_tree_attn(const float *q, int64_t ldq, const TreeIn &in, float *kc, float *vc, KvGeom kg, int hq_l, const TreeView &tv, const int32_t *lens,
                          const TreePlan &tp, float *o, hipStream_t s) {
    const int G = hq_l / kg.hkv_l, nrb = tree_row_blocks(tv.max_n, G, 16);
    const dim3 grid((unsigned)nrb * (unsigned)((tv.batch * kg.hkv_l * tp.nsplit + 7) / 8 * 8));
    if (kg.d == 128) hipLaunchKernelGGL((f32_tree_attn_kernel<128, 4>), grid, dim3(256), 0, s, q, ldq, in, kc, vc, kg, hq_l, G, nrb, tv, lens, tp, o);
    else hipLaunchKernelGGL((f32_tree_attn_kernel<64, 4>), grid, dim3(256), 0, s, q, ldq, in, kc, vc, kg, hq_l, G, nrb, tv, lens, tp, o);
}
void f32_launch_tree_keep(float *kc, float *vc, int64_t layer_stride, int layers, KvGeom kg, int batch, const int32_t *lens, const int32_t *cu,
                          const int32_t *kept, const int32_t *path, hipStream_t s) {
    for (int l0 = 0; l0 < layers; l0 += 65535) {
        const dim3 grid((kg.hkv_l * kg.d + 255) / 256, batch, layers - l0 < 65535 ? layers - l0 : 65535);
        hipLaunchKernelGGL(f32_tree_keep_kernel, grid, dim3(256), 0, s, kc + l0 * layer_stride, vc + l0 * layer_stride, layer_stride, kg, lens, cu, kept, path);
    }
}
