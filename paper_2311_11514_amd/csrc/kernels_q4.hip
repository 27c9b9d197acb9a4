// Products of a few rows with a matrix of 4-bit weights that carry a scale, and possibly a zero point, per group of input features:
//   y[t][n] = sum over groups g of s[g][n] * sum over k in g of (q[k][n] - z[g][n]) * x[t][k],   q, z = 0 .. 15.
//
// The matrix instructions take the weights as 16 + q: a nibble in the top mantissa bits of 1.0 * 2^4 (bf16: bits 3 .. 6 under
// 0x4180, fp16: bits 6 .. 9 under 0x4c00) is that number exactly, one shift and one and-or per pair.  A group's sum S over (16 + q) x and
// the sum X over x alone (the same operand against ones: it arrives in the lanes that need it) give s * (S - (16 + z) X); products of
// 5-bit and 8- or 11-bit numbers are exact in fp32, and 16 is the smallest offset that needs no arithmetic on the weights, so that S
// and its sum with X lose little of what the group's sum has.
// fp32 rows are cut into three bf16 parts of 8 bits each, exactly, that take three columns of the operand; their products are added
// up per part and joined at the end.
//
// Layout: blocks of 16 columns x 128 input features, 1 KB, [k / 128][n / 16][lane][4 words]: word i of lane l holds features
// 128 kq + 32 i + 8 (l / 16) + 0 .. 7 of column 16 tile + l % 16, feature 2 p + h in bits 16 h + 4 p: what one lane of
// v_mfma_f32_16x16x32 contributes to four steps, in one 16-byte request.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((__vector_size__(16))) __bf16 b16x8;
typedef __attribute__((__vector_size__(16))) _Float16 f16x8;

__device__ __forceinline__ float bf16_f32(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float f16_f32(uint32_t v) {
    const uint16_t u = (uint16_t)v;
    _Float16 h;
    __builtin_memcpy(&h, &u, 2);
    return (float)h;
}
__device__ __forceinline__ uint16_t to_bf16(float x) {
    const __bf16 b = (__bf16)x;
    uint16_t u;
    __builtin_memcpy(&u, &b, 2);
    return u;
}
__device__ __forceinline__ uint16_t to_f16(float x) {
    const _Float16 b = (_Float16)x;
    uint16_t u;
    __builtin_memcpy(&u, &b, 2);
    return u;
}

template <bool F16>
__device__ __forceinline__ floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
}
// eight nibbles -> eight times 16 + q
template <bool F16>
__device__ __forceinline__ u32x4 widen(uint32_t w) {
    if constexpr (F16)
        return u32x4{((w << 6) & 0x03c003c0u) | 0x4c004c00u, ((w << 2) & 0x03c003c0u) | 0x4c004c00u, ((w >> 2) & 0x03c003c0u) | 0x4c004c00u,
                     ((w >> 6) & 0x03c003c0u) | 0x4c004c00u};
    else
        return u32x4{((w << 3) & 0x00780078u) | 0x41804180u, ((w >> 1) & 0x00780078u) | 0x41804180u, ((w >> 5) & 0x00780078u) | 0x41804180u,
                     ((w >> 9) & 0x00780078u) | 0x41804180u};
}

// four neighbouring columns' scales, as they are loaded and as fp32
template <int ST> using scale_raw = std::conditional_t<ST == HX_T_F32, floatx4, uint2>;
template <int ST>
__device__ __forceinline__ floatx4 scale4(const scale_raw<ST> &v) {
    if constexpr (ST == HX_T_F32) return v;
    else if constexpr (ST == HX_T_BF16) return floatx4{bf16_f32(v.x & 0xffffu), bf16_f32(v.x >> 16), bf16_f32(v.y & 0xffffu), bf16_f32(v.y >> 16)};
    else return floatx4{f16_f32(v.x & 0xffffu), f16_f32(v.x >> 16), f16_f32(v.y & 0xffffu), f16_f32(v.y >> 16)};
}

// x columns of one 32-feature step (fragments of the second operand) for a 128-feature block of UT weight tiles: acc += this block's share
template <bool F16, int ST, int NB, int UT, int FL, typename XF>
__device__ __forceinline__ void contract_block(const u32x4 (&w)[UT], const scale_raw<ST> (&s)[UT][4 / FL], const uint32_t (&z)[UT][4 / FL], bool zeros, XF x,
                                               floatx4 (&acc)[UT][NB]) {
    const uint32_t one = F16 ? 0x3c003c00u : 0x3f803f80u;
    const u32x4 ones = {one, one, one, one};
#pragma unroll
    for (int f = 0; f < 4 / FL; ++f) {
        floatx4 X[NB], S[UT][NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            X[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < UT; ++u) S[u][b] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int st = f * FL; st < f * FL + FL; ++st) {
            u32x4 a[UT];
#pragma unroll
            for (int u = 0; u < UT; ++u) a[u] = widen<F16>(w[u][st]);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const u32x4 xb = x(st, b);
                X[b] = mfma<F16>(ones, xb, X[b]);
#pragma unroll
                for (int u = 0; u < UT; ++u) S[u][b] = mfma<F16>(a[u], xb, S[u][b]);
            }
        }
#pragma unroll
        for (int u = 0; u < UT; ++u) {
            const floatx4 s4 = scale4<ST>(s[u][f]);
            floatx4 z4 = {24.f, 24.f, 24.f, 24.f};
            if (zeros) {
#pragma unroll
                for (int r = 0; r < 4; ++r) z4[r] = 16.f + (float)((z[u][f] >> (8 * r)) & 255u);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[u][b][r] = fmaf(s4[r], fmaf(-z4[r], X[b][r], S[u][b][r]), acc[u][b][r]);
        }
        if (FL < 4) {                                           // one group's sums at a time: side by side they do not fit the registers
#pragma unroll
            for (int u = 0; u < UT; ++u)
#pragma unroll
                for (int b = 0; b < NB; ++b) asm volatile("" : "+v"(acc[u][b]));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}
// the scales (and zero points) of a 128-feature block for four columns from `col` on
template <int ST, int NF>
__device__ __forceinline__ void load_scales(const Q4View &m, int kq, int col, scale_raw<ST> (&s)[NF], uint32_t (&z)[NF]) {
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        const size_t at = (size_t)((kq * 128 + f * (128 / NF)) / m.group) * (m.n_tiles * 16) + col;
        s[f] = *reinterpret_cast<const scale_raw<ST> *>(static_cast<const unsigned char *>(m.scales) + at * (ST == HX_T_F32 ? 4 : 2));
        if (m.zeros != nullptr) z[f] = *reinterpret_cast<const uint32_t *>(m.zeros + at);
    }
}
__device__ __forceinline__ void store_pair(const Q4Out &out, size_t at, float a, float b) {
    if (out.type == HX_T_F32) *reinterpret_cast<float2 *>(static_cast<float *>(out.y) + at) = float2{a, b};
    else if (out.type == HX_T_BF16) *reinterpret_cast<uint32_t *>(static_cast<h16_t *>(out.y) + at) = to_bf16(a) | (uint32_t)to_bf16(b) << 16;
    else *reinterpret_cast<uint32_t *>(static_cast<h16_t *>(out.y) + at) = to_f16(a) | (uint32_t)to_f16(b) << 16;
}
// four columns from n0 on of row t (n_valid is even, so that columns come in pairs)
__device__ __forceinline__ void store_columns(const Q4View &m, const Q4Out &out, int t, int n0, floatx4 v) {
#pragma unroll
    for (int h = 0; h < 4; h += 2)
        if (n0 + h < m.n_valid) store_pair(out, (size_t)t * m.n_valid + n0 + h, v[h], v[h + 1]);
}
__device__ __forceinline__ void take_best(const Q4View &m, int n0, floatx4 v, float &bv, int &bi) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (n0 + r < m.n_valid && (v[r] > bv || (v[r] == bv && n0 + r < bi))) { bv = v[r]; bi = n0 + r; }
}
template <int N>
__device__ __forceinline__ void best_of_lanes(float &bv, int &bi) {
#pragma unroll
    for (int o = 1; o < N; o <<= 1) {
        const float ov = __shfl_xor(bv, o, 64);
        const int oi = __shfl_xor(bi, o, 64);
        if (ov > bv || (ov == bv && oi < bi)) { bv = ov; bi = oi; }
    }
}

// Up to 16 operand columns (rows times parts; columns beyond C repeat the last one and are not stored).  A block of eight waves owns UT
// tiles of 16 columns over the whole contraction; its waves take the 128-feature blocks in turn and are summed through LDS in wave order, so
// that no partial result leaves the block.  A wave holds R blocks with their operands and scales in registers, requested that far ahead.
// Bound by HBM on wide matrices, on small ones by the launch and one round trip.
// FL: 32-feature steps of a scale's group inside a 128-feature block (4: groups of 128 and more).
template <bool F16, int ST, int UT, int FL>
__global__ __launch_bounds__(512) void q4_few_kernel(Q4View m, const h16_t *__restrict__ x, int64_t ldx, int C, int T, Q4Out out) {
    constexpr int W = 8, NF = 4 / FL, R = FL == 4 ? 4 : 2;
    __shared__ floatx4 red[W][UT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int tile0 = blockIdx.x * UT;
    const u32x4 *wp[UT];
    int col[UT];
#pragma unroll
    for (int u = 0; u < UT; ++u) {
        const int t = min(tile0 + u, m.n_tiles - 1);           // a last tile of its own: the block's second repeats it, not stored
        wp[u] = static_cast<const u32x4 *>(m.w) + (size_t)t * 64 + lane;
        col[u] = t * 16 + 4 * g;
    }
    const h16_t *xp = x + (size_t)min(j, C - 1) * ldx + 8 * g;
    floatx4 acc[UT][1];
#pragma unroll
    for (int u = 0; u < UT; ++u) acc[u][0] = floatx4{0.f, 0.f, 0.f, 0.f};
    u32x4 wr[R][UT], xr[R][4];
    scale_raw<ST> sr[R][UT][NF];
    uint32_t zr[R][UT][NF];
    const size_t kstride = (size_t)m.n_tiles * 64;
    auto request = [&](int i, int kq) {
#pragma unroll
        for (int u = 0; u < UT; ++u) wr[i][u] = __builtin_nontemporal_load(wp[u] + (size_t)kq * kstride);
#pragma unroll
        for (int u = 0; u < UT; ++u) load_scales<ST, NF>(m, kq, col[u], sr[i][u], zr[i][u]);
#pragma unroll
        for (int s = 0; s < 4; ++s) xr[i][s] = *reinterpret_cast<const u32x4 *>(xp + kq * 128 + s * 32);
    };
    // ring slot i holds block wave + i W of the round; past the last block a slot re-reads it and is not used
    const int last = m.k_blocks - 1;
#pragma unroll
    for (int i = 0; i < R; ++i) request(i, min(wave + i * W, last));
    for (int k0 = wave; k0 <= last; k0 += R * W) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (k0 + i * W <= last) contract_block<F16, ST, 1, UT, FL>(wr[i], sr[i], zr[i], m.zeros != nullptr, [&](int s, int) { return xr[i][s]; }, acc);
            request(i, min(k0 + (i + R) * W, last));
        }
    }
#pragma unroll
    for (int u = 0; u < UT; ++u) red[wave][u][lane] = acc[u][0];
    __syncthreads();
    // four columns of one row per thread: waves in order, parts in order
    const int P = C / T, idx = threadIdx.x;
    if (idx >= T * UT * 4) return;
    const int t = idx / (UT * 4), u = (idx >> 2) % UT, gg = idx & 3;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < P; ++p) {
        floatx4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) a += red[w][u][p * T + t + 16 * gg];
        v += a;
    }
    const int n0 = (tile0 + u) * 16 + 4 * gg;
    if (out.best_val == nullptr) {
        store_columns(m, out, t, n0, v);
        return;
    }
    float bv = -INFINITY;
    int bi = 0x7fffffff;
    take_best(m, n0, v, bv, bi);
    best_of_lanes<UT * 4>(bv, bi);                              // the row's UT * 4 threads are neighbours
    if (idx % (UT * 4) == 0) {
        out.best_val[(size_t)t * gridDim.x + blockIdx.x] = bv;
        out.best_id[(size_t)t * gridDim.x + blockIdx.x] = bi;
    }
}

// More operand columns: the operand outweighs the weights that a tile of 16 columns has, so the eight waves of a block own eight times UT
// neighbouring tiles and walk the same 128-feature blocks, whose operand they share through LDS (two buffers, one barrier a step).  The contraction
// is split over blockIdx.y where the matrix has too few columns for the chip.  Results that need no more adding up (one split, one
// part) are stored from here; everything else goes to `part` [split][column of the operand][16 n_tiles] and q4_finish_kernel.
// Bound by HBM up to some 40 columns, beyond by the matrix instructions and the work on the weights beside them.
template <bool F16, int ST, int NB, int UT, int FL>
__global__ __launch_bounds__(512) void q4_shared_kernel(Q4View m, const h16_t *__restrict__ x, int64_t ldx, int C, int T, Q4Out out, int per, float *__restrict__ part) {
    constexpr int NF = 4 / FL, R = 2, XL = NB / 2;              // XL: operand pieces a wave fetches per step, of 4 NB
    static_assert(NB % 2 == 0, "pieces divide over the waves");
    __shared__ u32x4 xs[2][4 * NB][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int tile0 = (blockIdx.x * 8 + wave) * UT;
    const int k0 = blockIdx.y * per, k1 = min(k0 + per, m.k_blocks);
    const u32x4 *wp[UT];
    int col[UT];
#pragma unroll
    for (int u = 0; u < UT; ++u) {
        const int t = min(tile0 + u, m.n_tiles - 1);
        wp[u] = static_cast<const u32x4 *>(m.w) + (size_t)t * 64 + lane;
        col[u] = t * 16 + 4 * g;
    }
    const h16_t *xp[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        const int f = wave + 8 * i, b = f % NB, s = f / NB;
        xp[i] = x + (size_t)min(16 * b + j, C - 1) * ldx + s * 32 + 8 * g;
    }
    floatx4 acc[UT][NB];
#pragma unroll
    for (int u = 0; u < UT; ++u)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[u][b] = floatx4{0.f, 0.f, 0.f, 0.f};
    u32x4 wr[R][UT], xg[XL];
    scale_raw<ST> sr[R][UT][NF];
    uint32_t zr[R][UT][NF];
    const size_t kstride = (size_t)m.n_tiles * 64;
    auto request = [&](int i, int kq) {
#pragma unroll
        for (int u = 0; u < UT; ++u) wr[i][u] = __builtin_nontemporal_load(wp[u] + (size_t)kq * kstride);
#pragma unroll
        for (int u = 0; u < UT; ++u) load_scales<ST, NF>(m, kq, col[u], sr[i][u], zr[i][u]);
    };
    auto fetch = [&](int kq) {
#pragma unroll
        for (int i = 0; i < XL; ++i) xg[i] = *reinterpret_cast<const u32x4 *>(xp[i] + kq * 128);
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < XL; ++i) xs[buf][wave + 8 * i][lane] = xg[i];
    };
    fetch(k0);
#pragma unroll
    for (int i = 0; i < R; ++i) request(i, min(k0 + i, k1 - 1));
    put(0);
    fetch(min(k0 + 1, k1 - 1));
    HX_LDS_BARRIER();
    for (int k = k0; k < k1; k += R) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (k + i >= k1) break;                             // uniform over the block
            contract_block<F16, ST, NB, UT, FL>(wr[i], sr[i], zr[i], m.zeros != nullptr, [&](int s, int b) { return xs[i & 1][s * NB + b][lane]; }, acc);
            request(i, min(k + i + R, k1 - 1));
            put((i & 1) ^ 1);                                   // the buffer that every wave left at the last barrier
            fetch(min(k + i + 2, k1 - 1));
            HX_LDS_BARRIER();
        }
    }
    const bool own = part == nullptr;
#pragma unroll
    for (int u = 0; u < UT; ++u) {
        if (tile0 + u >= m.n_tiles) continue;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int c = 16 * b + j, n0 = (tile0 + u) * 16 + 4 * g;
            if (c >= C) continue;
            if (own) store_columns(m, out, c, n0, acc[u][b]);
            else *reinterpret_cast<floatx4 *>(part + ((size_t)blockIdx.y * C + c) * (m.n_tiles * 16) + n0) = acc[u][b];
        }
    }
}

// adds up splits and parts, in that order of loops; a block takes 1024 columns of a row
__global__ __launch_bounds__(256) void q4_finish_kernel(Q4View m, const float *__restrict__ part, int splits, int C, int T, Q4Out out) {
    __shared__ float s_v[4];
    __shared__ int s_i[4];
    const int t = blockIdx.y, n0 = blockIdx.x * 1024 + threadIdx.x * 4, np = m.n_tiles * 16;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    if (n0 < np) {
        for (int c = t; c < C; c += T) {
            floatx4 a = {0.f, 0.f, 0.f, 0.f};
            for (int s = 0; s < splits; ++s) a += *reinterpret_cast<const floatx4 *>(part + ((size_t)s * C + c) * np + n0);
            v += a;
        }
    }
    if (out.best_val == nullptr) {
        if (n0 < np) store_columns(m, out, t, n0, v);
        return;
    }
    float bv = -INFINITY;
    int bi = 0x7fffffff;
    if (n0 < np) take_best(m, n0, v, bv, bi);
    best_of_lanes<64>(bv, bi);
    if ((threadIdx.x & 63) == 0) { s_v[threadIdx.x >> 6] = bv; s_i[threadIdx.x >> 6] = bi; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w)
            if (s_v[w] > bv || (s_v[w] == bv && s_i[w] < bi)) { bv = s_v[w]; bi = s_i[w]; }
        out.best_val[(size_t)t * gridDim.x + blockIdx.x] = bv;
        out.best_id[(size_t)t * gridDim.x + blockIdx.x] = bi;
    }
}

template <int FROM>
__device__ __forceinline__ float load_as(const void *p, size_t at) {
    if constexpr (FROM == HX_T_F32) return static_cast<const float *>(p)[at];
    else if constexpr (FROM == HX_T_BF16) return bf16_f32(static_cast<const h16_t *>(p)[at]);
    else return f16_f32(static_cast<const h16_t *>(p)[at]);
}

// Rows as operand columns: x (+ x2), normalised with the gain g when there is one, as three bf16 parts [3 T][Kp] whose sum is the fp32
// value; zero beyond K.  A block takes a row.  What is not finite has its value in the first part.
template <int FROM>
__global__ __launch_bounds__(1024) void q4_parts_kernel(const void *__restrict__ x, const void *__restrict__ x2, int64_t ldx, const float *__restrict__ g,
                                                        float eps, int K, int Kp, int T, h16_t *__restrict__ out) {
    __shared__ float red[16];
    const int t = blockIdx.x;
    float r = 1.0f;
    auto value = [&](int k) { return load_as<FROM>(x, (size_t)t * ldx + k) + (x2 != nullptr ? load_as<FROM>(x2, (size_t)t * ldx + k) : 0.f); };
    if (g != nullptr) {
        float ss = 0.f;
        for (int k = threadIdx.x; k < K; k += 1024) {
            const float v = value(k);
            ss = fmaf(v, v, ss);
        }
        ss = wave_sum(ss);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
        __syncthreads();
        ss = 0.f;
        for (int w = 0; w < 16; ++w) ss += red[w];
        r = 1.0f / sqrtf(ss / (float)K + eps);
    }
    for (int k = threadIdx.x; k < Kp; k += 1024) {
        float v = 0.f;
        if (k < K) v = g != nullptr ? value(k) * r * g[k] : value(k);
        uint32_t p[3] = {__float_as_uint(v) >> 16, 0u, 0u};      // cut off, not rounded: what is left has the same sign and 16 bits
        if (__builtin_isfinite(v)) {
            const float rest = v - bf16_f32(p[0]);
            p[1] = __float_as_uint(rest) >> 16;
            p[2] = __float_as_uint(rest - bf16_f32(p[1])) >> 16;
        } else if (v != v) {
            p[0] = 0x7fc0u;
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) out[((size_t)i * T + t) * Kp + k] = (h16_t)p[i];
    }
}

// 16-bit rows that are not 16-byte pieces: a dense copy, zero beyond K
__global__ __launch_bounds__(256) void q4_copy_kernel(const h16_t *__restrict__ x, int64_t ldx, int K, int Kp, h16_t *__restrict__ out) {
    for (int k = threadIdx.x; k < Kp; k += 256) out[(size_t)blockIdx.x * Kp + k] = k < K ? x[(size_t)blockIdx.x * ldx + k] : (h16_t)0;
}

// [K][N / 2] bytes, column 2 i in the low nibble of byte i -> the layout above, columns n0 .. n0 + n - 1; a word per thread
__global__ __launch_bounds__(256) void q4_pack_kernel(const uint8_t *__restrict__ src, int64_t ld, int K, int n0, int n, int n_tiles, int k_blocks, uint32_t *__restrict__ dst) {
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (size_t)k_blocks * n_tiles * 256) return;
    const int i = idx & 3, lane = (idx >> 2) & 63, col = (int)((idx >> 8) % n_tiles) * 16 + (lane & 15);
    const int k0 = (int)((idx >> 8) / n_tiles) * 128 + 32 * i + 8 * (lane >> 4);
    uint32_t w = 0;
    if (col < n) {
        const int at = n0 + col;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t q = k0 + e < K ? (src[(size_t)(k0 + e) * ld + (at >> 1)] >> (4 * (at & 1))) & 15u : 0u;
            w |= q << (16 * (e & 1) + 4 * (e >> 1));
        }
    }
    dst[idx] = w;
}
// scales [groups][N] -> [rows][16 n_tiles], zero beyond; zero points [groups][N / 2] nibbles -> bytes
__global__ __launch_bounds__(256) void q4_pack_scales_kernel(const void *__restrict__ src, int es, const uint8_t *__restrict__ zsrc, int64_t ld, int groups, int rows, int n0,
                                                             int n, int np, void *__restrict__ dst, uint8_t *__restrict__ zdst) {
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (size_t)rows * np) return;
    const int row = (int)(idx / np), col = (int)(idx % np);
    const bool there = row < groups && col < n;
    const size_t at = (size_t)row * ld + n0 + col;
    if (es == 4) static_cast<float *>(dst)[idx] = there ? static_cast<const float *>(src)[at] : 0.f;
    else static_cast<h16_t *>(dst)[idx] = there ? static_cast<const h16_t *>(src)[at] : (h16_t)0;
    if (zdst != nullptr) zdst[idx] = there ? (uint8_t)((zsrc[(size_t)row * (ld / 2) + ((n0 + col) >> 1)] >> (4 * ((n0 + col) & 1))) & 15) : (uint8_t)0;
}

// Tiles of 16 columns per wave of the shared form, and splits of its contraction: one round of blocks for the chip.  Two tiles a wave halve the
// operand's way through LDS; with 96 operand columns their sums do not fit the registers.
int shared_tiles(const Q4View &m, int nb) { return m.n_tiles >= 256 * 16 && nb <= 4 ? 2 : 1; }
int shared_splits(const Q4View &m, int tiles) {
    const int blocks = (m.n_tiles + 8 * tiles - 1) / (8 * tiles);
    return std::max(1, std::min({256 / blocks, m.k_blocks / 4, 16}));
}

template <bool F16, int ST, int FL>
void launch_few(const Q4View &m, const h16_t *x, int64_t ldx, int C, int T, const Q4Out &out, hipStream_t s) {
    if (m.n_tiles >= kQ4PairTiles) hipLaunchKernelGGL((q4_few_kernel<F16, ST, 2, FL>), dim3((m.n_tiles + 1) / 2), dim3(512), 0, s, m, x, ldx, C, T, out);
    else hipLaunchKernelGGL((q4_few_kernel<F16, ST, 1, FL>), dim3(m.n_tiles), dim3(512), 0, s, m, x, ldx, C, T, out);
}
template <bool F16, int ST, int NB, int FL>
void launch_shared(const Q4View &m, const h16_t *x, int64_t ldx, int C, int T, const Q4Out &out, float *part, hipStream_t s) {
    const int ut = shared_tiles(m, NB), splits = shared_splits(m, ut), per = (m.k_blocks + splits - 1) / splits, used = (m.k_blocks + per - 1) / per;
    const bool own = used == 1 && C == T && out.best_val == nullptr;
    const dim3 grid((m.n_tiles + 8 * ut - 1) / (8 * ut), used);
    if constexpr (NB <= 4) {
        if (ut == 2) hipLaunchKernelGGL((q4_shared_kernel<F16, ST, NB, 2, FL>), grid, dim3(512), 0, s, m, x, ldx, C, T, out, per, own ? nullptr : part);
    }
    if (ut == 1) hipLaunchKernelGGL((q4_shared_kernel<F16, ST, NB, 1, FL>), grid, dim3(512), 0, s, m, x, ldx, C, T, out, per, own ? nullptr : part);
    if (!own) hipLaunchKernelGGL(q4_finish_kernel, dim3((m.n_tiles * 16 + 1023) / 1024, T), dim3(256), 0, s, m, part, used, C, T, out);
}
template <bool F16, int ST, int FL>
void launch_cols(const Q4View &m, const h16_t *x, int64_t ldx, int C, int T, const Q4Out &out, float *part, hipStream_t s) {
    if (C <= 16) launch_few<F16, ST, FL>(m, x, ldx, C, T, out, s);
    else if (C <= 32) launch_shared<F16, ST, 2, FL>(m, x, ldx, C, T, out, part, s);
    else if (C <= 64) launch_shared<F16, ST, 4, FL>(m, x, ldx, C, T, out, part, s);
    else launch_shared<F16, ST, 6, FL>(m, x, ldx, C, T, out, part, s);
}
template <bool F16, int ST>
void launch_type(const Q4View &m, const h16_t *x, int64_t ldx, int C, int T, const Q4Out &out, float *part, hipStream_t s) {
    if (m.group >= 128) launch_cols<F16, ST, 4>(m, x, ldx, C, T, out, part, s);
    else if (m.group == 64) launch_cols<F16, ST, 2>(m, x, ldx, C, T, out, part, s);
    else launch_cols<F16, ST, 1>(m, x, ldx, C, T, out, part, s);
}

}  // namespace

size_t q4_part_floats(const Q4View &m) { return (size_t)std::max(shared_splits(m, 1), shared_splits(m, 2)) * 3 * kQ4PartRows * m.n_tiles * 16; }
int q4_best_units(const Q4View &m, int T) {
    if (3 * T > 16) return (m.n_tiles * 16 + 1023) / 1024;
    return m.n_tiles >= kQ4PairTiles ? (m.n_tiles + 1) / 2 : m.n_tiles;
}
void launch_q4(const Q4View &m, bool parts, const h16_t *x, int64_t ldx, int T, const Q4Out &out, float *part, hipStream_t s) {
    const int C = parts ? 3 * T : T;
    if (m.type == HX_T_F32) launch_type<false, HX_T_F32>(m, x, ldx, C, T, out, part, s);
    else if (m.type == HX_T_BF16) launch_type<false, HX_T_BF16>(m, x, ldx, C, T, out, part, s);
    else if (parts) launch_type<false, HX_T_F16>(m, x, ldx, C, T, out, part, s);
    else launch_type<true, HX_T_F16>(m, x, ldx, C, T, out, part, s);
}
void launch_q4_parts(int type, const void *x, const void *x2, int64_t ldx, const float *g, float eps, int K, int Kp, int T, h16_t *out, hipStream_t s) {
    if (type == HX_T_F32) hipLaunchKernelGGL(q4_parts_kernel<HX_T_F32>, dim3(T), dim3(1024), 0, s, x, x2, ldx, g, eps, K, Kp, T, out);
    else if (type == HX_T_BF16) hipLaunchKernelGGL(q4_parts_kernel<HX_T_BF16>, dim3(T), dim3(1024), 0, s, x, x2, ldx, g, eps, K, Kp, T, out);
    else hipLaunchKernelGGL(q4_parts_kernel<HX_T_F16>, dim3(T), dim3(1024), 0, s, x, x2, ldx, g, eps, K, Kp, T, out);
}
void launch_q4_copy(const h16_t *x, int64_t ldx, int K, int Kp, int T, h16_t *out, hipStream_t s) {
    hipLaunchKernelGGL(q4_copy_kernel, dim3(T), dim3(256), 0, s, x, ldx, K, Kp, out);
}
void launch_q4_pack(const Q4View &m, const uint8_t *w4, const void *scales, const uint8_t *zeros, int64_t ld, int K, int n0, hipStream_t s) {
    const size_t words = (size_t)m.k_blocks * m.n_tiles * 256, cells = (size_t)m.scale_rows * m.n_tiles * 16;
    hipLaunchKernelGGL(q4_pack_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, s, w4, ld / 2, K, n0, m.n_valid, m.n_tiles, m.k_blocks, const_cast<uint32_t *>(static_cast<const uint32_t *>(m.w)));
    hipLaunchKernelGGL(q4_pack_scales_kernel, dim3((unsigned)((cells + 255) / 256)), dim3(256), 0, s, scales, m.type == HX_T_F32 ? 4 : 2, zeros, ld, (K + m.group - 1) / m.group,
                       m.scale_rows, n0, m.n_valid, m.n_tiles * 16, const_cast<void *>(m.scales), const_cast<uint8_t *>(m.zeros));
}
