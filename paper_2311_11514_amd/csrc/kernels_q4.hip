// Products of a few rows with a matrix of 4-bit weights that carry a scale, and possibly a zero point, per group of input features:
//   y[t][n] = sum over groups g of s[g][n] * sum over k in g of (q[k][n] - z[g][n]) * x[t][k],   q, z = 0 .. 15.
//
// The matrix instructions take the weights as q - z, exactly: a nibble in the mantissa bits of 16 (256) is 16 + q (256 + q), from which one packed
// subtraction takes 16 + z (256 + z).  Products with 11-bit numbers are exact in fp32, so that a group's sum is off by its own roundings alone, in
// relation to |q - z| |x|.  (Sums over 16 + q with the offset taken off behind them need no subtraction, but then a large x whose weight is its zero
// point drowns the rest of its group.)
// The operand is fp16, or bf16 where a small matrix meets few of them and the weights can be converted once more.  Other bf16 rows and fp32 rows are
// scaled to fp16, x 2^e with e such that the row's largest value fits the type, and the results scaled
// back: no sum over a group passes fp32's range on the way.  A bf16 row takes one column of the operand (exact down to 2^-29 of the row's
// largest value, and to 2^-40 of that below); an fp32 row two, x 2^e = hi + lo (22 bits of a value, 2^-39 of the row's largest), whose products are
// added up per part and joined at the end.
//
// Layout: blocks of 16 columns x 128 input features, 1 KB, [k / 128][n / 16][lane][4 words]: word i of lane l holds features
// 128 kq + 32 i + 8 (l / 16) + 0 .. 7 of column 16 tile + l % 16, what one lane of v_mfma_f32_16x16x32 contributes to four steps, in one
// 16-byte request.  Feature 2 p + h sits in bits 16 h + 4 p (p = 3: 16 (1 - h) + 12) of the word turned left by 6: pairs 0 and 3 are where fp16 has
// them under the exponents of 16 and 256, pairs 2 and 1 after one turn by 8.
// Scales have a row for every group, or for every 128 features where groups are larger; zero points are bytes, or one row of 8s.
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
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

template <bool BF>
__device__ __forceinline__ floatx4 mfma(u32x4 a, u32x4 b, floatx4 c) {
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// Eight nibbles -> eight times q - z, as fp16, or, through fp32, as bf16 (BF; 21 operations instead of 9).  The constants are kept in registers out of the compiler's sight: an and-or takes no literals on this
// processor, and with constants that it knows the compiler makes two operations of it.
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
struct Zero { uint32_t of16, of256; };                          // -(16 + z) and -(256 + z), twice each
struct Widen {
    uint32_t mask16, mask256, is16, is256;
    __device__ __forceinline__ static Widen make() {
        Widen w;
        asm("s_mov_b32 %0, %1" : "=s"(w.mask16) : "i"(0x03c003c0));
        asm("s_mov_b32 %0, %1" : "=s"(w.mask256) : "i"(0x003c003c));
        asm("v_mov_b32 %0, %1" : "=v"(w.is16) : "i"(0x4c004c00));
        asm("v_mov_b32 %0, %1" : "=v"(w.is256) : "i"(0x5c005c00));
        return w;
    }
    __device__ __forceinline__ static Zero zero(uint32_t z) { return Zero{0xcc00cc00u + __umul24(z, 0x400040u), 0xdc00dc00u + __umul24(z, 0x40004u)}; }
    __device__ __forceinline__ static uint32_t add(uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, a) + __builtin_bit_cast(f16x2, b));
    }
    template <bool BF>
    __device__ __forceinline__ u32x4 operator()(uint32_t w, const Zero &z) const {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
        const uint32_t r = __builtin_amdgcn_alignbit(w, w, 8);
        u32x4 v = {add((w & mask16) | is16, z.of16), add((r & mask256) | is256, z.of256), add((r & mask16) | is16, z.of16), add((w & mask256) | is256, z.of256)};
        if constexpr (BF) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(__builtin_convertvector(__builtin_bit_cast(f16x2, (uint32_t)v[i]), f32x2), b16x2));
        }
        return v;
    }
};

// four neighbouring columns' scales, as they are loaded and as fp32
template <int ST> using scale_raw = std::conditional_t<ST == HX_T_F32, floatx4, uint2>;
template <int ST>
__device__ __forceinline__ floatx4 scale4(const scale_raw<ST> &v) {
    if constexpr (ST == HX_T_F32) return v;
    else if constexpr (ST == HX_T_BF16) return floatx4{bf16_f32(v.x & 0xffffu), bf16_f32(v.x >> 16), bf16_f32(v.y & 0xffffu), bf16_f32(v.y >> 16)};
    else return floatx4{f16_f32(v.x & 0xffffu), f16_f32(v.x >> 16), f16_f32(v.y & 0xffffu), f16_f32(v.y >> 16)};
}

// acc += a 128-feature block's share: UT weight tiles against NB operand tiles, x(step, tile) the operand of 32 features
template <int ST, int NB, int UT, int FL, bool BF, typename XF>
__device__ __forceinline__ void contract_block(const Widen &widen, const u32x4 (&w)[UT], const scale_raw<ST> (&s)[UT][4 / FL], const uint32_t (&z)[UT][4 / FL], XF x,
                                               floatx4 (&acc)[UT][NB]) {
#pragma unroll
    for (int f = 0; f < 4 / FL; ++f) {
        floatx4 S[UT][NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int u = 0; u < UT; ++u) S[u][b] = floatx4{0.f, 0.f, 0.f, 0.f};
        Zero zero[UT];
#pragma unroll
        for (int u = 0; u < UT; ++u) zero[u] = Widen::zero(z[u][f]);
#pragma unroll
        for (int st = f * FL; st < f * FL + FL; ++st) {
            u32x4 a[UT];
#pragma unroll
            for (int u = 0; u < UT; ++u) a[u] = widen.template operator()<BF>(w[u][st], zero[u]);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const u32x4 xb = x(st, b);
#pragma unroll
                for (int u = 0; u < UT; ++u) S[u][b] = mfma<BF>(a[u], xb, S[u][b]);
            }
            if (UT > 1 && NB == 1) __builtin_amdgcn_sched_barrier(0);      // one step's weights at a time: more of them do not fit the registers
        }
        floatx4 s4[UT];
#pragma unroll
        for (int u = 0; u < UT; ++u) s4[u] = scale4<ST>(s[u][f]);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int u = 0; u < UT; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[u][b][r] = fmaf(s4[u][r], S[u][b][r], acc[u][b][r]);
        if (FL < 4) {                                           // one group's sums at a time: side by side they do not fit the registers
#pragma unroll
            for (int u = 0; u < UT; ++u)
#pragma unroll
                for (int b = 0; b < NB; ++b) asm volatile("" : "+v"(acc[u][b]));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}
// the scales of a 128-feature block for four columns from `col` on, what the lane has of the result, and the zero points of column `zcol`, of whose
// weights it holds a part
template <int ST, int NF>
__device__ __forceinline__ void load_scales(const Q4View &m, int kq, uint32_t col, uint32_t zcol, scale_raw<ST> (&s)[NF], uint32_t (&z)[NF]) {
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        const size_t row = kq * NF + f;                         // the same in every lane
        s[f] = *reinterpret_cast<const scale_raw<ST> *>(static_cast<const unsigned char *>(m.scales) + row * (m.n_tiles * 16) * (ST == HX_T_F32 ? 4 : 2) + col * (ST == HX_T_F32 ? 4u : 2u));
        z[f] = m.zeros[row * m.zeros_row + zcol];
    }
}
__device__ __forceinline__ u32x4 load_weights(const Q4View &m, int kq, uint32_t off) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(static_cast<const unsigned char *>(m.w) + (size_t)kq * m.n_tiles * 1024 + off));
}
__device__ __forceinline__ void store_pair(const Q4Out &out, size_t at, float a, float b) {
    if (out.type == HX_T_F32) *reinterpret_cast<float2 *>(static_cast<float *>(out.y) + at) = float2{a, b};
    else if (out.type == HX_T_BF16) *reinterpret_cast<uint32_t *>(static_cast<h16_t *>(out.y) + at) = to_bf16(a) | (uint32_t)to_bf16(b) << 16;
    else *reinterpret_cast<uint32_t *>(static_cast<h16_t *>(out.y) + at) = to_f16(a) | (uint32_t)to_f16(b) << 16;
}
// the power of two that a row whose largest magnitude is mx is scaled with: to [2^14, 2^15); a row of zeros or with an infinity as it is
__device__ __forceinline__ int row_power(float mx) {
    int e = 15;
    if (mx > 0.f && mx < INFINITY) (void)frexpf(mx, &e);
    return 15 - e;
}
// The result of a row: sums that are not finite (the row holds an infinity or a NaN) become NaN, and the power of two that the row was scaled with
// is taken off.
__device__ __forceinline__ void settle(int e, floatx4 &v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = __builtin_isfinite(v[r]) ? ldexpf(v[r], -e) : NAN;
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

// Few operand columns (rows times parts), or a small matrix: a block takes up to 16 of them, whole rows (blockIdx.y; columns that are not there repeat
// the last one and are not stored).  A block of W waves owns UT tiles of 16 columns over the whole contraction; its waves take the 128-feature
// blocks in turn and are summed through LDS in wave order, so that no partial result leaves the block.  A wave holds R blocks with their scales in registers, requested that far ahead; every request is
// unconditional (past the end it repeats the last block's), so that the compiler can count what is in flight and waits for the oldest
// alone.  XLDS: the operand is staged in LDS once, else a wave requests its pieces one block ahead, from L2.
// Bound by HBM on wide matrices, on small ones by the launch and one round trip (bf16, one row: 8192 x 10240 13.9 us, 3.1 TB/s; the arg-max form, 8192 x
// 32000, two columns 28.4, 4.7 TB/s; 4096 x 4096 6.1).
// FL: 32-feature steps of a scale's group inside a 128-feature block (4: groups of 128 and more).
// OP_BF16: the operand is bf16 as it is.  Its sums, which have not seen their scale yet, may leave fp32's range (from values of 1.8e35 on): columns whose
// result is not finite are done once more, with the operand 2^-64 of itself.  OP_SCALED (with XLDS): the operand is bf16 and becomes fp16 on its way to LDS.
// The first costs 48 operations for every weight tile's block, the second a round trip and two barriers a launch, a launch in front of this one 2.7 us
// (us, one row: 2048 x 1024 4.3 / 4.6 / 7.0, 4096 x 4096 6.8 / 6.2 / 8.2, 8192 x 10240 17.2 / 13.9 / 16.4; four rows of 4096 x 4096 6.9 / 8.5 / 9.0).
enum { OP_F16, OP_BF16, OP_SCALED };
constexpr int kScaled = 32 * 1024;                              // bytes of an operand that is scaled so: 8 pieces for each of 256 threads
__device__ __forceinline__ uint32_t max_of_16_lanes(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));       // the lanes turned by 1, 2, 4 and 8
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));
}
template <int ST, int UT, int FL, int W, int R, bool XLDS, int OP>
__global__ __launch_bounds__(64 * W, UT == 1 || FL == 4 ? 4 : FL == 2 ? 3 : 2) void q4_few_kernel(Q4View m, const h16_t *__restrict__ x, int64_t ldx, int parts, int rows, Q4Out out) {
    constexpr int NF = 4 / FL;
    const int t0 = blockIdx.y * (16 / parts), T = min(16 / parts, rows - t0), C = parts * T;
    auto operand = [&](int c) { return x + (size_t)(c / T * rows + t0 + c % T) * ldx; };
    static_assert(R % 2 == 0, "the operand's two slots alternate");
    constexpr bool BF = OP == OP_BF16;
    static_assert(OP != OP_SCALED || (XLDS && 8 * 64 * W * 16 >= kScaled), "rows are scaled on their way to LDS, all at once");
    __shared__ floatx4 red[W][UT][64];
    __shared__ uint32_t s_most[16];                             // OP_SCALED: bits of a column's largest magnitude, and its power of two
    __shared__ int s_power[16];
    extern __shared__ __align__(16) u32x4 xs[];                 // XLDS: [k / 8][column]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
    const int tile0 = blockIdx.x * UT;
    uint32_t off[UT], col[UT], zcol[UT];
#pragma unroll
    for (int u = 0; u < UT; ++u) {
        const uint32_t t = min(tile0 + u, m.n_tiles - 1);      // a last tile of its own: the block's second repeats it, not stored
        off[u] = t * 1024u + lane * 16u;
        col[u] = t * 16u + 4u * g;
        zcol[u] = t * 16u + j;
    }
    const h16_t *xp = operand(min(j, C - 1)) + 8 * g;
    const Widen widen = Widen::make();
    floatx4 acc[UT][1];
#pragma unroll
    for (int u = 0; u < UT; ++u) acc[u][0] = floatx4{0.f, 0.f, 0.f, 0.f};
    u32x4 wr[R][UT], xr[XLDS ? 1 : 2][4];
    scale_raw<ST> sr[R][UT][NF];
    uint32_t zr[R][UT][NF];
    auto request = [&](int i, int kq) {
#pragma unroll
        for (int u = 0; u < UT; ++u) wr[i][u] = load_weights(m, kq, off[u]);
#pragma unroll
        for (int u = 0; u < UT; ++u) load_scales<ST, NF>(m, kq, col[u], zcol[u], sr[i][u], zr[i][u]);
    };
    auto fetch = [&](int i, int kq) {
#pragma unroll
        for (int s = 0; s < 4; ++s) xr[i][s] = *reinterpret_cast<const u32x4 *>(xp + kq * 128 + s * 32);
    };
    // OP_SCALED: a thread's pieces of the operand, every 64 W-th, so that 16 lanes have neighbours of one column; requested in front of the weights
    u32x4 raw[OP == OP_SCALED ? 8 : 1];
    int raw_col[OP == OP_SCALED ? 8 : 1], raw_piece[OP == OP_SCALED ? 8 : 1], mine_of_operand = 0;
    if constexpr (OP == OP_SCALED) {
        const int pieces = m.k_blocks * 16, step_c = 64 * W / pieces, step_p = 64 * W % pieces;
        mine_of_operand = (C * pieces + 64 * W - 1) / (64 * W);
        int c = threadIdx.x / pieces, p = threadIdx.x - c * pieces;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= mine_of_operand) break;
            raw_col[i] = c;                                     // C and more: past the end
            raw_piece[i] = p;
            raw[i] = *reinterpret_cast<const u32x4 *>(operand(min(c, C - 1)) + 8 * p);
            c += step_c;
            p += step_p;
            if (p >= pieces) { p -= pieces; ++c; }
        }
    }
    // ring slot i holds block wave + i W of the round
    const int last = m.k_blocks - 1, mine = (last - wave + W) / W, full = mine / R;
#pragma unroll
    for (int i = 0; i < R; ++i) request(i, min(wave + i * W, last));
    if constexpr (XLDS) {
        const int pieces = m.k_blocks * 16;
        if constexpr (OP == OP_SCALED) {
            if (threadIdx.x < 16) s_most[threadIdx.x] = 0;
            HX_LDS_BARRIER();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= mine_of_operand) break;
                uint32_t most = 0;
#pragma unroll
                for (int x = 0; x < 4; ++x) most = max(most, max(raw[i][x] & 0x7fffu, (raw[i][x] >> 16) & 0x7fffu));
                most = max_of_16_lanes(most);
                if ((lane & 15) == 0 && raw_col[i] < C) atomicMax(&s_most[raw_col[i]], most);
            }
            HX_LDS_BARRIER();
            if ((int)threadIdx.x < C) s_power[threadIdx.x] = row_power(bf16_f32(s_most[threadIdx.x]));
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= mine_of_operand || raw_col[i] >= C) break;
                const int e = row_power(bf16_f32(s_most[raw_col[i]]));
                u32x4 h;
#pragma unroll
                for (int x = 0; x < 4; ++x) h[x] = to_f16(ldexpf(bf16_f32(raw[i][x] & 0xffffu), e)) | (uint32_t)to_f16(ldexpf(bf16_f32(raw[i][x] >> 16), e)) << 16;
                xs[raw_piece[i] * C + raw_col[i]] = h;
            }
        } else {
            for (int c = 0; c < C; ++c)
                for (int p = threadIdx.x; p < pieces; p += 64 * W) xs[p * C + c] = *reinterpret_cast<const u32x4 *>(operand(c) + 8 * p);
        }
        HX_LDS_BARRIER();
    } else {
        fetch(0, min(wave, last));
        fetch(1, min(wave + W, last));
    }
    const u32x4 *xl = xs + g * C + min(j, C - 1);
    auto contract = [&](int i, int kq) {
        contract_block<ST, 1, UT, FL, BF>(widen, wr[i], sr[i], zr[i], [&](int s, int) { return XLDS ? xl[(kq * 4 + s) * 4 * C] : xr[XLDS ? 0 : i & 1][s]; }, acc);
    };
    int kq = wave;
    for (int rd = 0; rd < full; ++rd) {
#pragma unroll
        for (int i = 0; i < R; ++i, kq += W) {
            contract(i, kq);
            request(i, min(kq + R * W, last));
            if constexpr (!XLDS) fetch(i & 1, min(kq + 2 * W, last));
            __builtin_amdgcn_sched_barrier(0);                  // each refill right behind its slot's use
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (i < mine - full * R) {                              // uniform over the wave
            contract(i, kq + i * W);
            if constexpr (!XLDS) fetch(i & 1, min(kq + (i + 2) * W, last));
        }
    }
    if constexpr (BF) {
        bool odd = false;
#pragma unroll
        for (int u = 0; u < UT; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) odd = odd || !__builtin_isfinite(acc[u][0][r]);
        unsigned long long any = __builtin_amdgcn_ballot_w64(odd);
        if (any != 0) {
            any |= any >> 32;
            const bool mine_odd = ((any | any >> 16) >> j) & 1;        // this lane's column
            floatx4 again[UT][1];
#pragma unroll
            for (int u = 0; u < UT; ++u) again[u][0] = floatx4{0.f, 0.f, 0.f, 0.f};
            for (int k = wave; k <= last; k += W) {
                request(0, k);
                u32x4 xs64[4];
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const u32x4 v = XLDS ? xl[(k * 4 + s) * 4 * C] : *reinterpret_cast<const u32x4 *>(xp + k * 128 + s * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        xs64[s][i] = to_bf16(bf16_f32(v[i] & 0xffffu) * 0x1p-64f) | (uint32_t)to_bf16(bf16_f32(v[i] >> 16) * 0x1p-64f) << 16;
                }
                contract_block<ST, 1, UT, FL, BF>(widen, wr[0], sr[0], zr[0], [&](int s, int) { return xs64[s]; }, again);
            }
#pragma unroll
            for (int u = 0; u < UT; ++u)
                if (mine_odd) acc[u][0] = again[u][0] * 0x1p64f;
        }
    }
#pragma unroll
    for (int u = 0; u < UT; ++u) red[wave][u][lane] = acc[u][0];
    __syncthreads();
    // four columns of one row per thread: waves in order, parts in order
    const int idx = threadIdx.x;
    if (idx >= T * UT * 4) return;
    const int t = idx / (UT * 4), u = (idx >> 2) % UT, gg = idx & 3;
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) {
        floatx4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) a += red[w][u][p * T + t + 16 * gg];
        v += a;
    }
    const int n0 = (tile0 + u) * 16 + 4 * gg;
    settle(OP == OP_SCALED ? s_power[t] : out.exps == nullptr ? 0 : out.exps[t0 + t], v);
    if (out.best_val == nullptr) {
        store_columns(m, out, t0 + t, n0, v);
        return;
    }
    float bv = -INFINITY;
    int bi = 0x7fffffff;
    take_best(m, n0, v, bv, bi);
    best_of_lanes<UT * 4>(bv, bi);                              // the row's UT * 4 threads are neighbours
    if (idx % (UT * 4) == 0) {
        out.best_val[(size_t)(t0 + t) * gridDim.x + blockIdx.x] = bv;
        out.best_id[(size_t)(t0 + t) * gridDim.x + blockIdx.x] = bi;
    }
}

// More operand columns: the operand outweighs the weights that a tile of 16 columns has, so the waves of a block share it through LDS.  Two groups
// of six to eight waves take the 128-feature blocks in turn; a wave owns two neighbouring tiles, and its group's operand, weights, scales and zero points
// go to LDS without passing registers, up to S - 1 steps ahead, one barrier a step: sixteen waves with few registers, of which some widen and scale
// while others are at the matrix unit.  The groups are joined through LDS at the end.  The contraction is split over blockIdx.y where the matrix
// has too few columns for the chip: splits leave partial sums, `part` [split][column of the operand][16 n_tiles], to q4_finish_kernel.  Without
// splits the parts are joined, and stored or searched for their largest, here.
// Bound by HBM up to 16 columns (8192 x 57344, twelve rows 46 us, 5.2 TB/s), beyond by the vector unit (36 operations a lane to widen a tile's block, some
// 8 for its scales and zero points, 4 per operand tile to apply them) and the matrix unit, which overlap little: 32 columns 57 us, 4096 x 50304
// with 48 columns 42.
template <int ST, int NB, int FL> struct SharedStage {
    static constexpr int ES = ST == HX_T_F32 ? 4 : 2, NF = 4 / FL, SP = (NF * 256 * ES + 1023) / 1024;      // SP: requests of 1 KB for the scales of 16 tiles
    u32x4 x[4 * NB][64], w[16][64];
    unsigned char s[SP * 1024], z[1024];
};
template <int ST, int NB, int FL>
__global__ __launch_bounds__(1024, 4) void q4_shared_kernel(Q4View m, const h16_t *__restrict__ x, uint32_t ldx, int C, int T, Q4Out out, int per, float *__restrict__ part) {
    typedef SharedStage<ST, NB, FL> Stage;
    constexpr int NF = Stage::NF, ES = Stage::ES, SP = Stage::SP, UT = 2, XL = (4 * NB + 5) / 6;            // XL: operand pieces a wave fetches (the last ones more than once)
    constexpr int S = 3 * 2 * sizeof(Stage) <= 159 * 1024 ? 3 : 2, L = UT + XL + 1;     // L: requests of a wave per step
    constexpr int YS = 260;
    static_assert((S - 2) * L < 64 && 16 * NB * YS * 4 <= 2 * S * sizeof(Stage), "waits, and the results in the stages' place");
    __shared__ __align__(16) Stage st[2][S];
    const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4, waves = blockDim.x >> 7;
    const int nth = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = nth >= waves ? 1 : 0, wave = nth - grp * waves;
    const int first = blockIdx.x * waves * UT, np = m.n_tiles * 16;
    const int k0 = blockIdx.y * per, k1 = min(k0 + per, m.k_blocks);
    // what this wave requests: its tiles (one past the last repeats that and is not stored), its pieces of the operand, a part of the scales or the zeros
    uint32_t woff[UT], xoff[XL], xat[XL];
#pragma unroll
    for (int u = 0; u < UT; ++u) woff[u] = min(first + wave * UT + u, m.n_tiles - 1) * 1024u + lane * 16u;
#pragma unroll
    for (int i = 0; i < XL; ++i) {
        xat[i] = min(wave + waves * i, 4 * NB - 1);
        xoff[i] = (min(16 * (int)(xat[i] % NB) + j, C - 1) * ldx + (xat[i] / NB) * 32 + 8 * g) * 2;
    }
    const int sp = min(wave, SP);
    const unsigned char *sbase = sp < SP ? static_cast<const unsigned char *>(m.scales) : m.zeros;
    const uint32_t srow = sp < SP ? np * ES : m.zeros_row;
    const int sf = sp < SP ? (sp * 1024 + lane * 16) / (256 * ES) : lane >> 4, scol = sp < SP ? (sp * 1024 + lane * 16) % (256 * ES) / ES : 16 * (lane & 15);
    const uint32_t soff = min(sf, NF - 1) * srow + (sp < SP ? min(first * 16 + scol, np - 16 / ES) * ES : min(first * 16 + scol, np - 16));
    const unsigned lds = hx_lds_addr(&st[grp][0]);
    auto issue = [&](int k, int b) {
        const int kq = min(k, k1 - 1);
        const unsigned at = lds + b * sizeof(Stage);
        const unsigned char *wk = static_cast<const unsigned char *>(m.w) + (size_t)kq * m.n_tiles * 1024;
#pragma unroll
        for (int u = 0; u < UT; ++u) hx_load_lds16(at + offsetof(Stage, w) + (wave * UT + u) * 1024, woff[u], wk);
#pragma unroll
        for (int i = 0; i < XL; ++i) hx_load_lds16(at + xat[i] * 1024, xoff[i], x + kq * 128);
        hx_load_lds16(at + offsetof(Stage, s) + sp * 1024, soff, sbase + (size_t)kq * NF * srow);
    };
    const Widen widen = Widen::make();
    floatx4 acc[UT][NB];
#pragma unroll
    for (int u = 0; u < UT; ++u)
#pragma unroll
        for (int b = 0; b < NB; ++b) acc[u][b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < S - 1; ++i) issue(k0 + grp + 2 * i, i);
    int b0 = 0, bl = S - 1;                                     // buffers of this step and of the one that is S - 1 steps ahead
    for (int k = k0 + grp; k - grp < k1; k += 2) {
        HX_WAIT_VM((S - 2) * L);                                // this step's share of this wave; behind the barrier everybody's
        HX_LDS_BARRIER();
        issue(k + 2 * (S - 1), bl);                             // (everybody has left that buffer)
        bl = b0;
        const Stage &cur = st[grp][b0];
        b0 = b0 + 1 == S ? 0 : b0 + 1;
        if (k >= k1) break;                                     // the second group, after an odd number of steps
        u32x4 w[UT];
        scale_raw<ST> sc[UT][NF];
        uint32_t zc[UT][NF];
#pragma unroll
        for (int u = 0; u < UT; ++u) {
            const int tile = wave * UT + u;
            w[u] = cur.w[tile][lane];
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                sc[u][f] = *reinterpret_cast<const scale_raw<ST> *>(cur.s + (f * 256 + tile * 16 + 4 * g) * ES);
                zc[u][f] = cur.z[f * 256 + tile * 16 + j];
            }
        }
        contract_block<ST, NB, UT, FL, false>(widen, w, sc, zc, [&](int i, int b) { return cur.x[i * NB + b][lane]; }, acc);
    }
    HX_WAIT_VM(0);                                              // nothing is on its way into the stages any more
    HX_LDS_BARRIER();
    float *ys = reinterpret_cast<float *>(&st[0][0]);
    if (grp == 1) {
#pragma unroll
        for (int u = 0; u < UT; ++u)
#pragma unroll
            for (int b = 0; b < NB; ++b) *reinterpret_cast<floatx4 *>(ys + (16 * b + j) * YS + (wave * UT + u) * 16 + 4 * g) = acc[u][b];
    }
    HX_LDS_BARRIER();
    if (grp == 0) {
#pragma unroll
        for (int u = 0; u < UT; ++u) {
            const int tile = first + wave * UT + u;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int c = 16 * b + j;
                floatx4 *at = reinterpret_cast<floatx4 *>(ys + c * YS + (wave * UT + u) * 16 + 4 * g);
                const floatx4 v = acc[u][b] + *at;
                if (part == nullptr) *at = v;
                else if (c < C && tile < m.n_tiles) *reinterpret_cast<floatx4 *>(part + ((size_t)blockIdx.y * C + c) * np + tile * 16 + 4 * g) = v;
            }
        }
    }
    if (part != nullptr) return;
    HX_LDS_BARRIER();
    // parts in order, a wave per row, four columns per lane
    const int n0 = first * 16 + 4 * lane;
    const bool there = lane < waves * UT * 4 && n0 < np;
    for (int t = nth; t < T; t += 2 * waves) {
        floatx4 v = *reinterpret_cast<const floatx4 *>(ys + t * YS + 4 * lane);
        for (int c = t + T; c < C; c += T) v += *reinterpret_cast<const floatx4 *>(ys + c * YS + 4 * lane);
        settle(out.exps == nullptr ? 0 : out.exps[t], v);
        if (out.best_val == nullptr) {
            if (there) store_columns(m, out, t, n0, v);
            continue;
        }
        float bv = -INFINITY;
        int bi = 0x7fffffff;
        if (there) take_best(m, n0, v, bv, bi);
        best_of_lanes<64>(bv, bi);
        if (lane == 0) {
            out.best_val[(size_t)t * gridDim.x + blockIdx.x] = bv;
            out.best_id[(size_t)t * gridDim.x + blockIdx.x] = bi;
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
    settle(out.exps == nullptr ? 0 : out.exps[t], v);
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

// Rows as operand columns: x (+ x2), normalised with the gain g when there is one, times 2^exps[t] as one fp16 number [T][Kp], or as two [2 T][Kp] whose
// sum is that value; zero beyond K.  A block takes a row, a thread eight neighbouring values at a time, of which the first KEEP stay in registers for the
// second pass.  V: 16-byte pieces.  A value that is not finite stays so in the first part.
template <int FROM, bool V, int PARTS>
__global__ __launch_bounds__(1024) void q4_parts_kernel(const void *__restrict__ x, const void *__restrict__ x2, int64_t ldx, const float *__restrict__ g,
                                                        float eps, int K, int Kp, int T, h16_t *__restrict__ out, int32_t *__restrict__ exps) {
    constexpr int KEEP = 4;
    __shared__ float red[16], red2[16];
    const int t = blockIdx.x;
    struct Eight { float v[8]; };
    auto raw = [&](const void *p, int k) {
        Eight r;
        if constexpr (!V) {
#pragma unroll
            for (int i = 0; i < 8; ++i) r.v[i] = k + i < K ? load_as<FROM>(p, (size_t)t * ldx + k + i) : 0.f;
        } else if constexpr (FROM == HX_T_F32) {
            const float *q = static_cast<const float *>(p) + (size_t)t * ldx + k;
            const floatx4 a = *reinterpret_cast<const floatx4 *>(q), b = *reinterpret_cast<const floatx4 *>(q + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { r.v[i] = a[i]; r.v[4 + i] = b[i]; }
        } else {
            const u32x4 a = *reinterpret_cast<const u32x4 *>(static_cast<const h16_t *>(p) + (size_t)t * ldx + k);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t h = (a[i >> 1] >> (16 * (i & 1))) & 0xffffu;
                r.v[i] = FROM == HX_T_BF16 ? bf16_f32(h) : f16_f32(h);
            }
        }
        return r;
    };
    // eight values from k on, times the gain; their squares without it
    auto eight = [&](int k, float &ss) {
        Eight r = raw(x, k);
        if (x2 != nullptr) {
            const Eight y = raw(x2, k);
#pragma unroll
            for (int i = 0; i < 8; ++i) r.v[i] += y.v[i];
        }
        if (g != nullptr) {
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(r.v[i], r.v[i], ss);
#pragma unroll
            for (int i = 0; i < 8; ++i) r.v[i] *= V || k + i < K ? g[k + i] : 0.f;
        }
        return r;
    };
    Eight kept[KEEP];
    float ss = 0.f, mx = 0.f;
#pragma unroll
    for (int c = 0; c < KEEP; ++c) {
        const int k = (c * 1024 + threadIdx.x) * 8;
        if (k < K) {
            kept[c] = eight(k, ss);
#pragma unroll
            for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(kept[c].v[i]));
        }
    }
    for (int k = (KEEP * 1024 + threadIdx.x) * 8; k < K; k += 8192) {
        const Eight r = eight(k, ss);
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(r.v[i]));
    }
    ss = wave_sum(ss);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
    if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = ss; red2[threadIdx.x >> 6] = mx; }
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) { ss += red[w]; mx = fmaxf(mx, red2[w]); }
    const float r = g != nullptr ? 1.0f / sqrtf(ss / (float)K + eps) : 1.0f;
    const int e = row_power(mx * r);
    if (threadIdx.x == 0) exps[t] = e;
    auto put = [&](int k, const Eight &v) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = ldexpf(v.v[i] * r, e);
            const uint32_t h = to_f16(y), l = __builtin_isfinite(y) ? to_f16(y - f16_f32(h)) : 0u;
            if (i & 1) { hi[i >> 1] |= h << 16; lo[i >> 1] |= l << 16; }
            else { hi[i >> 1] = h; lo[i >> 1] = l; }
        }
        *reinterpret_cast<u32x4 *>(out + (size_t)t * Kp + k) = u32x4{hi[0], hi[1], hi[2], hi[3]};
        if constexpr (PARTS == 2) *reinterpret_cast<u32x4 *>(out + (size_t)(T + t) * Kp + k) = u32x4{lo[0], lo[1], lo[2], lo[3]};
    };
    const Eight none = {};
    float unused = 0.f;
#pragma unroll
    for (int c = 0; c < KEEP; ++c) {
        const int k = (c * 1024 + threadIdx.x) * 8;
        if (k < Kp) put(k, k < K ? kept[c] : none);
    }
    for (int k = (KEEP * 1024 + threadIdx.x) * 8; k < Kp; k += 8192) put(k, k < K ? eight(k, unused) : none);
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
            w |= q << (16 * ((e & 1) ^ (e >> 1 == 3)) + 4 * (e >> 1));
        }
    }
    dst[idx] = w << 6 | w >> 26;
}
// scales [groups][N] -> [rows][16 n_tiles], row r from group r / repeat, zero beyond; zero points: nibbles [groups][N / 2] -> bytes, zrows rows
__global__ __launch_bounds__(256) void q4_pack_scales_kernel(const void *__restrict__ src, int es, const uint8_t *__restrict__ zsrc, int64_t ld, int groups, int rows, int zrows,
                                                             int repeat, int n0, int n, int np, void *__restrict__ dst, uint8_t *__restrict__ zdst) {
    const size_t idx = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (idx >= (size_t)rows * np) return;
    const int row = (int)(idx / np), col = (int)(idx % np), group = row / repeat;
    const bool there = group < groups && col < n;
    const size_t at = (size_t)group * ld + n0 + col;
    if (es == 4) static_cast<float *>(dst)[idx] = there ? static_cast<const float *>(src)[at] : 0.f;
    else static_cast<h16_t *>(dst)[idx] = there ? static_cast<const h16_t *>(src)[at] : (h16_t)0;
    if (row < zrows) zdst[idx] = (uint8_t)(zsrc == nullptr ? 8 : there ? (zsrc[(size_t)group * (ld / 2) + ((n0 + col) >> 1)] >> (4 * ((n0 + col) & 1))) & 15 : 0);
}

// ---- which form --------------------------------------------------------------------------------------------------
// By tiles of 16 columns (n), 128-feature blocks (k) and operand columns (C).  us for group 128, fp16 where nothing else is said:
//   n >= 512: the few form with the operand in LDS up to 4 columns, or 8 of a matrix below n = 1024, and 32 KB, else the shared form (k = 64, n = 1792:
//   one column 26.2 / 27.9, four 31.2 / 27.7; k = 16, n = 1792: four 10.6 / 12.2, eight 13.3 / 12.5; eight, n = 1020: 9.2 / 10.8, 1280: 11.5 / 11.1; k = 32:
//   n = 640: 12.6 / 11.4, 1032: 19.3 / 14.4).  One tile a block with one or two columns while that makes no more than three blocks a CU, else two (one column,
//   k = 32: n = 640: one tile 8.8, two 9.6, n = 800: 10.2, 9.5, n = 1536: 15.7, 13.3; k = 64: n = 520: 12.5, 13.9, n = 640: 13.2, 14.9, n = 800: 16.0, 15.4).
//   bf16 rows of the few form save the launch that scales them: up to 16 columns and 16 KB (k = 4, n = 640, sixteen 6.2 / 9.4; n = 1792, eight 6.5 / 9.4)
//   n < 512, k > 64: eight waves and the operand in LDS up to 64 KB of it, else the shared form (k = 64, n = 160, one column 6.9, four waves from L2 8.4,
//   shared 12.1; k = 224 14.2 / 20.9 / 17.0)
//   else the few form with the operand from L2, in groups of 16 columns: four waves while it makes 256 blocks, eight waves and two tiles while it makes
//   512, or 1024 where contractions are short, else the shared form (k = 32, n = 160: 8 columns 6.6 / 7.6 / 10.2, 24: 11.7 / 9.5 / 11.6, 64: 18.5 / 16.2 / 13.9; k = 16, n = 256, 64 columns:
//   15.8 / 11.5 / 12.4)
// Groups of 32 have four times the scales, for which two tiles leave no registers: one tile a block while that makes 256 blocks, or little work, and with
// n >= 512 up to 8 columns of a matrix below n = 1024 (k = 64, n = 1792, one column: one tile 41.6, shared 33.2; n = 640: 20.1, 18.0; k = 4, n = 640, four: 5.2,
// 6.2; k = 64, n = 256, 24 columns 23.1 / 14.4; k = 4, n = 256, 48 6.6 / 9.2)
// bf16 operands, below n = 512: with one or two columns through LDS, where they are scaled, from n = 256 on, else as they are (k = 32, n = 480: one column
// 7.6 / 8.7, two 8.4 / 8.9, four 10.3 / 9.0; n = 256: one 6.2 / 6.8, two 6.9 / 6.8; k = 64, n = 80: one 8.3 / 8.2, two 9.6 / 8.5).
enum { FEW_LDS_WIDE, FEW_LDS, FEW_LDS_NARROW, FEW_WIDE, FEW, SHARED };
int form_of(const Q4View &m, int C, bool bf16) {
    const int n = m.n_tiles, k = m.k_blocks, blocks = n * ((C + 15) / 16), operand = C > 16 ? INT32_MAX : C * k * 256;
    const bool one = m.group == 32;
    if (n >= 512) {
        const int most = bf16 && !one && operand <= kScaled / 2 ? 16 : n < 1024 ? 8 : one ? 0 : 4;
        if (operand > kScaled || C > most) return SHARED;
        return one || (n <= 768 && C <= 2) ? FEW_LDS : FEW_LDS_WIDE;
    }
    if (bf16 && n >= 256 && C <= 2 && operand <= kScaled) return FEW_LDS;
    if (k >= 64 && operand <= 64 * 1024) return FEW_LDS_NARROW;
    if (k > 64) return SHARED;
    if (one) return blocks <= 256 || (long)blocks * k <= 8192 ? FEW : SHARED;
    return blocks <= 256 ? FEW : blocks <= (k <= 16 ? 1024 : 512) ? FEW_WIDE : SHARED;
}
int few_tiles(int form) { return form == FEW_LDS_WIDE || form == FEW_WIDE ? 2 : 1; }

// The shared form's blocks: waves per group (two tiles of 16 columns each) and splits of the contraction, by the steps that the fullest CU has to
// do; a split costs its partial sums and, the first one, a launch (us, fp16: 8192 x 57344, 32 columns: 8 waves 57, 8 and two splits 68; 8192 x
// 10240, 32 columns: 6 waves and four splits 19, 8 and four 21, 7 and two 30; 28672 x 8192, 40 columns: 8 waves and eight splits 42, 7 and four 55).
struct SharedShape { int waves, splits; };
SharedShape shared_shape(const Q4View &m, int C) {
    SharedShape best{8, 1};
    float least = INFINITY;
    for (int w = 8; w >= 6; --w)
        for (int sp = 1; sp <= 16 && sp * 4 <= std::max(4, m.k_blocks); ++sp) {
            const int blocks = (m.n_tiles + 2 * w - 1) / (2 * w) * sp, steps = (m.k_blocks + sp - 1) / sp;
            const float cost = (float)((blocks + 255) / 256) * w * (steps + 4) * (1.0f + (sp > 1 ? 0.1f + 0.01f * sp : 0.f));
            if (cost < least) { least = cost; best = SharedShape{w, sp}; }
        }
    const int per = (m.k_blocks + best.splits - 1) / best.splits;
    best.splits = (m.k_blocks + per - 1) / per;
    return best;
}

int shared_blocks(const Q4View &m, const SharedShape &sh) { return (m.n_tiles + 2 * sh.waves - 1) / (2 * sh.waves); }

template <int ST, int FL>
void launch_few(const Q4View &m, int form, const Q4In &in, int C, int T, const Q4Out &out, hipStream_t s) {
    const int parts = C / T, rows = 16 / parts;
    const dim3 grid((m.n_tiles + few_tiles(form) - 1) / few_tiles(form), (T + rows - 1) / rows);
    const size_t lds = (size_t)std::min(C, 16) * m.k_blocks * 256;
#define HX_FEW(UT, W, R, XLDS, BF16_AS)                                                                                                                       \
    do {                                                                                                                                                      \
        if constexpr (ST == HX_T_BF16) {                                                                                                                      \
            if (in.bf16) {                                                                                                                                    \
                hipLaunchKernelGGL((q4_few_kernel<ST, UT, FL, W, R, XLDS, BF16_AS>), grid, dim3(64 * W), XLDS ? lds : 0, s, m, in.x, in.ldx, parts, T, out);  \
                break;                                                                                                                                        \
            }                                                                                                                                                 \
        }                                                                                                                                                     \
        hipLaunchKernelGGL((q4_few_kernel<ST, UT, FL, W, R, XLDS, OP_F16>), grid, dim3(64 * W), XLDS ? lds : 0, s, m, in.x, in.ldx, parts, T, out);           \
    } while (0)
    if constexpr (FL > 1) {
        if (form == FEW_LDS_WIDE) HX_FEW(2, 4, 2, true, OP_SCALED);
        else if (form == FEW_WIDE) HX_FEW(2, 8, 2, false, OP_BF16);
    }
    if (form == FEW_LDS) HX_FEW(1, 4, (FL == 1 ? 2 : 4), true, OP_SCALED);
    else if (form == FEW_LDS_NARROW) HX_FEW(1, 8, (FL == 1 ? 2 : 4), true, OP_BF16);
    else if (form == FEW) HX_FEW(1, 4, (FL == 1 ? 2 : 4), false, OP_BF16);
#undef HX_FEW
}
template <int ST, int NB, int FL>
void launch_shared(const Q4View &m, const Q4In &in, int C, int T, const Q4Out &out, float *part, hipStream_t s) {
    const SharedShape sh = shared_shape(m, C);
    const int per = (m.k_blocks + sh.splits - 1) / sh.splits;
    const dim3 grid(shared_blocks(m, sh), sh.splits);
    hipLaunchKernelGGL((q4_shared_kernel<ST, NB, FL>), grid, dim3(128 * sh.waves), 0, s, m, in.x, (uint32_t)in.ldx, C, T, out, per, sh.splits == 1 ? nullptr : part);
    if (sh.splits > 1) hipLaunchKernelGGL(q4_finish_kernel, dim3((m.n_tiles * 16 + 1023) / 1024, T), dim3(256), 0, s, m, part, sh.splits, C, T, out);
}
template <int ST, int FL>
void launch_cols(const Q4View &m, const Q4In &in, int C, int T, const Q4Out &out, float *part, hipStream_t s) {
    const int form = form_of(m, C, in.bf16);
    if (form != SHARED) launch_few<ST, FL>(m, form, in, C, T, out, s);
    else if (C <= 16) launch_shared<ST, 1, FL>(m, in, C, T, out, part, s);
    else if (C <= 32) launch_shared<ST, 2, FL>(m, in, C, T, out, part, s);
    else if (C <= 48) launch_shared<ST, 3, FL>(m, in, C, T, out, part, s);
    else launch_shared<ST, 4, FL>(m, in, C, T, out, part, s);
}
template <int ST>
void launch_type(const Q4View &m, const Q4In &in, int C, int T, const Q4Out &out, float *part, hipStream_t s) {
    if (m.group >= 128) launch_cols<ST, 4>(m, in, C, T, out, part, s);
    else if (m.group == 64) launch_cols<ST, 2>(m, in, C, T, out, part, s);
    else launch_cols<ST, 1>(m, in, C, T, out, part, s);
}

}  // namespace

size_t q4_part_floats(const Q4View &m) {
    size_t most = 0;
    for (int c = 1; c <= kQ4Rows; ++c)
        if (form_of(m, c, false) == SHARED && shared_shape(m, c).splits > 1) most = std::max(most, (size_t)shared_shape(m, c).splits * c * m.n_tiles * 16);
    return most;
}
int q4_best_units(const Q4View &m, int T) {
    const int form = form_of(m, 2 * T, false);
    if (form != SHARED) return (m.n_tiles + few_tiles(form) - 1) / few_tiles(form);
    const SharedShape sh = shared_shape(m, 2 * T);
    return sh.splits > 1 ? (m.n_tiles * 16 + 1023) / 1024 : shared_blocks(m, sh);
}
bool q4_takes_bf16(const Q4View &m, int T) { return form_of(m, T, true) != SHARED; }
void launch_q4(const Q4View &m, const Q4In &in, int T, const Q4Out &out, float *part, hipStream_t s) {
    const int C = out.parts * T;
    if (m.type == HX_T_F32) launch_type<HX_T_F32>(m, in, C, T, out, part, s);
    else if (m.type == HX_T_F16) launch_type<HX_T_F16>(m, in, C, T, out, part, s);
    else launch_type<HX_T_BF16>(m, in, C, T, out, part, s);
}
void launch_q4_parts(int type, const void *x, const void *x2, int64_t ldx, const float *g, float eps, int K, int Kp, int T, int parts, h16_t *out, int32_t *exps,
                     hipStream_t s) {
    const size_t es = type == HX_T_F32 ? 4 : 2;
    const bool pieces = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(x2)) % 16 == 0) && (ldx * es) % 16 == 0 && K % 8 == 0;
#define HX_PARTS(TY, N)                                                                                                                                \
    do {                                                                                                                                               \
        if (pieces) hipLaunchKernelGGL((q4_parts_kernel<TY, true, N>), dim3(T), dim3(1024), 0, s, x, x2, ldx, g, eps, K, Kp, T, out, exps);            \
        else hipLaunchKernelGGL((q4_parts_kernel<TY, false, N>), dim3(T), dim3(1024), 0, s, x, x2, ldx, g, eps, K, Kp, T, out, exps);                  \
    } while (0)
    if (type == HX_T_F32) HX_PARTS(HX_T_F32, 2);
    else if (type == HX_T_F16) HX_PARTS(HX_T_F16, 2);
    else if (parts == 2) HX_PARTS(HX_T_BF16, 2);
    else HX_PARTS(HX_T_BF16, 1);
#undef HX_PARTS
}
void launch_q4_copy(const h16_t *x, int64_t ldx, int K, int Kp, int T, h16_t *out, hipStream_t s) {
    hipLaunchKernelGGL(q4_copy_kernel, dim3(T), dim3(256), 0, s, x, ldx, K, Kp, out);
}
void launch_q4_pack(const Q4View &m, const uint8_t *w4, const void *scales, const uint8_t *zeros, int64_t ld, int K, int group, int n0, hipStream_t s) {
    const size_t words = (size_t)m.k_blocks * m.n_tiles * 256, cells = (size_t)m.scale_rows * m.n_tiles * 16;
    hipLaunchKernelGGL(q4_pack_kernel, dim3((unsigned)((words + 255) / 256)), dim3(256), 0, s, w4, ld / 2, K, n0, m.n_valid, m.n_tiles, m.k_blocks,
                       const_cast<uint32_t *>(static_cast<const uint32_t *>(m.w)));
    hipLaunchKernelGGL(q4_pack_scales_kernel, dim3((unsigned)((cells + 255) / 256)), dim3(256), 0, s, scales, m.type == HX_T_F32 ? 4 : 2, zeros, ld, (int)(((int64_t)K + group - 1) / group),
                       m.scale_rows, m.zeros_row != 0 ? m.scale_rows : 1, std::max(1, group / 128), n0, m.n_valid, m.n_tiles * 16, const_cast<void *>(m.scales),
                       const_cast<uint8_t *>(m.zeros));
}
