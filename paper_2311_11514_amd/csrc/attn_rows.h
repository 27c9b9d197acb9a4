// Attention of a few hundred to a few thousand query rows over the cache, 16-bit types: what the kernels of drafted trees and of windowed rows share.
// Scores are transposed, S^T = K . Q^T: a lane owns query row lane % 32 and, in register x, position 8 (x / 4) + 4 (lane / 32) + x % 4 of a tile of 32.
#pragma once
#include "kernels.h"
#include "kvlayout.h"

#define NEG_INF (-INFINITY)

namespace HX_NS {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

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

// fp16 has no numbers below 2^-24, which both parts of a weight would be cut off at, so that many positions of 2^-20 beside a heavy one lost a tenth and more of their sum.
// Its weights are carried times 2^14, sums and results with them: a weight is exact to 2^-38 of the row's largest one.  bf16 has fp32's exponents.
#ifdef HX_ELEM_F16
constexpr float kWeightShift = 14.f, kWeightUnit = 16384.f;
#else
constexpr float kWeightShift = 0.f, kWeightUnit = 1.f;
#endif
// The running softmax over one tile's scores (sc becomes the weights, times kWeightUnit): m, l and the factor for what was summed up before
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
        sc[x] = __builtin_amdgcn_exp2f(fmaf(sc[x] - base, scale_log2e, kWeightShift));
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

}  // namespace HX_NS
