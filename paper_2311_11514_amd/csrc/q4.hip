// Host side of the products with 4-bit weights: argument checks, the repacked matrix, and the choice of how rows reach the kernels.
#include <algorithm>
#include <new>

#include "host.h"
#include "q4.h"

static_assert((int)HX_T_F32 == (int)HEXGEN_F32 && (int)HX_T_BF16 == (int)HEXGEN_BF16 && (int)HX_T_F16 == (int)HEXGEN_F16, "one set of codes");

bool q4_group_ok(int group) { return group == 32 || group == 64 || (group > 0 && group % 128 == 0); }

void q4_free(Q4Store *q) {
    void *ptrs[] = {const_cast<void *>(q->v.w), const_cast<void *>(q->v.scales), const_cast<uint8_t *>(q->v.zeros), q->planes, q->exps, q->part};
    for (void *p : ptrs)
        if (p) (void)hipFree(p);
    *q = Q4Store();
}

namespace {
hexgen_status_t load_into(Q4Store *q, hexgen_dtype_t dtype, int n_in, int total, int n0, int n, int group, const void *w4, const void *scales,
                          const void *zeros, void **tmp) {
    const size_t es = dtype == HEXGEN_F32 ? 4 : 2, groups = ((size_t)n_in + group - 1) / group;
    Q4View &v = q->v;
    q->n_in = n_in;
    v.type = (int)dtype;
    v.group = std::min(group, 128);
    v.n_valid = n;
    v.n_tiles = (n + 15) / 16;
    v.k_blocks = (n_in + 127) / 128;
    v.scale_rows = v.k_blocks * (128 / v.group);
    v.zeros_row = zeros != nullptr ? v.n_tiles * 16 : 0;
    void *p = nullptr;
    HX_HIP(hipMalloc(&p, (size_t)v.k_blocks * v.n_tiles * 1024));
    v.w = p;
    HX_HIP(hipMalloc(&p, (size_t)v.scale_rows * v.n_tiles * 16 * es));
    v.scales = p;
    HX_HIP(hipMalloc(&p, (size_t)(zeros != nullptr ? v.scale_rows : 1) * v.n_tiles * 16));
    v.zeros = static_cast<uint8_t *>(p);
    static_assert(kQ4Rows == 2 * kQ4PartRows, "one size of planes");
    HX_HIP(hipMalloc(reinterpret_cast<void **>(&q->planes), (size_t)q->padded() * kQ4Rows * sizeof(h16_t)));
    HX_HIP(hipMalloc(reinterpret_cast<void **>(&q->exps), kQ4Rows * sizeof(int32_t)));
    HX_HIP(hipMalloc(reinterpret_cast<void **>(&q->part), q4_part_floats(v) * sizeof(float)));
    const size_t wb = (size_t)n_in * (total / 2), sb = groups * total * es, zb = zeros != nullptr ? groups * (total / 2) : 0;
    const size_t s_at = (wb + 255) / 256 * 256, z_at = s_at + (sb + 255) / 256 * 256;
    HX_HIP(hipMalloc(tmp, z_at + zb + 1));
    unsigned char *t = static_cast<unsigned char *>(*tmp);
    HX_HIP(hipMemcpy(t, w4, wb, hipMemcpyDefault));
    HX_HIP(hipMemcpy(t + s_at, scales, sb, hipMemcpyDefault));
    if (zeros != nullptr) HX_HIP(hipMemcpy(t + z_at, zeros, zb, hipMemcpyDefault));
    launch_q4_pack(v, t, t + s_at, zeros != nullptr ? t + z_at : nullptr, total, n_in, group, n0, nullptr);
    HX_HIP(hipGetLastError());
    HX_HIP(hipDeviceSynchronize());
    return HEXGEN_OK;
}
}  // namespace

hexgen_status_t q4_load(Q4Store *q, hexgen_dtype_t dtype, int n_in, int total, int n0, int n, int group, const void *w4, const void *scales, const void *zeros) {
    HX_HIP(hipDeviceSynchronize());
    q4_free(q);
    void *tmp = nullptr;
    const hexgen_status_t rc = load_into(q, dtype, n_in, total, n0, n, group, w4, scales, zeros, &tmp);
    if (tmp) (void)hipFree(tmp);
    if (rc != HEXGEN_OK) q4_free(q);
    return rc;
}

struct hexgen_q4 {
    int n_in, n_out, group;
    hexgen_dtype_t dtype;
    Q4Store store;
};

extern "C" {

hexgen_status_t hexgen_q4_create(int n_in, int n_out, int group, hexgen_dtype_t dtype, hexgen_q4_t **out) {
    if (!out || n_in <= 0 || n_out <= 0 || group <= 0) return HEXGEN_ERR_INVALID_ARG;
    if (dtype != HEXGEN_F32 && dtype != HEXGEN_BF16 && dtype != HEXGEN_F16) return HEXGEN_ERR_INVALID_ARG;
    if (n_out % 2 || !q4_group_ok(group) || n_in > (1 << 24) || n_out > (1 << 24)) return HEXGEN_ERR_SHAPE;
    hexgen_q4 *q = new (std::nothrow) hexgen_q4();
    if (!q) return HEXGEN_ERR_OOM;
    q->n_in = n_in;
    q->n_out = n_out;
    q->group = group;
    q->dtype = dtype;
    *out = q;
    return HEXGEN_OK;
}

void hexgen_q4_destroy(hexgen_q4_t *q) {
    if (!q) return;
    if (q->store.v.w != nullptr) (void)hipDeviceSynchronize();
    q4_free(&q->store);
    delete q;
}

hexgen_status_t hexgen_q4_load(hexgen_q4_t *q, const void *w4, const void *scales, const void *zeros) {
    if (!q || !w4 || !scales) return HEXGEN_ERR_INVALID_ARG;
    return q4_load(&q->store, q->dtype, q->n_in, q->n_out, 0, q->n_out, q->group, w4, scales, zeros);
}

hexgen_status_t hexgen_q4_project(hexgen_q4_t *q, const void *x, int64_t ldx, int n_rows, void *out, void *stream) {
    if (!q || !x || !out || n_rows <= 0 || ldx < q->n_in) return HEXGEN_ERR_INVALID_ARG;
    const size_t es = q->dtype == HEXGEN_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(x) % es || reinterpret_cast<uintptr_t>(out) % (2 * es)) return HEXGEN_ERR_INVALID_ARG;
    const Q4Store &st = q->store;
    if (st.v.w == nullptr) return HEXGEN_ERR_STATE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int parts = q->dtype == HEXGEN_F32 ? 2 : 1, chunk = parts == 2 ? kQ4PartRows : kQ4Rows;
    // 16-bit rows of whole 128-feature blocks in 16-byte pieces are an operand as they are
    const bool pieces = parts == 1 && reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx % 8 == 0 && ldx <= (1 << 24) && q->n_in % 128 == 0;
    for (int r0 = 0; r0 < n_rows; r0 += chunk) {
        const int n = std::min(chunk, n_rows - r0);
        const unsigned char *xr = static_cast<const unsigned char *>(x) + (size_t)r0 * ldx * es;
        const bool bf16 = q->dtype == HEXGEN_BF16 && q4_takes_bf16(st.v, n), scaled = q->dtype != HEXGEN_F16 && !bf16;
        const Q4Out o{static_cast<unsigned char *>(out) + (size_t)r0 * q->n_out * es, (int)q->dtype, nullptr, nullptr, scaled ? st.exps : nullptr, parts};
        Q4In in{st.planes, st.padded(), bf16};
        if (scaled) launch_q4_parts((int)q->dtype, xr, nullptr, ldx, nullptr, 0.f, q->n_in, st.padded(), n, parts, st.planes, st.exps, s);
        else if (pieces) in = Q4In{reinterpret_cast<const h16_t *>(xr), ldx, bf16};
        else launch_q4_copy(reinterpret_cast<const h16_t *>(xr), ldx, q->n_in, st.padded(), n, st.planes, s);
        launch_q4(st.v, in, n, o, st.part, s);
    }
    HX_HIP(hipGetLastError());
    return HEXGEN_OK;
}

}  // extern "C"
