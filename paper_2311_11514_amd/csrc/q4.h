// A matrix of 4-bit weights on the device, as hexgen_q4_* and the 4-bit head hold it.
#pragma once
#include "../../include/hexgen.h"
#include "kernels.h"

struct Q4Store {
    Q4View v{};
    int n_in = 0;
    h16_t *planes = nullptr;      // operand columns of a launch, where they are not taken from the caller's rows
    int32_t *exps = nullptr;      // the rows' powers of two
    float *part = nullptr;        // q4_part_floats
    int padded() const { return v.k_blocks * 128; }
};
// group sizes the kernels take
bool q4_group_ok(int group);
// columns n0 .. n0 + n - 1 of w4 [n_in][total / 2], scales [groups][total], zeros [groups][total / 2] or NULL (host or device); waits for
// the device.  The store is empty afterwards if that fails.
hexgen_status_t q4_load(Q4Store *q, hexgen_dtype_t dtype, int n_in, int total, int n0, int n, int group, const void *w4, const void *scales, const void *zeros);
void q4_free(Q4Store *q);
