// What the translation units of the 4-bit matrices share.
#pragma once

#include "hbp_ops.h"

namespace hbp {

struct Q4 {
    const uint8_t *codes;
    const void *scales, *zeros;
    int64_t pitch;   // bytes of a row of codes
    int32_t n_rows, n_cols, groups, shift;  // column k is of group k >> shift
};

// A product y = x W^T of one launch.
struct Q4Product {
    Q4 a;
    const void *x;
    void *y;
    int64_t ldx, ldy, vectors;
    int32_t scale_type;
};

int launch_q4_mv_f32(const Q4Product &p, hipStream_t st);   // by the type of x and y, and whether there are zero points
int launch_q4_mv_f16(const Q4Product &p, hipStream_t st);
int launch_q4_mv_bf16(const Q4Product &p, hipStream_t st);
int launch_q4_mv_f32_zeros(const Q4Product &p, hipStream_t st);
int launch_q4_mv_f16_zeros(const Q4Product &p, hipStream_t st);
int launch_q4_mv_bf16_zeros(const Q4Product &p, hipStream_t st);

}  // namespace hbp
