// Layout and device helpers of 8-bit rows (buddy_mx8), shared by the kernels
// that write, read and multiply them.  gfx950 only.
//
// Elements are e4m3, 32 of a row share an E8M0 scale (2^(code - 127), code
// 255: NaN): the form that gfx950's scaled MFMA takes as it lies in memory.
#pragma once

#include "buddy_internal.h"

namespace buddy {

constexpr int kMx8Group = 32;            // elements that share a scale
constexpr int kMx8MinScale = 10;         // scale codes that are written: 2^-117, whose least element
constexpr int kMx8MaxScale = 247;        // 2^-126 is a normal bf16 number, .. 2^120 (448 * 2^120 < 2^129)
constexpr int kMx8NanScale = 255;
constexpr int kMx8MaxWidth = 1 << 20;
constexpr int kMaxRows = 1 << 24;        // of a call: grids stay within 32 bits of threads

// Scale code of a group whose largest magnitude has these fp32 bits: the
// least exponent e with amax <= 448 * 2^e (448 = 1.75 * 2^8), so that nothing
// is clipped.  An infinity or NaN makes the group NaN.
__host__ __device__ inline int mx8_scale_code(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return kMx8NanScale;
    const int c = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return c < kMx8MinScale ? kMx8MinScale : c > kMx8MaxScale ? kMx8MaxScale : c;
}

// Rows with 16-byte aligned starts and whole 16-byte units apart.
inline bool rows16(const void* p, int64_t stride, int64_t width, int64_t n_rows, int size) {
    return p && ((uintptr_t)p & 15) == 0 && stride >= 0 && stride <= INT64_MAX / 64 / (n_rows > 0 ? n_rows : 1) &&
           stride * size % 16 == 0 && (n_rows <= 1 || stride >= width);
}

// Sizes of 8-bit rows (pointers are not looked at).
inline buddy_status mx8_check_sizes(const buddy_mx8* m) {
    if (!m || m->n_rows < 0 || m->width < 1) return BUDDY_EINVAL;
    if (m->width % 16 || m->width > kMx8MaxWidth) return BUDDY_ESHAPE;
    if (m->n_rows > kMaxRows) return BUDDY_ECAPACITY;
    return BUDDY_OK;
}
inline buddy_status mx8_check(const buddy_mx8* m) {
    const buddy_status st = mx8_check_sizes(m);
    if (st != BUDDY_OK) return st;
    const int64_t room = 16 * (int64_t)((m->width + 511) / 512);
    if (m->n_rows > 0 && (!rows16(m->codes, m->code_stride, m->width, m->n_rows, 1) ||
                          !rows16(m->scales, m->scale_stride, room, m->n_rows, 1)))
        return BUDDY_EINVAL;
    return BUDDY_OK;
}

inline bool is_dtype(int32_t t) { return t == BUDDY_F32 || t == BUDDY_BF16; }

}  // namespace buddy
