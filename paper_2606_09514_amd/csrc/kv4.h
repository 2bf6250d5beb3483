// Layout and device helpers of the paged 4-bit KV cache, shared by its
// translation units (kv4.hip, kv4_attn.hip).  gfx950 only.
//
// Elements are e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives), 32 of
// a row share an E8M0 scale (2^(code - 127), code 255: NaN), so a row of hd
// elements takes hd / 2 + hd / 32 bytes, 4.25 bits an element.  The format is
// the one gfx950's conversion instructions read and write: a row goes from
// memory to bf16 MFMA operands at two elements an instruction, scale included.
#pragma once

#include "buddy_internal.h"

namespace buddy {

constexpr int kKv4Group = 32;            // elements that share a scale
constexpr int kKv4MinScale = 2;          // scale codes that are written: 2^-125 ..
constexpr int kKv4MaxScale = 252;        // .. 2^125, so that no value overflows or is subnormal
constexpr int kKv4NanScale = 255;
constexpr int kKv4MaxSeqs = 1024;        // sequences of one call (one thread each in a plan)

// Byte offsets of (page, KV head, row): codes [page][head][row][hd / 2],
// scales [page][head][hd / 32][row].  64-bit: a pool passes 4 GiB.
struct Kv4Dims { int32_t n_pages, page_shift, n_kv, hd; };

__host__ __device__ inline int64_t kv4_head(const Kv4Dims& d, int32_t page, int32_t head) {
    return (int64_t)page * d.n_kv + head;
}
__host__ __device__ inline int64_t kv4_code_offset(const Kv4Dims& d, int32_t page, int32_t head, int32_t row) {
    return ((kv4_head(d, page, head) << d.page_shift) + row) * (d.hd / 2);
}
__host__ __device__ inline int64_t kv4_scale_offset(const Kv4Dims& d, int32_t page, int32_t head, int32_t group,
                                                    int32_t row) {
    return ((kv4_head(d, page, head) * (d.hd / kKv4Group) + group) << d.page_shift) + row;
}
// A page id from a table, or -1 for one that the pool does not have.
__host__ __device__ inline int32_t kv4_page_or_none(const Kv4Dims& d, int32_t page) {
    return page >= 0 && page < d.n_pages ? page : -1;
}
// Page and row of a slot, false for a slot that the pool does not have.
__host__ __device__ inline bool kv4_slot(const Kv4Dims& d, int32_t slot, int32_t* page, int32_t* row) {
    if (slot < 0) return false;
    *page = slot >> d.page_shift;
    *row = slot & ((1 << d.page_shift) - 1);
    return *page < d.n_pages;
}

// A slab: 32 consecutive rows of a sequence, from row j (a multiple of 32) on.
// page0 and page1 are the pages of its halves of 16 rows (the same page unless
// page_rows is 16), -1 for none.

// Bit i: row j + i is below `end` and in a page of the pool.
__host__ __device__ inline uint32_t kv4_slab_rows(int32_t page0, int32_t page1, int32_t j, int32_t end) {
    uint32_t rows = end - j >= 32 ? 0xffffffffu : end > j ? (1u << (end - j)) - 1 : 0u;
    if (page0 < 0) rows &= 0xffff0000u;
    if (page1 < 0) rows &= 0x0000ffffu;
    return rows;
}

// Where a lane of an attention wavefront reads a slab, in bytes of the codes'
// and the scales' arrays: a base for the slab's first or second 16 rows (the
// same unless page_rows is 16) plus the lane's offset, with lane = m + 16 r:
//   k:  row 8 (m / 4) + m % 4 (and 4 rows on), hd / 8 bytes, elements hd / 4 r ..
//   ks: the scales of rows 8 (m / 4) .. + 7 for the group of those elements
//   v:  row 8 r (and the 7 after it), hd / 32 bytes, elements hd / 16 m ..
//   vs: the scales of rows 8 r .. + 7 for the group of those elements
// K lanes with m >= 8 and V lanes with r >= 2 take the second base.  Rows
// without a page read page 0: they are not in kv4_slab_rows.
// One base serves all lanes only if both its parts are equal: with one KV head
// and pages p and p + 1 of 16 rows the codes' are and the scales' are not.
struct Kv4SlabBase { int64_t codes, scales; };
struct Kv4SlabLane { uint32_t k, ks, v, vs; };

__host__ __device__ inline Kv4SlabBase kv4_slab_base(const Kv4Dims& d, int32_t page, int32_t head, int32_t j,
                                                     int half) {
    const int64_t first = kv4_head(d, page < 0 ? 0 : page, head) << d.page_shift;
    const int32_t row = ((j + 16 * half) & ((1 << d.page_shift) - 1)) - 16 * half;
    return Kv4SlabBase{(first + row) * (d.hd / 2), first * (d.hd / kKv4Group) + row};
}
__host__ __device__ inline bool kv4_one_base(const Kv4SlabBase& x, const Kv4SlabBase& y) {
    return ((x.codes ^ y.codes) | (x.scales ^ y.scales)) == 0;
}
__host__ __device__ inline Kv4SlabLane kv4_slab_lane(const Kv4Dims& d, int lane) {
    const uint32_t m = lane & 15, r = lane >> 4, hd = d.hd;
    return Kv4SlabLane{(8 * (m >> 2) + (m & 3)) * (hd / 2) + r * (hd / 8),
                       ((r * (hd / 4) / kKv4Group) << d.page_shift) + 8 * (m >> 2),
                       8 * r * (hd / 2) + m * (hd / 32),
                       ((m * (hd / 16) / kKv4Group) << d.page_shift) + 8 * r};
}

struct Kv4Pool {
    uint8_t *k, *v, *ks, *vs;
    Kv4Dims d;
};

// Scale code of a group whose largest magnitude has these fp32 bits: the
// least exponent e with amax <= 7 * 2^e.  Elements up to 7 round to 6 (half a
// step), so no element is off by more than half a step of its own, where the
// usual floor(log2 amax) - 2 clips those in (7, 8) * 2^e to 6.  An infinity
// or NaN makes the group NaN rather than a finite value.
__host__ __device__ inline int kv4_scale_code(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return kKv4NanScale;
    const int c = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return c < kKv4MinScale ? kKv4MinScale : c > kKv4MaxScale ? kKv4MaxScale : c;
}

// A pool that the kernels take: 16-byte aligned arrays, pages of a power of
// two of 16..256 rows, slots within 31 bits.
buddy_status kv4_check_pool(const buddy_kv4* c, Kv4Pool* out);

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace buddy
