// Test driver for the paged 4-bit cache's host code and address arithmetic
// under AddressSanitizer and UndefinedBehaviorSanitizer (test infrastructure
// only): every refusal of its entry points, none of which reaches the device,
// and the offsets that the kernels compute, with damaged page ids and slots,
// against the sizes of the arrays.  Exit status 0 means that every check held.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../../include/buddy.h"
#include "../../paper_2606_09514_amd/csrc/kv4.h"

using namespace buddy;

static int failures = 0;
#define EXPECT(cond, what)                                                                             \
    do {                                                                                               \
        if (!(cond)) { fprintf(stderr, "FAILED: %s (line %d)\n", what, __LINE__); ++failures; }        \
    } while (0)

struct At { int64_t k, ks, v, vs; };

// What a lane of the kernels computes.
static At slab_at(const Kv4Dims& d, int32_t p0, int32_t p1, int32_t head, int32_t j, int lane) {
    const Kv4SlabBase b[2] = {kv4_slab_base(d, p0, head, j, 0), kv4_slab_base(d, p1, head, j, 1)};
    const Kv4SlabLane l = kv4_slab_lane(d, lane);
    const int kh = (lane & 15) >= 8, vh = lane >= 32;
    return At{b[kh].codes + l.k, b[kh].scales + l.ks, b[vh].codes + l.v, b[vh].scales + l.vs};
}

static void offsets() {
    const int32_t bad[] = {-1, -7, INT32_MIN, INT32_MAX};
    for (int hd : {64, 128})
        for (int shift = 4; shift <= 8; ++shift)
            for (int n_kv : {1, 3, 40}) {
                const Kv4Dims d{5, shift, n_kv, hd};
                const int rows = 1 << shift;
                const int64_t codes = (int64_t)d.n_pages * n_kv * rows * hd / 2, scales = codes / 16;
                // rows and scales of the pool: each byte once
                EXPECT(kv4_code_offset(d, d.n_pages - 1, n_kv - 1, rows - 1) + hd / 2 == codes, "last row");
                EXPECT(kv4_scale_offset(d, d.n_pages - 1, n_kv - 1, hd / 32 - 1, rows - 1) + 1 == scales, "last scale");
                EXPECT(kv4_code_offset(d, 1, 0, 0) == codes / d.n_pages, "page stride");
                for (int32_t id : bad) EXPECT(kv4_page_or_none(d, id) == -1, "bad page");
                EXPECT(kv4_page_or_none(d, d.n_pages) == -1 && kv4_page_or_none(d, 4) == 4, "page bound");
                int32_t page, row;
                EXPECT(!kv4_slot(d, -1, &page, &row) && !kv4_slot(d, INT32_MIN, &page, &row), "negative slot");
                EXPECT(!kv4_slot(d, d.n_pages * rows, &page, &row) && !kv4_slot(d, INT32_MAX, &page, &row), "far slot");
                EXPECT(kv4_slot(d, d.n_pages * rows - 1, &page, &row) && page == 4 && row == rows - 1, "last slot");
                // every lane of an attention slab, whatever the pages are
                for (int32_t p0 : {-1, 0, 4})
                    for (int32_t p1 : {-1, 0, 4})
                        for (int j = 0; j < 512; j += 32)
                            for (int lane = 0; lane < 64; ++lane) {
                                const At at = slab_at(d, p0, rows > 16 ? p0 : p1, n_kv - 1, j, lane);
                                EXPECT(at.k >= 0 && at.k + 4 * (hd / 2) + hd / 8 <= codes && at.k % (hd / 8) == 0, "k");
                                EXPECT(at.v >= 0 && at.v + 7 * (hd / 2) + hd / 32 <= codes && at.v % (hd / 32) == 0, "v");
                                EXPECT(at.ks >= 0 && at.ks + 8 <= scales && at.ks % 8 == 0, "k scales");
                                EXPECT(at.vs >= 0 && at.vs + 8 <= scales && at.vs % 8 == 0, "v scales");
                            }
                if (rows > 16)
                    for (int j = 0; j < 512; j += 32) {
                        const Kv4SlabBase x = kv4_slab_base(d, 3, n_kv - 1, j, 0), y = kv4_slab_base(d, 3, n_kv - 1, j, 1);
                        EXPECT(x.codes == y.codes && x.scales == y.scales, "one base a page");
                    }
                // the scales are those of the lane's rows and elements
                for (int lane = 0; lane < 64; ++lane) {
                    const int m = lane & 15, r = lane >> 4;
                    const At at = slab_at(d, 2, rows > 16 ? 2 : 1, 0, 64, lane);
                    const int krow = 64 + 8 * (m / 4), vrow = 64 + 8 * r;
                    const int32_t kp = rows > 16 || m < 8 ? 2 : 1, vp = rows > 16 || r < 2 ? 2 : 1;
                    EXPECT(at.k == kv4_code_offset(d, kp, 0, (krow + m % 4) & (rows - 1)) + r * hd / 8, "k place");
                    EXPECT(at.ks == kv4_scale_offset(d, kp, 0, r * hd / 4 / 32, krow & (rows - 1)), "k scale place");
                    EXPECT(at.v == kv4_code_offset(d, vp, 0, vrow & (rows - 1)) + m * hd / 32, "v place");
                    EXPECT(at.vs == kv4_scale_offset(d, vp, 0, m * hd / 16 / 32, vrow & (rows - 1)), "v scale place");
                }
                // the lanes of a slab read each of its rows' bytes, once
                static uint8_t seen[5 * 40 * 256 * 64];
                for (int which = 0; which < 2; ++which) {
                    memset(seen, 0, codes);
                    for (int lane = 0; lane < 64; ++lane) {
                        const At at = slab_at(d, 3, rows > 16 ? 3 : 1, 0, 32, lane);
                        if (which == 0)
                            for (int u = 0; u < 2; ++u)
                                for (int i = 0; i < hd / 8; ++i) ++seen[at.k + u * 4 * (hd / 2) + i];
                        else
                            for (int r = 0; r < 8; ++r)
                                for (int i = 0; i < hd / 32; ++i) ++seen[at.v + r * (hd / 2) + i];
                    }
                    int64_t total = 0;
                    for (int64_t i = 0; i < codes; ++i) { total += seen[i]; EXPECT(seen[i] <= 1, "byte read twice"); }
                    EXPECT(total == 32 * hd / 2, "bytes of a slab");
                    for (int i = 0; i < 32; ++i) {
                        const int32_t pg = rows > 16 || i < 16 ? 3 : 1;
                        EXPECT(seen[kv4_code_offset(d, pg, 0, (32 + i) & (rows - 1))] == 1, "row of a slab");
                    }
                }
            }
    // a pool past 4 GiB
    const Kv4Dims big{1 << 23, 8, 40, 128};
    EXPECT(kv4_code_offset(big, (1 << 23) - 1, 39, 255) + 64 == ((int64_t)1 << 31) * 40 * 64, "64-bit offsets");
    EXPECT(kv4_slab_rows(0, 0, 32, 32) == 0 && kv4_slab_rows(0, 0, 32, 0) == 0 && kv4_slab_rows(0, 0, 32, 33) == 1, "ends");
    EXPECT(kv4_slab_rows(0, 0, 0, 31) == 0x7fffffffu && kv4_slab_rows(0, 0, 0, INT32_MAX) == 0xffffffffu, "ends");
    EXPECT(kv4_slab_rows(-1, 2, 0, 20) == 0xf0000u && kv4_slab_rows(2, -1, 0, 20) == 0xffffu, "no page");
}

// The scales and codes that the lanes of an attention slab read, by the
// kernel's choice of bases, are those of their rows for every pair of pages of
// 16 rows, neighbours in the pool among them.
static void bases() {
    for (int hd : {64, 128})
        for (int n_kv : {1, 2, 3})
            for (int shift : {4, 5}) {
                const Kv4Dims d{6, shift, n_kv, hd};
                const int rows = 1 << shift;
                for (int p0 = 0; p0 < 6; ++p0)
                    for (int p1 = shift == 4 ? 0 : p0; p1 < (shift == 4 ? 6 : p0 + 1); ++p1)
                        for (int head = 0; head < n_kv; ++head)
                            for (int lane = 0; lane < 64; ++lane) {
                                const int m = lane & 15, r = lane >> 4, j = 64;
                                const Kv4SlabBase b0 = kv4_slab_base(d, p0, head, j, 0), b1 = kv4_slab_base(d, p1, head, j, 1);
                                const Kv4SlabBase kb = kv4_one_base(b0, b1) || m < 8 ? b0 : b1;
                                const Kv4SlabBase vb = kv4_one_base(b0, b1) || r < 2 ? b0 : b1;
                                const Kv4SlabLane at = kv4_slab_lane(d, lane);
                                const int krow = 8 * (m / 4), vrow = 8 * r, kp = krow < 16 ? p0 : p1, vp = vrow < 16 ? p0 : p1;
                                EXPECT(kb.codes + at.k == kv4_code_offset(d, kp, head, (krow + m % 4) & (rows - 1)) + r * hd / 8, "k base");
                                EXPECT(kb.scales + at.ks == kv4_scale_offset(d, kp, head, r * hd / 4 / 32, krow & (rows - 1)), "k scale base");
                                EXPECT(vb.codes + at.v == kv4_code_offset(d, vp, head, vrow & (rows - 1)) + m * hd / 32, "v base");
                                EXPECT(vb.scales + at.vs == kv4_scale_offset(d, vp, head, m * hd / 16 / 32, vrow & (rows - 1)), "v scale base");
                            }
            }
}

static uint32_t bits(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }

static void scales() {
    for (int e = -125; e <= 125; ++e) {
        EXPECT(kv4_scale_code(bits(ldexpf(7.f, e))) == e + 127, "7 * 2^e");
        if (e < 125) EXPECT(kv4_scale_code(bits(nextafterf(ldexpf(7.f, e), INFINITY))) == e + 128, "past 7 * 2^e");
    }
    EXPECT(kv4_scale_code(0) == 2 && kv4_scale_code(1) == 2 && kv4_scale_code(bits(1e-38f)) == 2, "tiny");
    EXPECT(kv4_scale_code(bits(3.4e38f)) == 252, "huge");
    EXPECT(kv4_scale_code(bits(INFINITY)) == 255 && kv4_scale_code(0x7fc00000u) == 255, "not finite");
}

static void refusals() {
    alignas(16) static uint8_t mem[64];
    int32_t* i = (int32_t*)mem;
    const buddy_kv4 good{mem, mem, mem, mem, 4, 64, 8, 128};
    struct { void (*edit)(buddy_kv4&); buddy_status want; } pools[] = {
        {[](buddy_kv4& c) { c.k = nullptr; }, BUDDY_EINVAL},
        {[](buddy_kv4& c) { c.v_scale = nullptr; }, BUDDY_EINVAL},
        {[](buddy_kv4& c) { c.v += 8; }, BUDDY_EINVAL},
        {[](buddy_kv4& c) { c.k_scale += 4; }, BUDDY_EINVAL},
        {[](buddy_kv4& c) { c.head_dim = 96; }, BUDDY_ESHAPE},
        {[](buddy_kv4& c) { c.head_dim = 0; }, BUDDY_ESHAPE},
        {[](buddy_kv4& c) { c.page_rows = 8; }, BUDDY_ESHAPE},
        {[](buddy_kv4& c) { c.page_rows = 48; }, BUDDY_ESHAPE},
        {[](buddy_kv4& c) { c.page_rows = 512; }, BUDDY_ESHAPE},
        {[](buddy_kv4& c) { c.n_kv_heads = 0; }, BUDDY_ESHAPE},
        {[](buddy_kv4& c) { c.n_pages = 0; }, BUDDY_EINVAL},
        {[](buddy_kv4& c) { c.n_pages = 1 << 25; }, BUDDY_ECAPACITY},
    };
    buddy_kv4_attn at;
    memset(&at, 0, sizeof(at));
    at.q = mem; at.out = mem; at.q_stride = at.out_stride = 4096; at.dtype = BUDDY_BF16; at.n_heads = 32;
    at.n_rows = 2; at.max_rows = 1; at.max_len = 100; at.max_pages = 4; at.table = i; at.len = i; at.cu_rows = i;
    at.scale = 1.f; at.workspace = mem; at.workspace_bytes = (size_t)1 << 40;
    for (auto& p : pools) {
        buddy_kv4 c = good;
        p.edit(c);
        EXPECT(buddy_kv4_append(&c, BUDDY_BF16, mem, 1024, mem, 1024, i, 1, nullptr) == p.want, "append pool");
        EXPECT(buddy_kv4_read(&c, i, 1, BUDDY_BF16, mem, 1024, mem, 1024, nullptr) == p.want, "read pool");
        EXPECT(buddy_kv4_attention(&c, &at, 2, nullptr) == p.want, "attention pool");
        EXPECT(buddy_kv4_attention_workspace(&c, &at, 2) == 0, "workspace pool");
    }
    EXPECT(buddy_kv4_append(nullptr, BUDDY_BF16, mem, 1024, mem, 1024, i, 1, nullptr) == BUDDY_EINVAL, "no cache");
    EXPECT(buddy_kv4_append(&good, 7, mem, 1024, mem, 1024, i, 1, nullptr) == BUDDY_EINVAL, "dtype");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, 1024, mem, 1024, i, -1, nullptr) == BUDDY_EINVAL, "rows");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, 1020, mem, 1024, i, 1, nullptr) == BUDDY_EINVAL, "stride");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, 512, mem, 1024, i, 2, nullptr) == BUDDY_EINVAL, "short stride");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, -1024, mem, 1024, i, 1, nullptr) == BUDDY_EINVAL, "back");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, INT64_MAX & ~15LL, mem, 1024, i, 2, nullptr) == BUDDY_EINVAL, "far");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem + 2, 1024, mem, 1024, i, 1, nullptr) == BUDDY_EINVAL, "odd k");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, 1024, nullptr, 1024, i, 1, nullptr) == BUDDY_EINVAL, "no v");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, 1024, mem, 1024, nullptr, 1, nullptr) == BUDDY_EINVAL, "no slots");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, nullptr, 0, nullptr, 0, nullptr, 0, nullptr) == BUDDY_OK, "no rows");
    EXPECT(buddy_kv4_read(&good, nullptr, 0, BUDDY_F32, nullptr, 0, nullptr, 0, nullptr) == BUDDY_OK, "no rows");
    EXPECT(buddy_kv4_read(&good, i, 1, BUDDY_F32, mem, 1024, mem + 4, 1024, nullptr) == BUDDY_EINVAL, "odd v");

    const buddy_qk_form form{32, 8, 128, 128, 0, BUDDY_BF16, 1e-6f, 1e4f, nullptr, nullptr};
    struct { void (*edit)(buddy_qk_form&); buddy_status want; } forms[] = {
        {[](buddy_qk_form& f) { f.n_heads = 0; }, BUDDY_ESHAPE},
        {[](buddy_qk_form& f) { f.n_kv_heads = 2000; }, BUDDY_ESHAPE},
        {[](buddy_qk_form& f) { f.head_dim = 80; }, BUDDY_ESHAPE},
        {[](buddy_qk_form& f) { f.rope_dim = 24; }, BUDDY_ESHAPE},
        {[](buddy_qk_form& f) { f.rope_dim = 144; }, BUDDY_ESHAPE},
        {[](buddy_qk_form& f) { f.rope_dim = -16; }, BUDDY_ESHAPE},
        {[](buddy_qk_form& f) { f.dtype = 2; }, BUDDY_EINVAL},
        {[](buddy_qk_form& f) { f.rms_eps = -1.f; }, BUDDY_EINVAL},
        {[](buddy_qk_form& f) { f.rms_eps = NAN; }, BUDDY_EINVAL},
        {[](buddy_qk_form& f) { f.rope_theta = 0.f; }, BUDDY_EINVAL},
        {[](buddy_qk_form& f) { f.k_norm = (void*)8; }, BUDDY_EINVAL},
    };
    for (auto& p : forms) {
        buddy_qk_form f = form;
        p.edit(f);
        EXPECT(buddy_qk_norm_rope(&f, mem, 4096, mem, 1024, i, 1, mem, 4096, mem, 1024, nullptr) == p.want, "form");
        EXPECT(buddy_kv4_append_qkv(&good, &f, mem, 4096, mem, 1024, mem, 1024, i, i, 1, mem, 4096, nullptr) == p.want, "form");
    }
    EXPECT(buddy_qk_norm_rope(nullptr, mem, 4096, mem, 1024, i, 1, mem, 4096, mem, 1024, nullptr) == BUDDY_EINVAL, "none");
    EXPECT(buddy_qk_norm_rope(&form, mem, 4096, mem, 1024, nullptr, 1, mem, 4096, mem, 1024, nullptr) == BUDDY_EINVAL, "pos");
    EXPECT(buddy_qk_norm_rope(&form, mem, 4096, mem, 1024, i, 2, mem, 4088, mem, 1024, nullptr) == BUDDY_EINVAL, "out");
    EXPECT(buddy_qk_norm_rope(&form, mem, 4096, mem, 1024, i, -2, mem, 4096, mem, 1024, nullptr) == BUDDY_EINVAL, "rows");
    EXPECT(buddy_qk_norm_rope(&form, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, 0, nullptr) == BUDDY_OK, "none");
    buddy_qk_form other = form;
    other.n_kv_heads = 4;
    EXPECT(buddy_kv4_append_qkv(&good, &other, mem, 4096, mem, 1024, mem, 1024, i, i, 1, mem, 4096, nullptr) == BUDDY_EINVAL, "heads");
    other = form; other.head_dim = other.rope_dim = 64;
    EXPECT(buddy_kv4_append_qkv(&good, &other, mem, 4096, mem, 1024, mem, 1024, i, i, 1, mem, 4096, nullptr) == BUDDY_EINVAL, "width");
    EXPECT(buddy_kv4_append_qkv(&good, &form, mem, 4096, mem, 1024, mem, 1024, i, nullptr, 1, mem, 4096, nullptr) == BUDDY_EINVAL, "slots");

    const int32_t many = (1 << 24) + 1;
    EXPECT(buddy_qk_norm_rope(&form, mem, 4096, mem, 1024, i, many, mem, 4096, mem, 1024, nullptr) == BUDDY_ECAPACITY, "many rows");
    EXPECT(buddy_kv4_append_qkv(&good, &form, mem, 4096, mem, 1024, mem, 1024, i, i, many, mem, 4096, nullptr) == BUDDY_ECAPACITY, "many rows");
    EXPECT(buddy_kv4_append(&good, BUDDY_BF16, mem, 1024, mem, 1024, i, many, nullptr) == BUDDY_ECAPACITY, "many rows");
    EXPECT(buddy_kv4_read(&good, i, many, BUDDY_F32, mem, 1024, mem, 1024, nullptr) == BUDDY_ECAPACITY, "many rows");

    struct { void (*edit)(buddy_kv4_attn&); buddy_status want; } attns[] = {
        {[](buddy_kv4_attn& a) { a.q = nullptr; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.out = (char*)a.out + 8; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.q_stride = 4088; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.out_stride = 4100; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.q_stride = -4096; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.out_stride = INT64_MAX - 15; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.dtype = 5; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.n_heads = 30; }, BUDDY_ESHAPE},
        {[](buddy_kv4_attn& a) { a.n_heads = 17 * 8; }, BUDDY_ESHAPE},
        {[](buddy_kv4_attn& a) { a.n_rows = -1; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.max_rows = 0; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.max_rows = INT32_MAX; }, BUDDY_ECAPACITY},
        {[](buddy_kv4_attn& a) { a.n_rows = (1 << 24) + 1; }, BUDDY_ECAPACITY},
        {[](buddy_kv4_attn& a) { a.max_len = -5; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.max_pages = 0; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.max_pages = INT32_MAX; }, BUDDY_ECAPACITY},
        {[](buddy_kv4_attn& a) { a.table = nullptr; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.len = nullptr; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.cu_rows = nullptr; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.mask = (const uint8_t*)a.q; a.mask_stride = 99; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.scale = NAN; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.scale = INFINITY; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.scale = 0.f; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.scale = -1e-35f; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.scale = 3e38f; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.scale = -2e30f; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.workspace = nullptr; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.workspace = (char*)a.workspace + 4; }, BUDDY_EINVAL},
        {[](buddy_kv4_attn& a) { a.workspace_bytes = 0; }, BUDDY_EINVAL},
    };
    for (auto& p : attns) {
        buddy_kv4_attn a = at;
        p.edit(a);
        EXPECT(buddy_kv4_attention(&good, &a, 2, nullptr) == p.want, "attention");
    }
    EXPECT(buddy_kv4_attention(&good, nullptr, 2, nullptr) == BUDDY_EINVAL, "no arguments");
    EXPECT(buddy_kv4_attention(&good, &at, -1, nullptr) == BUDDY_EINVAL, "negative batch");
    EXPECT(buddy_kv4_attention(&good, &at, 1025, nullptr) == BUDDY_ECAPACITY, "batch");
    EXPECT(buddy_kv4_attention(&good, &at, 0, nullptr) == BUDDY_OK, "no sequences");
    // a byte less than the workspace of these sizes is refused
    for (int rows : {1, 5, 16, 17, 1000})
        for (int len : {0, 1, 33, 2048, 120000, INT32_MAX}) {
            buddy_kv4_attn a = at;
            a.n_rows = rows; a.max_rows = rows; a.max_len = len;
            const size_t n = buddy_kv4_attention_workspace(&good, &a, 1);
            EXPECT(n >= 16, "workspace size");
            a.workspace_bytes = n - 1;
            EXPECT(buddy_kv4_attention(&good, &a, 1, nullptr) == BUDDY_EINVAL, "a byte less");
        }

    uint8_t* u = mem;
    auto plan = [&](int32_t B, int32_t pr, int32_t mp, int32_t np, int32_t rows, int32_t* table) {
        return buddy_plan_pages(i, i, B, pr, table, mp, i, np, i, i, i, i, i, i, rows, u, nullptr);
    };
    EXPECT(plan(0, 64, 4, 4, 4, i) == BUDDY_OK, "no requests");
    EXPECT(plan(-1, 64, 4, 4, 4, i) == BUDDY_EINVAL && plan(2, 64, 4, 4, -4, i) == BUDDY_EINVAL, "negative");
    EXPECT(plan(1025, 64, 4, 4, 4, i) == BUDDY_ECAPACITY && plan(2, 64, 4, 4, 1 << 30, i) == BUDDY_ECAPACITY, "too many");
    EXPECT(plan(2, 24, 4, 4, 4, i) == BUDDY_ESHAPE && plan(2, 8, 4, 4, 4, i) == BUDDY_ESHAPE, "page rows");
    EXPECT(plan(2, 64, 0, 4, 4, i) == BUDDY_EINVAL && plan(2, 64, 4, 0, 4, i) == BUDDY_EINVAL, "no pages");
    EXPECT(plan(2, 64, 1 << 25, 4, 4, i) == BUDDY_ECAPACITY && plan(2, 64, 4, 1 << 25, 4, i) == BUDDY_ECAPACITY, "pages");
    EXPECT(plan(2, 64, 4, 4, 4, nullptr) == BUDDY_EINVAL, "no table");
    EXPECT(buddy_plan_pages(i, i, 2, 64, i, 4, i, 4, i, i, i, i, nullptr, i, 4, u, nullptr) == BUDDY_EINVAL, "no positions");
    EXPECT(buddy_release_pages(i, nullptr, 2, 64, i, 4, i, 4, i, i, i, nullptr) == BUDDY_EINVAL, "no flags");
    EXPECT(buddy_release_pages(i, u, 2, 100, i, 4, i, 4, i, i, i, nullptr) == BUDDY_ESHAPE, "page rows");
    EXPECT(buddy_release_pages(i, u, 0, 64, i, 4, i, 4, i, i, i, nullptr) == BUDDY_OK, "no requests");
}

int main() {
    offsets();
    bases();
    scales();
    refusals();
    if (failures) return 1;
    printf("kv4 driver ok\n");
    return 0;
}
