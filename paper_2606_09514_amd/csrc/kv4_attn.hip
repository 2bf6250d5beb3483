// Grouped-query attention over the paged 4-bit KV cache (gfx950).
//
// out = sum_j softmax_j(scale q . k_j) v_j over the cached rows j that a new
// row may see: at or before its own position, and not masked out.  One pass
// over the rows with the running maximum and sum of the softmax; the rows of
// a sequence are split into chunks over workgroups where there are too few
// sequences and heads to fill the chip, and a second kernel joins the chunks.
#include <math.h>

#include "kv4.h"

namespace buddy {

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

constexpr int kKv4Slab = 32;             // cache rows of one step of a wavefront
constexpr int kKv4MaxChunks = 256;

struct Kv4AttnArgs {
    const char* q;
    char* out;
    int64_t q_stride, out_stride;        // bytes
    Kv4Pool pool;
    const int32_t *table, *len, *cu;
    const uint8_t* mask;
    int64_t mask_stride;
    int32_t B, nq, G, n_rows, max_pages;
    uint32_t inv_G, inv_B, inv_chunks;   // inverses (see quotient)
    int32_t chunks, chunk_slabs;         // of the longest sequence
    int32_t chunk_unit;                  // slabs that a chunk is a multiple of, a power of two
    int32_t fold;                        // prompt form: the order of the tiles (see there)
    int32_t tiles;                       // column tiles that a sequence's new rows take, at most
    float scale_log2;                    // |scale| log2(e)
    uint32_t q_flip;                     // the sign bits of queries, for a negative scale
    float* part_o;                       // [n_rows][nq][chunks][hd]
    float2* part_ml;                     // [n_rows][nq][chunks] maximum and sum
};

// x / n or one more, for x < 2^31, by n's inverse, 2^32 / n rounded up (0 for
// n = 1); exact if x (n - 1) < 2^32.  A division would put its preparation,
// some 20 instructions, before a kernel's first load.
__host__ __device__ inline uint32_t inverse_of(uint32_t n) { return n == 1 ? 0 : (uint32_t)(((1ull << 32) + n - 1) / n); }
__device__ __forceinline__ int quotient(int x, uint32_t inverse) {
    return inverse ? (int)__umulhi((uint32_t)x, inverse) : x;
}

// Slabs of a chunk of a sequence of len rows: those of the longest expected,
// or more, so that the launch's chunks hold all rows.
__device__ __forceinline__ int chunk_slabs_of(const Kv4AttnArgs& a, int len) {
    const int slabs = (len + kKv4Slab - 1) / kKv4Slab;
    if ((int64_t)a.chunk_slabs * a.chunks >= slabs) return a.chunk_slabs;   // a multiple of the unit
    // a sequence longer than max_len said; one more does no harm, every kernel
    // finds the same
    const int per = quotient(slabs + a.chunks - 1, a.inv_chunks);
    return (per + a.chunk_unit - 1) & -a.chunk_unit;
}

// The query row of column c (at most 2^28 + 15) of a sequence, c / G, G <= 16.
__device__ __forceinline__ int column_row(const Kv4AttnArgs& a, int c) { return quotient(c, a.inv_G); }

// A value of a table in the constant address space: a scalar load.  The
// tables are written before the launch, never by it.
typedef const int32_t __attribute__((address_space(4)))* kv4_cptr;
__device__ __forceinline__ int32_t scalar_load(const int32_t* p, int64_t i) {
    return ((kv4_cptr)(uintptr_t)p)[i];
}

__device__ __forceinline__ uint32_t cvt_bf16(uint32_t w, float s, int byte) {
    switch (byte) {
        case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
        case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
        case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
        default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
    }
}

// The scale of byte 0..3 of w for cvt_bf16: the conversions take an fp32
// scale's exponent bits and nothing else of it, so the other bytes may stay.
__device__ __forceinline__ float scale_at(uint32_t w, int byte) {
    return __uint_as_float(byte < 3 ? w << (23 - 8 * byte) : w >> 1);
}
// The same for a byte that lanes differ in: a rotation.
__device__ __forceinline__ float scale_turned(uint32_t w, int byte) {
    return __uint_as_float(__builtin_amdgcn_alignbit(w, w, 8 * byte + 9));
}

// The larger, NaN if either is: fmaxf would first quieten each product's
// result, an instruction a score.  A column with a NaN score is NaN anyway.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float kv4_max16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float kv4_max32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float kv4_sum4(float v) {   // over the four lanes of a column
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 2^x by v_exp_f32: results below 2^-126 are 0, which no sum here notices.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// 2^x for a whole x of at most 0 (-inf among them), exactly; 0 below -149.
__device__ __forceinline__ float power_of_two(float x) {
    return __builtin_amdgcn_ldexpf(1.f, (int)fmaxf(x, -200.f));
}

// Eight fp32 values as PARTS bf16 vectors that add up to them: two parts keep
// 16 bits, three all 24.
template <int PARTS>
__device__ __forceinline__ void split8(const float* x, bf16x8v* out) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        u32x4v w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = pack_bf16x2(r[2 * i], r[2 * i + 1]);
            w[i] = u;
            if (p + 1 < PARTS) {
                r[2 * i] -= __uint_as_float(u << 16);
                r[2 * i + 1] -= __uint_as_float(u & 0xffff0000u);
            }
        }
        out[p] = __builtin_bit_cast(bf16x8v, w);
    }
}

template <int N> struct Bytes;
template <> struct Bytes<1> { typedef uint8_t type; };
template <> struct Bytes<2> { typedef uint16_t type; };
template <> struct Bytes<4> { typedef uint32_t type; };

// One slab's loads.  Lane m + 16 r (m < 16, r < 4) holds, of the 32 rows,
//   K: rows 8 (m / 4) + 4 u + m % 4 (u = 0, 1), elements hd / 4 r ..
//   V: rows 8 r + i (i < 8), elements hd / 16 m ..
// so that the scores of lane (column m, r) are those of rows 8 r + i, the
// rows its V operand has, and the softmax weights are the second product's
// operand as they stand.
template <int HD>
struct Slab {
    u32x4v k[2];                          // hd = 64: the first two words
    uint2 ks;                             // scales of the K rows' block of 8, one group
    uint32_t v[8];
    uint2 vs;                             // scales of V rows 8 r .. 8 r + 7, one group
    uint8_t on;                           // execution map, row `lane` of the slab
};

template <int HD>
__device__ __forceinline__ void load_keys(const uint8_t* codes, const uint8_t* scales, const Kv4SlabLane& at, u32x4v* k,
                                          uint2* ks) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const uint8_t* p = codes + at.k + u * 4 * (HD / 2);
        if constexpr (HD == 128) {
            k[u] = *reinterpret_cast<const u32x4v*>(p);
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            k[u][0] = x.x;
            k[u][1] = x.y;
        }
    }
    *ks = *reinterpret_cast<const uint2*>(scales + at.ks);
}
template <int HD>
__device__ __forceinline__ void load_values(const uint8_t* codes, const uint8_t* scales, const Kv4SlabLane& at,
                                            Slab<HD>& s) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        s.v[i] = *reinterpret_cast<const typename Bytes<HD / 32>::type*>(codes + at.v + i * (HD / 2));
    s.vs = *reinterpret_cast<const uint2*>(scales + at.vs);
}

// The decode form: one workgroup takes a chunk of a sequence's rows, one KV
// head, and 16 columns (query row t and head h of the group: t G + h), its
// four wavefronts every fourth slab.
//   S^T = K Q^T: v_mfma_f32_16x16x32_bf16, K as A from the cache by
//         v_cvt_scalef32_pk_bf16_fp4 (two elements an instruction, exact),
//         queries as B: as they are (bf16) or as three bf16 parts (fp32);
//   O^T += V^T P^T: V as A: eight rows' codes a lane, converted, and pairs of
//         rows joined by v_perm; P as B in two bf16 parts (16 bits, an eighth
//         of a bf16 output's rounding) or three (fp32).
// No operand passes LDS; the running maximum moves only when it grows by more
// than 2^8, so that the sums are rarely rescaled.
// Three workgroups a CU (two where the registers of fp32's parts and the
// execution map do not fit), a slab a wavefront in flight: 96 sequences of
// 2048 rows (40 heads) run at 5.7 TB/s, a large read's rate (two a CU: 5.3);
// one of 120011 (8 heads), where every workgroup has ten slabs a wavefront,
// 28 us or 4.6 TB/s, the difference being the first loads.  Short calls are
// bound by the way to the first product (4.3 us with two slabs): lengths and
// page ids, codes, two products, LDS, each waiting for the one before.
template <typename T, int HD, bool MASKED>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 4 && HD == 128 && MASKED ? 2 : 3)))
void kv4_decode_kernel(Kv4AttnArgs a) {
    constexpr int QP = sizeof(T) == 2 ? 1 : 3, PP = sizeof(T) == 2 ? 2 : 3;
    constexpr int STEPS = HD / 32, CT = HD / 16;
    __shared__ __attribute__((aligned(16))) float s_o[4][16][HD + 4];
    __shared__ float2 s_ml[4][16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, r = lane >> 4;
    const int g = blockIdx.y;
    const int shift = a.pool.d.page_shift;
    Kv4Dims d = a.pool.d;
    d.hd = HD;
    const Kv4SlabLane at = kv4_slab_lane(d, lane);

    for (int w = blockIdx.z; w < a.B * a.tiles; w += gridDim.z) {
        // w / B, which may come out one too large
        int tile0 = quotient(w, a.inv_B), b = w - tile0 * a.B;
        if (b < 0) { --tile0; b += a.B; }
        // the first slab's pages of the expected chunk: beside the loads of
        // the lengths, not behind them
        int32_t next_id[2];                                         // pages of the next slab's halves
        const int j_expected = (blockIdx.x * a.chunk_slabs + wave) * kKv4Slab;
        auto fetch_ids = [&](int j) {
            const int64_t t = (int64_t)b * a.max_pages;
            next_id[0] = scalar_load(a.table, t + min(j >> shift, a.max_pages - 1));
            next_id[1] = scalar_load(a.table, t + min((j + 16) >> shift, a.max_pages - 1));
        };
        fetch_ids(j_expected);
        int first = scalar_load(a.cu, b), last = scalar_load(a.cu, b + 1), cached = scalar_load(a.len, b);
        // all five on their way at once: the compiler would wait for some
        // before it asks for others
        asm volatile("" : "+s"(first), "+s"(last), "+s"(cached), "+s"(next_id[0]), "+s"(next_id[1]));
        const int r0 = max(first, 0), r1 = min(last, a.n_rows);
        const int n_new = r1 - r0;
        const int len = min(max(cached, 0), a.max_pages << shift);
        for (int tile = tile0; tile * 16 < n_new * a.G; tile += a.tiles) {
            const int c = tile * 16 + m;                            // this lane's column
            const bool live = c < n_new * a.G;
            const int t = live ? column_row(a, c) : n_new - 1, h = live ? c - t * a.G : 0;
            const int p_col = len - n_new + t;                      // position of the column's row
            // rows that the tile's last column sees; the chunk of this workgroup
            const int t_last = min(column_row(a, tile * 16 + 15), n_new - 1);
            const int p_first = len - n_new + column_row(a, tile * 16);
            const int end = min(len, len - n_new + t_last + 1);
            const int per = chunk_slabs_of(a, len);
            const int j0 = blockIdx.x * per * kKv4Slab, j1 = end - j0 > per * kKv4Slab ? j0 + per * kKv4Slab : end;
            if (j0 >= end && blockIdx.x > 0) continue;              // no row of this chunk is seen

            // queries: HD / 4 elements from HD / 4 r on; columns behind the
            // last repeat the last row's first head and are not written
            bf16x8v qf[STEPS][QP];
            {
                const char* qp = a.q + (int64_t)(r0 + t) * a.q_stride +
                                 ((int64_t)(g * a.G + h) * HD + r * (HD / 4)) * sizeof(T);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    if constexpr (QP == 1) {
                        u32x4v x = reinterpret_cast<const u32x4v*>(qp)[s];
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[i] = live ? x[i] ^ a.q_flip : 0;
                        qf[s][0] = __builtin_bit_cast(bf16x8v, x);
                    } else {
                        float x[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            x[i] = __uint_as_float(reinterpret_cast<const uint32_t*>(qp)[8 * s + i] ^ a.q_flip);
                        split8<QP>(x, qf[s]);
                    }
                }
            }

            f32x4v acc[CT];
#pragma unroll
            for (int i = 0; i < CT; ++i) acc[i] = f32x4v{0.f, 0.f, 0.f, 0.f};
            // running maximum in units of scale_log2, what the weights subtract
            // (it, or 0 before the first), the score past which it moves; sum
            float mx = -INFINITY, base = 0.f, most = -INFINITY, l = 0.f;
            const float inv_scale = __builtin_amdgcn_rcpf(a.scale_log2);

            // loads of the slab at row j (a multiple of 32 below j1); the page
            // of either half of it, or page 0 with the half left out
            uint32_t alive_next = 0;
            auto load = [&](int j, Slab<HD>& s) {
                // checked here, not where they are fetched: that would wait for them
                const int32_t pg0 = kv4_page_or_none(d, next_id[0]), pg1 = kv4_page_or_none(d, next_id[1]);
                fetch_ids(j + 4 * kKv4Slab);
                alive_next = kv4_slab_rows(pg0, pg1, j, end);
                const Kv4SlabBase b0 = kv4_slab_base(d, pg0, g, j, 0), b1 = kv4_slab_base(d, pg1, g, j, 1);
                if (kv4_one_base(b0, b1)) {
                    load_keys<HD>(a.pool.k + b0.codes, a.pool.ks + b0.scales, at, s.k, &s.ks);
                    load_values<HD>(a.pool.v + b0.codes, a.pool.vs + b0.scales, at, s);
                } else {
                    const Kv4SlabBase kb = m < 8 ? b0 : b1, vb = r < 2 ? b0 : b1;
                    load_keys<HD>(a.pool.k + kb.codes, a.pool.ks + kb.scales, at, s.k, &s.ks);
                    load_values<HD>(a.pool.v + vb.codes, a.pool.vs + vb.scales, at, s);
                }
                if constexpr (MASKED) {
                    const int jm = j + (lane & 31);
                    s.on = jm < end && jm < a.mask_stride ? a.mask[(int64_t)b * a.mask_stride + jm] : 0;
                }
            };

            Slab<HD> next;
            int j = j0 + wave * kKv4Slab;
            if (tile != tile0 || j != j_expected) fetch_ids(j);
            if (j < j1) load(j, next);
            for (; j < j1; j += 4 * kKv4Slab) {
                Slab<HD> s = next;
                uint32_t alive = alive_next;
                if (j + 4 * kKv4Slab < j1) load(j + 4 * kKv4Slab, next);
                if constexpr (MASKED) alive &= (uint32_t)__ballot(s.on != 0 && lane < 32);

                // scores of rows 8 r + i against this lane's column
                float sc[8];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float ks = scale_turned(u ? s.ks.y : s.ks.x, m & 3);
                    f32x4v dd = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int st = 0; st < STEPS; ++st) {
                        u32x4v kf;
#pragma unroll
                        for (int i = 0; i < 4; ++i) kf[i] = cvt_bf16(s.k[u][st], ks, i);
#pragma unroll
                        for (int p = 0; p < QP; ++p)
                            dd = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, kf), qf[st][p],
                                                                        dd, 0, 0, 0);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[4 * u + e] = dd[e];
                }
                // rows that this column does not see
                const bool full = alive == 0xffffffffu && j + kKv4Slab - 1 <= p_first;
                uint32_t vlo = s.vs.x, vhi = s.vs.y;
                uint32_t seen = 0xff;
                bool nan_rows = false;
                if (!full) {
                    asm volatile("; some rows left out");            // a branch, not selects
                    const uint32_t rows8 = (alive >> (8 * r)) & 0xff;
                    const int upto = min(max(p_col - (j + 8 * r) + 1, 0), 8);
                    seen = rows8 & ((1u << upto) - 1);
                    bool nan = false;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (!(seen >> i & 1)) sc[i] = -INFINITY;
                        uint32_t& w8 = i < 4 ? vlo : vhi;
                        const int sh = 8 * (i & 3);
                        // a row that is left out may hold anything: a finite
                        // scale, as 0 times NaN is NaN
                        if (!(rows8 >> i & 1)) w8 = (w8 & ~(0xffu << sh)) | 127u << sh;
                        nan = nan || ((w8 >> sh) & 0xff) == (uint32_t)kKv4NanScale;
                    }
                    nan_rows = __ballot(nan) != 0;
                }
                // running maximum
                float top = sc[0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = max_nan(top, sc[i]);
                if (__ballot(top > most) != 0) {
                    asm volatile("; the maximum grows");
                    const float t = fmaxf(mx, kv4_max32(kv4_max16(top)) * a.scale_log2);
                    base = t == -INFINITY ? 0.f : t;
                    const float al = exp2_hw(mx - base);
                    l *= al;
#pragma unroll
                    for (int i = 0; i < CT; ++i) acc[i] *= al;
                    mx = t;
                    most = (t + 8.f) * inv_scale;
                }
                // weights; a score that is NaN keeps its weight NaN
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = exp2_hw(fmaf(sc[i], a.scale_log2, -base));
#pragma unroll
                for (int i = 0; i < 8; ++i) l += p[i];
                bf16x8v pf[PP];
                split8<PP>(p, pf);
                if (nan_rows) {
                    // a NaN row that only some columns see: count it for them
                    // (all columns of a group of elements alike) and take it
                    // out of the product
                    u32x4v ind, vis;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t& w8 = i < 4 ? vlo : vhi;
                        const int sh = 8 * (i & 3);
                        const bool nan = ((w8 >> sh) & 0xff) == (uint32_t)kKv4NanScale;
                        if (nan) w8 = (w8 & ~(0xffu << sh)) | 127u << sh;
                        const uint32_t one = 0x3f80u << (16 * (i & 1));
                        if (!(i & 1)) ind[i / 2] = vis[i / 2] = 0;
                        if (nan) ind[i / 2] |= one;
                        if (seen >> i & 1) vis[i / 2] |= one;
                    }
                    f32x4v n = {0.f, 0.f, 0.f, 0.f};
                    n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, ind),
                                                                __builtin_bit_cast(bf16x8v, vis), n, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (n[e] > 0.f)
#pragma unroll
                            for (int i = 0; i < CT; ++i) acc[i][e] = NAN;
                }
                // O^T += V^T P^T, two column tiles a byte of codes
                float vsc[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) vsc[i] = scale_at(i < 4 ? vlo : vhi, i & 3);
#pragma unroll
                for (int byte = 0; byte < CT / 2; ++byte) {
                    u32x4v even, odd;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t x0 = cvt_bf16(s.v[2 * i], vsc[2 * i], byte);
                        const uint32_t x1 = cvt_bf16(s.v[2 * i + 1], vsc[2 * i + 1], byte);
                        even[i] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
                        odd[i] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
                    }
#pragma unroll
                    for (int q = 0; q < PP; ++q) {
                        acc[2 * byte] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, even),
                                                                               pf[q], acc[2 * byte], 0, 0, 0);
                        acc[2 * byte + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8v, odd), pf[q], acc[2 * byte + 1], 0, 0, 0);
                    }
                }
            }

            // the four wavefronts' columns, then this chunk's partial or the output
            l = kv4_sum4(l);
            if (r == 0) s_ml[wave][m] = make_float2(mx, l);
#pragma unroll
            for (int e = 0; e < 4; ++e)      // elements CT (4 r + e) + i of the head
#pragma unroll
                for (int i = 0; i < CT; i += 4)
                    *reinterpret_cast<float4*>(&s_o[wave][m][CT * (4 * r + e) + i]) =
                        make_float4(acc[i][e], acc[i + 1][e], acc[i + 2][e], acc[i + 3][e]);
            __syncthreads();
            const int cols = min(16, n_new * a.G - tile * 16);
            for (int x = tid; x < cols * (HD / 4); x += 256) {
                const int cc = x / (HD / 4), e = (x % (HD / 4)) * 4;
                float M = -INFINITY;
#pragma unroll
                for (int v = 0; v < 4; ++v) M = fmaxf(M, s_ml[v][cc].x);
                const float to = M == -INFINITY ? 0.f : M;
                float L = 0.f;
                float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float f = exp2_hw(s_ml[v][cc].x - to);
                    const float4 o = *reinterpret_cast<const float4*>(&s_o[v][cc][e]);
                    L += s_ml[v][cc].y * f;
                    A.x += o.x * f; A.y += o.y * f; A.z += o.z * f; A.w += o.w * f;
                }
                const int tt = column_row(a, tile * 16 + cc), head = g * a.G + tile * 16 + cc - tt * a.G;
                const int64_t row = r0 + tt;
                if (a.chunks == 1) {
                    const float inv = L == 0.f ? 0.f : 1.f / L;    // nothing seen: zeros
                    float y[4] = {A.x * inv, A.y * inv, A.z * inv, A.w * inv};
                    char* op = a.out + row * a.out_stride + ((int64_t)head * HD + e) * sizeof(T);
                    if constexpr (sizeof(T) == 2)
                        *reinterpret_cast<uint2*>(op) =
                            make_uint2(f2bf(y[0]) | (uint32_t)f2bf(y[1]) << 16, f2bf(y[2]) | (uint32_t)f2bf(y[3]) << 16);
                    else
                        *reinterpret_cast<float4*>(op) = make_float4(y[0], y[1], y[2], y[3]);
                } else {
                    const int64_t at = (row * a.nq + head) * a.chunks + blockIdx.x;
                    *reinterpret_cast<float4*>(a.part_o + at * HD + e) = A;
                    if (e == 0) a.part_ml[at] = make_float2(M, L);
                }
            }
            __syncthreads();
        }
    }
}

// The prompt form (bf16 queries, many columns): a workgroup takes 64 NT
// columns of a sequence and KV head, 16 NT a wavefront, and every tile of 64
// rows.  The products are the decode form's.  Tiles pass through LDS as the
// cache holds them (8.5 KB), loaded a tile and a half before they are needed.
// Keys are converted by each wavefront for its NT column tiles.  Values are
// converted once for the workgroup: a thread takes 8 rows of hd / 32 columns,
// joins pairs of rows and stores the product's operands in LDS in the order
// in which a wavefront reads them (16 bytes a lane, no conflicts), one tile
// ahead; two buffers, one barrier a tile.
// Weights are rounded to bf16 once (and the rounded ones added up, by a
// product with ones): each is off by at most half a bf16 step, as an output
// element is by its own rounding; a second part would cost half as many
// products again.  The maximum that they subtract is a whole power of two, so
// where the second slab of a tile moves it, the first slab's weights, in bf16
// by then, are scaled exactly.
// 1024 rows of 32 heads behind 4000 (four sequences, two workgroups a CU in
// whole rounds): 310 us, 970 TFLOP/s, where a large library product reaches
// 1250.  Matrix units are busy 40 % of the time and vector instructions issue
// in 55 %; neither fewer of them nor less LDS changed it: products of 32x32x16
// (a quarter fewer instructions) took 317 us with keys converted once for the
// workgroup and 327 with keys converted by each wavefront (308 then).  Two wavefronts a
// SIMD, all that the registers allow, do not cover each other's waits.
template <int HD>
struct ValueRows {
    uint32_t v[8];
    uint2 vs;
};

template <int HD, int NT, bool MASKED>
__global__ __launch_bounds__(256, 2) void kv4_prompt_kernel(Kv4AttnArgs a) {
    constexpr int STEPS = HD / 32, CT = HD / 16, CPT = HD / 32, GROUPS = HD / 32;
    constexpr int kCols = 64 * NT, kTile = 64;
    __shared__ __attribute__((aligned(16))) u32x4v s_v[2][2][CT][64];   // [buffer][slab][column tile][lane]
    __shared__ __attribute__((aligned(16))) uint8_t s_nan[2][GROUPS][8];  // NaN rows, a bit each
    // tiles as the cache holds them, [slot]: keys with a row's 16-byte pieces
    // at piece ^ (row / 8 % 4), so that a wavefront's reads (rows 8 apart in
    // turn) use all banks; values and scales in order
    constexpr int kSlots = 4, kRowBytes = HD / 2;
    __shared__ __attribute__((aligned(16))) uint8_t s_k[kSlots][kTile * kRowBytes], s_vr[kSlots][kTile * kRowBytes];
    __shared__ __attribute__((aligned(16))) uint8_t s_ks[kSlots][GROUPS][kTile], s_vs[kSlots][GROUPS][kTile];
    __shared__ __attribute__((aligned(4))) uint8_t s_page[kSlots][4];     // quarters that have a page
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, r = lane >> 4;
    // the KV head runs fastest: with eight, each XCD's L2 holds one head's rows
    const int g = blockIdx.x % a.pool.d.n_kv, chunk = blockIdx.x / a.pool.d.n_kv;
    const int shift = a.pool.d.page_shift;
    const int b = blockIdx.z;
    Kv4Dims d = a.pool.d;
    d.hd = HD;
    // the wavefront's 16 rows of a tile: 16 bytes a lane of keys and of values
    // (hd 64: keys in the lower lanes, values in the upper), four scales a lane
    constexpr int kPieces = kRowBytes / 16;                         // of a row
    const int q_row = (lane / kPieces) % 16, q_piece = lane % kPieces;
    const int q_swz = HD == 128 ? ((2 * wave + (q_row >> 3)) & 3) : 0;
    const uint32_t k_from = q_row * kRowBytes + 16 * (q_piece ^ q_swz), v_from = q_row * kRowBytes + 16 * q_piece;
    const uint32_t to = (16 * wave + q_row) * kRowBytes + 16 * q_piece;
    const int s_lane = lane % (4 * GROUPS);                         // K scales, then V scales
    const uint32_t s_from = ((s_lane >> 2) << shift) + 4 * (s_lane & 3);
    const uint32_t s_to = (s_lane >> 2) * kTile + 16 * wave + 4 * (s_lane & 3);
    const int r0 = max(scalar_load(a.cu, b), 0), r1 = min(scalar_load(a.cu, b + 1), a.n_rows);
    const int n_new = r1 - r0, n_cols = n_new * a.G;
    const int len = min(max(scalar_load(a.len, b), 0), a.max_pages << shift);
    const int per = chunk_slabs_of(a, len);
    const int n_tiles = (n_cols + kCols - 1) / kCols;
    for (int turn = blockIdx.y; turn < n_tiles; turn += gridDim.y) {
        // the tiles with the most rows first, or, where all workgroups run at
        // once, two on a CU (the first half of the launch and then the
        // second), the second half with the fewest first
        const int half = (n_tiles + 1) / 2;
        const int tile = !a.fold || turn < half ? n_tiles - 1 - turn : turn - half;
        const int c0 = tile * kCols + wave * 16 * NT;               // the wavefront's first column
        const int end = min(len, len - n_new + min(column_row(a, tile * kCols + kCols - 1), n_new - 1) + 1);
        const int wave_first = len - n_new + min(column_row(a, c0), n_new - 1);
        const int j0 = chunk * per * kKv4Slab, j1 = end - j0 > per * kKv4Slab ? j0 + per * kKv4Slab : end;
        if (j0 >= end && chunk > 0) continue;

        int p_col[NT];
        bf16x8v qf[NT][STEPS];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int c = c0 + 16 * n + m;
            const bool live = c < n_cols;
            const int t = live ? column_row(a, c) : n_new - 1, h = live ? c - t * a.G : 0;
            p_col[n] = len - n_new + t;
            const char* qp = a.q + (int64_t)(r0 + t) * a.q_stride + ((int64_t)(g * a.G + h) * HD + r * (HD / 4)) * 2;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                u32x4v x = reinterpret_cast<const u32x4v*>(qp)[s];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = live ? x[i] ^ a.q_flip : 0;
                qf[n][s] = __builtin_bit_cast(bf16x8v, x);
            }
        }
        f32x4v acc[NT][CT], sum[NT];       // sum: of the weights, the same in every element
        // running maximum in units of scale_log2 > 0, what the weights subtract
        // (it, or 0 before the first), and the score past which it moves
        float mx[NT], base[NT], most[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            mx[n] = -INFINITY;
            base[n] = 0.f;
            most[n] = -INFINITY;
            sum[n] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < CT; ++i) acc[n][i] = f32x4v{0.f, 0.f, 0.f, 0.f};
        }

        // loads of the wavefront's quarter of the tile at row j, and its
        // storing in a slot; a quarter without a page reads page 0
        const int last_page = max(len - 1, 0) >> shift;
        auto fetch_id = [&](int j) {
            return scalar_load(a.table, (int64_t)b * a.max_pages + min((j + 16 * wave) >> shift, last_page));
        };
        u32x4v kw[2][2];
        uint2 ksw[2];
        u32x4v kq, vq;
        uint32_t sq;
        uint8_t on;
        int32_t page_q = -1;
        auto load = [&](int j, int32_t id) {
            // checked here, not where it is fetched: that would wait for it
            const int32_t page = page_q = kv4_page_or_none(d, id);
            const Kv4SlabBase qb = kv4_slab_base(d, page, g, j + 16 * wave, 0);
            if constexpr (HD == 128) {
                kq = *reinterpret_cast<const u32x4v*>(a.pool.k + qb.codes + k_from);
                vq = *reinterpret_cast<const u32x4v*>(a.pool.v + qb.codes + v_from);
            } else {
                kq = *reinterpret_cast<const u32x4v*>((lane < 32 ? a.pool.k : a.pool.v) + qb.codes + k_from);
            }
            sq = *reinterpret_cast<const uint32_t*>((lane < 4 * GROUPS ? a.pool.ks : a.pool.vs) + qb.scales + s_from);
            if constexpr (MASKED) {
                const int jm = j + lane;
                on = jm < end && jm < a.mask_stride ? a.mask[(int64_t)b * a.mask_stride + jm] : 0;
            }
        };
        uint64_t on_stored = 0;                             // execution map of the tile stored last
        auto store = [&](int slot) {
            if constexpr (HD == 128) {
                *reinterpret_cast<u32x4v*>(&s_k[slot][to]) = kq;
                *reinterpret_cast<u32x4v*>(&s_vr[slot][to]) = vq;
            } else {
                *reinterpret_cast<u32x4v*>(lane < 32 ? &s_k[slot][to] : &s_vr[slot][to]) = kq;
            }
            if (lane < 8 * GROUPS)
                *reinterpret_cast<uint32_t*>((lane < 4 * GROUPS ? &s_ks[slot][0][0] : &s_vs[slot][0][0]) + s_to) = sq;
            if (lane == 0) s_page[slot][wave] = page_q >= 0;
            if constexpr (MASKED) on_stored = __ballot(on != 0);
        };
        // the stored tile's keys and values of this lane
        auto read_keys = [&](int slot) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int row = 32 * s + 8 * (m >> 2) + (m & 3);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if constexpr (HD == 128) {
                        kw[s][u] = *reinterpret_cast<const u32x4v*>(
                            &s_k[slot][(row + 4 * u) * kRowBytes + 16 * (r ^ ((m >> 2) & 3))]);
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2*>(&s_k[slot][(row + 4 * u) * kRowBytes + 8 * r]);
                        kw[s][u][0] = x.x;
                        kw[s][u][1] = x.y;
                    }
                }
                ksw[s] = *reinterpret_cast<const uint2*>(&s_ks[slot][r * (HD / 4) / kKv4Group][32 * s + 8 * (m >> 2)]);
            }
        };
        // rows 8 (lane / 32) .. + 7 of the wavefront's quarter, columns CPT (lane % 32) ..
        ValueRows<HD> vr;
        const int rb = tid >> 5, vu = tid & 31;
        auto read_values = [&](int slot) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                vr.v[i] = *reinterpret_cast<const typename Bytes<HD / 64>::type*>(
                    &s_vr[slot][(8 * rb + i) * kRowBytes + vu * (HD / 64)]);
            vr.vs = *reinterpret_cast<const uint2*>(&s_vs[slot][vu * CPT / kKv4Group][8 * rb]);
        };
        // rows of the stored tile at row j that any column may see
        uint32_t alive[2], alive_next[2];
        auto pages_of = [&](int slot) { return *reinterpret_cast<const uint32_t*>(&s_page[slot][0]); };
        auto find_alive = [&](int j, uint32_t pages) {
            const uint32_t has = __builtin_amdgcn_readfirstlane(pages);
            alive_next[0] = alive_next[1] = 0xffffffffu;
            if (has != 0x01010101u || j + kTile > end) {
                asm volatile("; the last rows, or no page");
                alive_next[0] = kv4_slab_rows((has & 0xff) ? 0 : -1, (has & 0xff00) ? 0 : -1, j, end);
                alive_next[1] = kv4_slab_rows((has & 0xff0000) ? 0 : -1, (has >> 24) ? 0 : -1, j + 32, end);
            }
            if constexpr (MASKED) {
                alive_next[0] &= (uint32_t)on_stored;
                alive_next[1] &= (uint32_t)(on_stored >> 32);
            }
        };
        // their scales made finite where a row is left out or NaN, then the
        // values as the product's operands in a buffer
        auto fix_v = [&](int buf) {
            uint32_t vlo = vr.vs.x, vhi = vr.vs.y, nan8 = 0;
            // a scale of 255 somewhere in the wavefront (a byte of zero in the
            // complement), or rows left out
            const uint32_t zl = ~vlo, zh = ~vhi;
            const uint32_t hit = ((zl - 0x01010101u) & ~zl) | ((zh - 0x01010101u) & ~zh);
            if (__ballot((hit & 0x80808080u) != 0) != 0 || (alive_next[0] & alive_next[1]) != 0xffffffffu) {
                asm volatile("; rows left out or NaN");           // a branch, not selects
                const uint32_t rows8 = ((wave < 2 ? alive_next[0] : alive_next[1]) >> (8 * (rb & 3))) & 0xff;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    uint32_t& w8 = i < 4 ? vlo : vhi;
                    const int sh = 8 * (i & 3);
                    const bool out = !(rows8 >> i & 1), nan = ((w8 >> sh) & 0xff) == (uint32_t)kKv4NanScale;
                    if (!out && nan) nan8 |= 1u << i;
                    // both finite here: rows left out may hold anything, NaN
                    // rows are taken care of at the product
                    if (out || nan) w8 = (w8 & ~(0xffu << sh)) | 127u << sh;
                }
            }
            vr.vs = make_uint2(vlo, vhi);
            if (vu * CPT % kKv4Group == 0) s_nan[buf][vu * CPT / kKv4Group][rb] = (uint8_t)nan8;
        };
        // step 0 .. 2 CPT - 1 of storing: a pair of rows, two columns of each
        u32x4v even, odd;
        auto store_step = [&](int buf, int step) {
            const int byte = step / 4, i = step % 4;
            const uint32_t w = i < 2 ? vr.vs.x : vr.vs.y;           // scales of rows 2 i and 2 i + 1
            const float s0 = scale_at(w, 2 * (i & 1)), s1 = scale_at(w, 2 * (i & 1) + 1);
            const uint32_t x0 = cvt_bf16(vr.v[2 * i], s0, byte), x1 = cvt_bf16(vr.v[2 * i + 1], s1, byte);
            even[i] = __builtin_amdgcn_perm(x1, x0, 0x05040100u);
            odd[i] = __builtin_amdgcn_perm(x1, x0, 0x07060302u);
            if (i == 3) {
                // column CPT vu + t in tile 2 t + vu / 16, lane vu % 16
                s_v[buf][rb >> 2][4 * byte + (vu >> 4)][(rb & 3) * 16 + (vu & 15)] = even;
                s_v[buf][rb >> 2][4 * byte + 2 + (vu >> 4)][(rb & 3) * 16 + (vu & 15)] = odd;
            }
        };

        // Tile x (counted from j0) is loaded during tile x - 3, stored in slot
        // x % 4 during tile x - 2, its values converted during tile x - 1.
        int32_t id = -1;
        if (j0 < j1) {
            load(j0, fetch_id(j0));
            store(0);
            load(j0 + kTile, fetch_id(j0 + kTile));
            __syncthreads();
            read_values(0);
            find_alive(j0, pages_of(0));
            fix_v(0);
#pragma unroll
            for (int k = 0; k < 2 * CPT; ++k) store_step(0, k);
            store(1);
            load(j0 + 2 * kTile, fetch_id(j0 + 2 * kTile));
            id = fetch_id(j0 + 3 * kTile);
        }
        __syncthreads();
        const float inv_scale = 1.f / a.scale_log2;
        const u32x4v ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        int buf = 0, slot = 0;
        for (int j = j0; j < j1; j += kTile, buf ^= 1, slot = (slot + 1) % kSlots) {
            alive[0] = alive_next[0];
            alive[1] = alive_next[1];
            // Two slabs, staggered so that each product has vector work of the
            // other slab beside it: scores of the second beside the weights of
            // the first, the first's product beside the weights of the second
            // (and then the next tile's values).
            float sc[2][NT][8];
            uint32_t seen[2][NT];
            bf16x8v pf[2][NT];
            f32x4v dd[2][NT];
            float ks[2];
            // step 0 .. 2 STEPS - 1 of a slab's scores: four words of 8 rows'
            // half against every column tile; their conversion a step ahead
            // (a product that follows it at once waits a cycle)
            u32x4v kf_next;
            auto key_step = [&](int sl, int step) {
                const int st = step / 2, u = step % 2;
                if (st == 0) ks[u] = scale_turned(u ? ksw[sl].y : ksw[sl].x, m & 3);
#pragma unroll
                for (int i = 0; i < 4; ++i) kf_next[i] = cvt_bf16(kw[sl][u][st], ks[u], i);
            };
            auto score_step = [&](int sl, int step) {
                const int st = step / 2, u = step % 2;
                if (st == 0) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) dd[u][n] = f32x4v{0.f, 0.f, 0.f, 0.f};
                }
                const u32x4v kf = kf_next;
                if (step + 1 < 2 * STEPS) key_step(sl, step + 1);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    dd[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, kf), qf[n][st],
                                                                      dd[u][n], 0, 0, 0);
                if (st == STEPS - 1)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[sl][n][4 * u + e] = dd[u][n][e];
            };
            // masks the scores and moves the maxima (in units of scale_log2 > 0)
            // where they grow
            auto settle = [&](int sl) {
                const int js = j + 32 * sl;
#pragma unroll
                for (int n = 0; n < NT; ++n) seen[sl][n] = 0xff;
                if (!(alive[sl] == 0xffffffffu && js + kKv4Slab - 1 <= wave_first)) {
                    asm volatile("; some rows left out");
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const int upto = min(max(p_col[n] - (js + 8 * r) + 1, 0), 8);
                        seen[sl][n] = (alive[sl] >> (8 * r)) & ((1u << upto) - 1);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (!(seen[sl][n] >> i & 1)) sc[sl][n][i] = -INFINITY;
                    }
                }
                float top[NT];
                bool grow = false;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    top[n] = sc[sl][n][0];
#pragma unroll
                    for (int i = 1; i < 8; ++i) top[n] = max_nan(top[n], sc[sl][n][i]);
                    grow = grow || top[n] > most[n];
                }
                if (__ballot(grow) != 0) {
                    asm volatile("; the maximum grows");
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        // rounded up to a whole number: its moves scale what is
                        // there by powers of two, bf16 weights exactly
                        const float t = fmaxf(mx[n], __builtin_ceilf(kv4_max32(kv4_max16(top[n])) * a.scale_log2));
                        base[n] = t == -INFINITY ? 0.f : t;
                        const float al = power_of_two(mx[n] - base[n]);
                        sum[n] *= al;
#pragma unroll
                        for (int i = 0; i < CT; ++i) acc[n][i] *= al;
                        // the first slab's weights wait for the product
                        if (sl == 1) {
                            u32x4v w = __builtin_bit_cast(u32x4v, pf[0][n]);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                w[i] = pack_bf16x2(__uint_as_float(w[i] << 16) * al,
                                                   __uint_as_float(w[i] & 0xffff0000u) * al);
                            pf[0][n] = __builtin_bit_cast(bf16x8v, w);
                        }
                        mx[n] = t;
                        most[n] = (t + 8.f) * inv_scale;
                    }
                }
            };
            // step 0 .. 4 NT - 1: two weights of a slab
            auto weight_step = [&](int sl, int step) {
                const int n = step / 4, i = step % 4;
                u32x4v w = __builtin_bit_cast(u32x4v, pf[sl][n]);
                uint32_t two = pack_bf16x2(exp2_hw(fmaf(sc[sl][n][2 * i], a.scale_log2, -base[n])),
                                           exp2_hw(fmaf(sc[sl][n][2 * i + 1], a.scale_log2, -base[n])));
                asm volatile("" : "+v"(two));                      // here, not at its use
                w[i] = two;
                pf[sl][n] = __builtin_bit_cast(bf16x8v, w);
            };
            const bool more = j + kTile < j1;
            read_keys(slot);
            read_values((slot + 1) % kSlots);
            // read here, where nothing waits for them
            const uint32_t pages = pages_of((slot + 1) % kSlots);
            const uint32_t nan_word = reinterpret_cast<const uint32_t*>(&s_nan[buf][0][0])[lane % (2 * GROUPS)];
            key_step(0, 0);
#pragma unroll
            for (int k = 0; k < 2 * STEPS; ++k) score_step(0, k);
            key_step(1, 0);
            settle(0);
#pragma unroll
            for (int n = 0; n < NT; ++n) pf[0][n] = pf[1][n] = __builtin_bit_cast(bf16x8v, u32x4v{0, 0, 0, 0});
            // Fixed order from here: each step's products start while the
            // vector work behind them issues.
#pragma unroll
            for (int k = 0; k < 2 * STEPS; ++k) {
                score_step(1, k);
#pragma unroll
                for (int i = 0; i < 2 * NT / STEPS; ++i) weight_step(0, k * (2 * NT / STEPS) + i);
                __builtin_amdgcn_sched_barrier(0);
            }
            settle(1);
            u32x4v vf[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) vf[k] = s_v[buf][k / CT][k % CT][lane];
            if (__ballot(nan_word != 0) != 0) {
                // NaN rows count for the columns that see them: (rows a group
                // has) x (rows a column sees)
                asm volatile("; NaN rows");
#pragma unroll
                for (int sl = 0; sl < 2; ++sl) {
                    u32x4v ind[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                   // column tiles of even and odd number
                        const uint32_t bits = s_nan[buf][CPT * (m + 16 * h) / kKv4Group][4 * sl + r];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            ind[h][i] = (bits >> (2 * i) & 1 ? 0x3f80u : 0u) | (bits >> (2 * i + 1) & 1 ? 0x3f800000u : 0u);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        u32x4v vis;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            vis[i] = (seen[sl][n] >> (2 * i) & 1 ? 0x3f80u : 0u) |
                                     (seen[sl][n] >> (2 * i + 1) & 1 ? 0x3f800000u : 0u);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            f32x4v cnt = {0.f, 0.f, 0.f, 0.f};
                            cnt = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, ind[h]),
                                                                          __builtin_bit_cast(bf16x8v, vis), cnt, 0, 0, 0);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (cnt[e] > 0.f)
#pragma unroll
                                    for (int i = h; i < CT; i += 2) acc[n][i][e] = NAN;
                        }
                    }
                }
            }
            if (more) {
                find_alive(j + kTile, pages);
                fix_v(buf ^ 1);
            }
            store((slot + 2) % kSlots);
            load(j + 3 * kTile, id);
            id = fetch_id(j + 4 * kTile);
            // the products with V, operands read four ahead; beside the first
            // slab's the second's weights, beside the second's the conversion
            // of the next tile's values (after the last tile: into the buffer
            // that nobody reads again)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < 2 * CT; ++k) {
                const bf16x8v v = __builtin_bit_cast(bf16x8v, vf[k % 4]);
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    acc[n][k % CT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[k / CT][n], acc[n][k % CT], 0, 0, 0);
                if (k + 4 < 2 * CT) vf[k % 4] = s_v[buf][(k + 4) / CT][(k + 4) % CT][lane];
                if (k < CT) {
#pragma unroll
                    for (int i = 0; i < 4 * NT / CT; ++i) weight_step(1, k * (4 * NT / CT) + i);
                } else {
                    store_step(buf ^ 1, k - CT);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int sl = 0; sl < 2; ++sl)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    sum[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8v, ones), pf[sl][n],
                                                                    sum[n], 0, 0, 0);
            __syncthreads();
        }

#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int c = c0 + 16 * n + m;
            const float L = sum[n][0];
            if (c >= n_cols) continue;
            const int t = column_row(a, c), head = g * a.G + c - t * a.G;
            const int64_t row = r0 + t;
            const float inv = a.chunks > 1 ? 1.f : L == 0.f ? 0.f : 1.f / L;
            // element CPT (4 r + e + 16 (i % 2)) + i / 2 is acc[i][e]
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float y[4 * CPT];
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int t2 = 0; t2 < CPT; ++t2) y[CPT * e + t2] = acc[n][2 * t2 + h][e] * inv;
                const int col = CPT * (4 * r + 16 * h);
                if (a.chunks == 1) {
                    char* op = a.out + row * a.out_stride + ((int64_t)head * HD + col) * 2;
#pragma unroll
                    for (int x = 0; x < 4 * CPT; x += 8)
                        *reinterpret_cast<uint4*>(op + 2 * x) = make_uint4(
                            f2bf(y[x]) | (uint32_t)f2bf(y[x + 1]) << 16, f2bf(y[x + 2]) | (uint32_t)f2bf(y[x + 3]) << 16,
                            f2bf(y[x + 4]) | (uint32_t)f2bf(y[x + 5]) << 16,
                            f2bf(y[x + 6]) | (uint32_t)f2bf(y[x + 7]) << 16);
                } else {
                    const int64_t at = (row * a.nq + head) * a.chunks + chunk;
#pragma unroll
                    for (int x = 0; x < 4 * CPT; x += 4)
                        *reinterpret_cast<float4*>(a.part_o + at * HD + col + x) =
                            make_float4(y[x], y[x + 1], y[x + 2], y[x + 3]);
                    if (r == 0 && h == 0) a.part_ml[at] = make_float2(mx[n], L);
                }
            }
        }
    }
}

// Joins the chunks of a (row, head): W wavefronts on one, HD / 4 lanes to a
// chunk's sums and the other lanes to the next chunks.  A row has the chunks
// that start at or before its position.  Four wavefronts where there are few
// (latency: 32 of 8 chunks 2.4 us, 3.9 with one wavefront each), one where
// there are many (2300 rows of 32 heads in two chunks took 95 us with four).
template <typename T, int HD, int W>
__global__ __launch_bounds__(256) void kv4_join_kernel(Kv4AttnArgs a) {
    constexpr int LPC = HD / 4, AT = 64 * W / LPC;    // lanes per chunk, chunks at a time
    constexpr int EARLY = W > 1 ? 2 : 1;
    __shared__ float s_f[4 / W][kKv4MaxChunks];
    __shared__ float s_red[4], s_l[4];
    __shared__ __attribute__((aligned(16))) float4 s_a[4][64];
    const int tid = threadIdx.x, wave = tid >> 6;
    const int unit = wave / W, t = tid % (64 * W);    // this (row, head) of the workgroup's, lane in it
    const int head = min((int)blockIdx.x * (4 / W) + unit, a.nq - 1);
    for (int row = blockIdx.y; row < a.n_rows; row += gridDim.y) {
        // partials are read while the row's sequence and length are looked up;
        // those of chunks that the row does not have are dropped
        const int64_t at = ((int64_t)row * a.nq + head) * a.chunks;
        const int lc = t % LPC, c0 = t / LPC;
        auto sums = [&](int ch) { return *reinterpret_cast<const float4*>(a.part_o + (at + ch) * HD + 4 * lc); };
        float2 ml = a.part_ml[at + min(t, a.chunks - 1)];
        float4 early[EARLY];
#pragma unroll
        for (int i = 0; i < EARLY; ++i) early[i] = sums(min(c0 + i * AT, a.chunks - 1));
        // the row's sequence: the last that starts at or before it
        if (row < scalar_load(a.cu, 0) || row >= scalar_load(a.cu, a.B)) continue;
        int lo = 0, hi = a.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (scalar_load(a.cu, mid) <= row) lo = mid; else hi = mid - 1;
        }
        const int len = min(max(scalar_load(a.len, lo), 0), a.max_pages << a.pool.d.page_shift);
        const int p = len - (min(scalar_load(a.cu, lo + 1), a.n_rows) - row);
        // the chunks that start at or before the row's position
        const uint32_t step = chunk_slabs_of(a, len) * kKv4Slab;
        auto has = [&](int ch) { return ch < a.chunks && (ch == 0 || (p >= 0 && ch * step <= (uint32_t)p)); };
        if (!has(t)) ml = make_float2(-INFINITY, 0.f);
        float M = wave_max(ml.x), L;
        if constexpr (W > 1) {
            if ((tid & 63) == 0) s_red[wave] = M;
            __syncthreads();
            M = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
        }
        const float f = exp2_hw(ml.x - (M == -INFINITY ? 0.f : M));
        s_f[unit][t] = f;
        L = wave_sum(ml.y * f);
        if constexpr (W > 1) {
            if ((tid & 63) == 0) s_l[wave] = L;
        }
        __syncthreads();
        if constexpr (W > 1) L = (s_l[0] + s_l[1]) + (s_l[2] + s_l[3]);
        float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float4& o, int ch) {
            const float w = s_f[unit][ch];
            A.x += o.x * w; A.y += o.y * w; A.z += o.z * w; A.w += o.w * w;
        };
#pragma unroll
        for (int i = 0; i < EARLY; ++i)
            if (has(c0 + i * AT)) add(early[i], c0 + i * AT);
        if (a.chunks > EARLY * AT) {
            const int n = p < 0 ? 1 : (int)min((uint32_t)p / step + 1, (uint32_t)a.chunks);
#pragma unroll 4
            for (int ch = c0 + EARLY * AT; ch < n; ch += AT) add(sums(ch), ch);
        }
        s_a[wave][tid & 63] = A;
        __syncthreads();
        if (t < LPC) {
#pragma unroll
            for (int i = 1; i < AT; ++i) {
                const float4 o = (&s_a[unit * W][0])[i * LPC + t];
                A.x += o.x; A.y += o.y; A.z += o.z; A.w += o.w;
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            float y[4] = {A.x * inv, A.y * inv, A.z * inv, A.w * inv};
            char* op = a.out + row * a.out_stride + ((int64_t)head * HD + 4 * t) * sizeof(T);
            if (blockIdx.x * (4 / W) + unit < a.nq) {
                if constexpr (sizeof(T) == 2)
                    *reinterpret_cast<uint2*>(op) =
                        make_uint2(f2bf(y[0]) | (uint32_t)f2bf(y[1]) << 16, f2bf(y[2]) | (uint32_t)f2bf(y[3]) << 16);
                else
                    *reinterpret_cast<float4*>(op) = make_float4(y[0], y[1], y[2], y[3]);
            }
        }
        __syncthreads();
    }
}

namespace {

// How a call is split: the form, its column tiles and its chunks.
struct Kv4Split {
    int nt;                              // prompt form: column tiles of 16 a wavefront; 0: decode form
    int tiles, chunks, chunk_slabs, chunk_unit;
};

// Partial sums (of a row, a head and a chunk) that a call may make: the output
// rows of two rounds of the prompt form's workgroups, of ten of the decode
// form's.  Calls of more rows and heads take fewer chunks than would be
// fastest, so that one workspace of 68 MB (heads of 128) is enough for any.
constexpr int64_t kMaxPartials = 1 << 17;

constexpr int kPromptTiles = 2;          // column tiles of 16 a wavefront of the prompt form
constexpr int kPromptMinCols = 64;       // fewer columns: always the decode form

int slabs_of(const buddy_kv4_attn& a) {
    const int max_len = a.max_len < INT32_MAX - 1024 ? a.max_len : INT32_MAX - 1024;   // no sequence has more
    return (max_len + kKv4Slab - 1) / kKv4Slab;
}

// Both forms can take any call.  Which is faster, and in how many chunks,
// follows from estimated times in us, of constants measured with eight KV
// heads of 128: the prompt form takes 1.4 a tile of 64 rows with a workgroup
// alone on its CU, 2.0 for two; the decode form 0.73 a slab of a wavefront
// with one workgroup on a CU, 1.0 with two, 1.5 with three; either 6 around
// that, and chunks their partial sums (written and read at about 4 TB/s) and
// another launch.
// Measured, us, prompt form and decode form, each in its best number of
// chunks: 1000 rows among 8000 (32 heads) 153 in 2 and 236; 1024 among as many
// 30 and 32; 64 among 4000 24 in 16 and 20 in 4; 20 among 4000 18 in 16 and 14
// in 4; 100 among 16000 56 in 16 and 72 in 8; 200 of 40 heads alone among 1024
// 25 in 2 and 19; four times 300 of 28 among 2000 71 and 77; three of up to
// 1024 among up to 5000 163 and 272.
Kv4Split split_rows(const Kv4Pool& pool, int G, const buddy_kv4_attn& a, int B, bool prompt) {
    Kv4Split s;
    const int64_t cols = (int64_t)(a.max_rows < a.n_rows ? a.max_rows : a.n_rows) * G;
    const int slabs = slabs_of(a);
    const int64_t limit = kMaxPartials / ((int64_t)a.n_rows * a.n_heads);
    const double wide = (pool.d.hd + 64) / 192.0;
    auto join_us = [&](int64_t c) { return c > 1 ? 4 + 2.3e-6 * a.n_rows * a.n_heads * c * (pool.d.hd + 2) : 0.0; };
    // column tiles of `tile` columns that the launch has and that hold rows
    auto tiles_of = [&](int tile, int64_t* busy) {
        const int64_t t = cols < (int64_t)tile * 65535 ? (cols + tile - 1) / tile : 65535;
        const int64_t full = ((int64_t)a.n_rows * G + tile - 1) / tile + B;
        *busy = (B * t < full ? B * t : full) * pool.d.n_kv;
        return (int)t;
    };
    int64_t busy;
    s.nt = 0;
    s.tiles = tiles_of(16, &busy);
    s.chunk_unit = 4;
    if (busy < 1) busy = 1;
    // as many chunks as run at once (three workgroups a CU with bf16 queries,
    // two with fp32), of two slabs a wavefront at least, or of one while that
    // leaves CUs without a workgroup (chunks of one slab a wavefront: 2048 rows
    // of 8 heads 2 % shorter, 16 sequences of up to 1000 rows 4 % longer)
    int64_t want = (prompt ? 768 : 512) / busy, most = 256 / busy;
    if (most > (slabs + 3) / 4) most = (slabs + 3) / 4;
    if (most < (slabs + 7) / 8) most = (slabs + 7) / 8;
    if (want > most) want = most;
    if (want > kKv4MaxChunks) want = kKv4MaxChunks;
    if (want > limit) want = limit;
    if (want < 1) want = 1;
    if (prompt && cols > kPromptMinCols) {
        // rounds of as many workgroups as run at once, and what is left over:
        // half as if all took the same time, half as if uneven ones filled gaps
        auto rounds_us = [](int64_t wgs, int64_t at_once, double full, double two, double one) {
            const int64_t rounds = wgs / at_once, rest = wgs % at_once;
            const double step = full * rounds + (rest > 512 ? full : rest > 256 ? two : rest > 0 ? one : 0.0);
            return rounds ? (step + full * wgs / at_once) / 2 : step;
        };
        double best = 6 + wide * rounds_us(busy * want, 768, 1.5, 1.0, 0.73) * slabs / (4 * want) + join_us(want);
        int64_t wgs;
        const int tiles = tiles_of(64 * kPromptTiles, &wgs);
        for (int64_t c = 1; c <= kKv4MaxChunks && (c == 1 || (4 * c <= slabs && c <= limit)); c += (c + 3) / 4) {
            const double us = 6 + wide * rounds_us(wgs * c, 512, 2.0, 2.0, 1.4) * (slabs / 2.0 / c) + join_us(c);
            if (us >= best) continue;
            best = us;
            want = c;
            s.nt = kPromptTiles;
        }
        if (s.nt) {
            s.tiles = tiles;
            s.chunk_unit = 2;
        }
    }
    const int per = (int)((slabs + want - 1) / want);
    s.chunk_slabs = per < s.chunk_unit ? s.chunk_unit : (per + s.chunk_unit - 1) / s.chunk_unit * s.chunk_unit;
    s.chunks = (slabs + s.chunk_slabs - 1) / s.chunk_slabs;
    if (s.chunks < 1) s.chunks = 1;
    return s;
}

buddy_status check_attn(const buddy_kv4* cache, const buddy_kv4_attn* a, int32_t B, Kv4Pool* pool) {
    const buddy_status st = kv4_check_pool(cache, pool);
    if (st != BUDDY_OK) return st;
    if (!a || B < 0) return BUDDY_EINVAL;
    if (a->dtype != BUDDY_F32 && a->dtype != BUDDY_BF16) return BUDDY_EINVAL;
    if (a->n_heads < 1 || a->n_heads % cache->n_kv_heads || a->n_heads / cache->n_kv_heads > 16) return BUDDY_ESHAPE;
    if (a->n_rows < 0 || a->max_rows < 0 || a->max_len < 0) return BUDDY_EINVAL;
    if (B > kKv4MaxSeqs) return BUDDY_ECAPACITY;
    // 24 bits of columns and rows: products with 16 heads stay in 31
    if (a->n_rows > (1 << 24) || a->max_rows > (1 << 24)) return BUDDY_ECAPACITY;
    return BUDDY_OK;
}

// Room for the partials of every call of as many rows and as long sequences or
// fewer: chunks of four slabs at least in either form, whatever the batch.
// (Those of the call alone are not monotone: few sequences are split, many are
// not.)
size_t workspace_bytes(const Kv4Pool& pool, const buddy_kv4_attn& a) {
    int64_t chunks = (slabs_of(a) + 3) / 4;
    if (chunks > kKv4MaxChunks) chunks = kKv4MaxChunks;
    if (chunks <= 1) return 16;
    int64_t partials = (int64_t)a.n_rows * a.n_heads * chunks;
    if (partials > kMaxPartials) partials = kMaxPartials;
    return (size_t)partials * (pool.d.hd + 2) * sizeof(float);
}

template <typename T, int HD>
hipError_t launch_attn(const Kv4AttnArgs& a, int nt, hipStream_t s) {
    const dim3 wg(256);
    if (nt) {
        if constexpr (sizeof(T) == 2) {
            const dim3 grid(a.pool.d.n_kv * a.chunks, a.tiles, a.B);
            if (a.mask) hipLaunchKernelGGL((kv4_prompt_kernel<HD, kPromptTiles, true>), grid, wg, 0, s, a);
            else hipLaunchKernelGGL((kv4_prompt_kernel<HD, kPromptTiles, false>), grid, wg, 0, s, a);
        }
    } else {
        const int64_t z = (int64_t)a.B * a.tiles;
        const dim3 grid(a.chunks, a.pool.d.n_kv, (unsigned)(z < 65535 ? z : 65535));
        if (a.mask) hipLaunchKernelGGL((kv4_decode_kernel<T, HD, true>), grid, wg, 0, s, a);
        else hipLaunchKernelGGL((kv4_decode_kernel<T, HD, false>), grid, wg, 0, s, a);
    }
    if (a.chunks > 1) {
        const int rows = a.n_rows < 65535 ? a.n_rows : 65535;
        if (a.chunks > 8 || (int64_t)a.n_rows * a.nq <= 4096)
            hipLaunchKernelGGL((kv4_join_kernel<T, HD, 4>), dim3(a.nq, rows), wg, 0, s, a);
        else
            hipLaunchKernelGGL((kv4_join_kernel<T, HD, 1>), dim3((a.nq + 3) / 4, rows), wg, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace
}  // namespace buddy

using namespace buddy;

extern "C" {

size_t buddy_kv4_attention_workspace(const buddy_kv4* cache, const buddy_kv4_attn* a, int32_t B) {
    Kv4Pool pool;
    if (check_attn(cache, a, B, &pool) != BUDDY_OK) return 0;
    if (B == 0 || a->n_rows == 0 || a->max_rows == 0) return 16;
    return workspace_bytes(pool, *a);
}

buddy_status buddy_kv4_attention_form(const buddy_kv4* cache, const buddy_kv4_attn* a, int32_t B, int32_t* weight_parts,
                                      int32_t* chunks) {
    Kv4Pool pool;
    const buddy_status st = check_attn(cache, a, B, &pool);
    if (st != BUDDY_OK) return st;
    const bool bf16 = a->dtype == BUDDY_BF16;
    Kv4Split sp;
    sp.nt = 0; sp.chunks = 1;
    if (B > 0 && a->n_rows > 0 && a->max_rows > 0) sp = split_rows(pool, a->n_heads / pool.d.n_kv, *a, B, bf16);
    if (weight_parts) *weight_parts = sp.nt ? 1 : bf16 ? 2 : 3;
    if (chunks) *chunks = sp.chunks;
    return BUDDY_OK;
}

buddy_status buddy_kv4_attention(const buddy_kv4* cache, const buddy_kv4_attn* a, int32_t B, void* stream) {
    Kv4AttnArgs k;
    const buddy_status st = check_attn(cache, a, B, &k.pool);
    if (st != BUDDY_OK) return st;
    if (B == 0 || a->n_rows == 0) return BUDDY_OK;
    const int hd = cache->head_dim, size = a->dtype == BUDDY_BF16 ? 2 : 4;
    const int64_t width = (int64_t)a->n_heads * hd, most = INT64_MAX / 64 / a->n_rows;
    if (!a->q || !a->out || !a->table || !a->len || !a->cu_rows || !aligned16(a->q) || !aligned16(a->out)) return BUDDY_EINVAL;
    if ((a->n_rows > 1 && (a->q_stride < width || a->out_stride < width)) || a->q_stride < 0 || a->out_stride < 0 ||
        a->q_stride > most || a->out_stride > most || a->q_stride * size % 16 || a->out_stride * size % 16)
        return BUDDY_EINVAL;
    // a scale's inverse and its product with log2(e) stay normal fp32 numbers
    if (a->max_rows < 1 || a->max_pages < 1 || !(fabsf(a->scale) >= 1e-30f && fabsf(a->scale) <= 1e30f)) return BUDDY_EINVAL;
    if ((int64_t)a->max_pages * cache->page_rows > INT32_MAX - 1024) return BUDDY_ECAPACITY;
    if (a->mask && a->mask_stride < a->max_len) return BUDDY_EINVAL;
    k.B = B; k.nq = a->n_heads; k.G = a->n_heads / cache->n_kv_heads;
    k.inv_G = inverse_of(k.G);
    k.inv_B = inverse_of(B);
    const Kv4Split sp = split_rows(k.pool, k.G, *a, B, a->dtype == BUDDY_BF16);
    k.fold = (int64_t)B * sp.tiles * sp.chunks * k.pool.d.n_kv <= 512;
    k.inv_chunks = inverse_of(sp.chunks);
    k.tiles = sp.tiles; k.chunks = sp.chunks; k.chunk_slabs = sp.chunk_slabs; k.chunk_unit = sp.chunk_unit;
    if (!a->workspace || !aligned16(a->workspace) || a->workspace_bytes < workspace_bytes(k.pool, *a))
        return BUDDY_EINVAL;
    k.q = (const char*)a->q; k.q_stride = a->q_stride * size;
    k.out = (char*)a->out; k.out_stride = a->out_stride * size;
    k.table = a->table; k.len = a->len; k.cu = a->cu_rows;
    k.mask = a->mask; k.mask_stride = a->mask_stride;
    k.n_rows = a->n_rows; k.max_pages = a->max_pages;
    // a negative scale turns the queries' signs
    k.scale_log2 = (float)(fabs((double)a->scale) * 1.4426950408889634);
    k.q_flip = a->scale < 0 ? (a->dtype == BUDDY_BF16 ? 0x80008000u : 0x80000000u) : 0;
    k.part_o = (float*)a->workspace;
    k.part_ml = (float2*)(k.part_o + (size_t)a->n_rows * a->n_heads * k.chunks * hd);
    hipStream_t s = (hipStream_t)stream;
    hipError_t e;
    if (a->dtype == BUDDY_BF16) e = hd == 128 ? launch_attn<bf16_t, 128>(k, sp.nt, s) : launch_attn<bf16_t, 64>(k, sp.nt, s);
    else e = hd == 128 ? launch_attn<float, 128>(k, 0, s) : launch_attn<float, 64>(k, 0, s);
    return e == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

}  // extern "C"
