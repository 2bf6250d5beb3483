// Serving from a paged 4-bit KV cache: page planning, per-head RMSNorm with
// rotary embedding, cache writes and reads, with their C ABI.  The attention
// over the cache is in kv4_attn.hip.
#include <math.h>
#include <string.h>

#include "kv4.h"

namespace buddy {

// ------------------------------------------------------------ page planning
//
// A pool's free pages are a ring: state[1] entries from entry state[0] on.
// Requests are threads of a workgroup (prefix sums of at most 1024 numbers
// each), and the pages and rows that the sums lay out are then shared by all
// threads, each finding the request of its entry by bisection.  Bound: latency
// (a launch, two or three dependent reads): 256 requests of one row 3.6 us,
// their release 2.7.

// Sums are capped here: both limits they are compared with (free pages, at
// most 2^27, and row entries) are below, and capped sums stay associative.
constexpr uint32_t kPlanCap = 1u << 30;

__device__ __forceinline__ uint32_t cap_add(uint32_t a, uint32_t b) { return min(a + b, kPlanCap); }

// A value from another lane by DPP, 0 where the row mask or the row's end
// leaves a lane out.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_0(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
// Inclusive prefix sum over a wavefront: rows of 16 by shifts of 1, 2, 4 and
// 8, then each row's last lane to the next row and lane 31 to the upper half.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    x = cap_add(x, dpp_or_0<0x111, 0xf>(x));
    x = cap_add(x, dpp_or_0<0x112, 0xf>(x));
    x = cap_add(x, dpp_or_0<0x114, 0xf>(x));
    x = cap_add(x, dpp_or_0<0x118, 0xf>(x));
    x = cap_add(x, dpp_or_0<0x142, 0xa>(x));
    return cap_add(x, dpp_or_0<0x143, 0xc>(x));
}

// Inclusive prefix sums of two numbers over the workgroup; s_w: 32 entries of
// this call's own.
__device__ __forceinline__ void wg_scan2(uint32_t& x, uint32_t& y, uint32_t* s_w) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x = wave_scan(x);
    y = wave_scan(y);
    if (lane == kWave - 1) { s_w[wave] = x; s_w[16 + wave] = y; }
    __syncthreads();
    uint32_t bx = 0, by = 0;
    for (int w = 0; w < wave; ++w) { bx = cap_add(bx, s_w[w]); by = cap_add(by, s_w[16 + w]); }
    x = cap_add(x, bx);
    y = cap_add(y, by);
}

// The request of entry e: the last whose range [ends[b - 1], ends[b]) starts
// at or before it (ends: inclusive sums of n requests, e < ends[n - 1]).
__device__ __forceinline__ int find_request(const int32_t* ends, int n, int e) {
    int lo = 0, hi = n - 1;              // the first b with ends[b] > e
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > e) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// First entry and number of the free pages, within the ring whatever is there.
__device__ __forceinline__ void ring_state(const int32_t* state, int n, int& head, int& count) {
    head = state[0];
    if ((uint32_t)head >= (uint32_t)n) {
        head %= n;
        if (head < 0) head += n;
    }
    count = min(max(state[1], 0), n);
}
// Entry x of the ring, x below twice its n (at most 2^27) entries.
__device__ __forceinline__ int ring_entry(int x, int n) { return x >= n ? x - n : x; }

struct PlanArgs {
    const int32_t *len, *n_new;
    int32_t B, shift, max_pages, n_pages, n_rows;
    int32_t* table;
    const int32_t* ring;
    const int32_t* state;
    int32_t *state_out, *len_out, *cu, *pos, *slots;
    uint8_t* refused;
    int32_t write, map;                  // which part this launch does
};

// Every workgroup lays out all requests (a few hundred numbers), the first
// writes what they get, and each maps its part of the rows: a row's page is
// the table's or, if the call adds it, still the ring's, so that no workgroup
// waits for another's writes.  Where lengths or state are written in place,
// many rows are mapped by a launch before the one that writes (39900 rows of
// 48 requests: one launch 5.7 us; two, with the rows mapped behind, 8.5).
__global__ __launch_bounds__(1024) void plan_kernel(PlanArgs a) {
    __shared__ uint32_t s_w[2][32];
    __shared__ int32_t s_rows[kKv4MaxSeqs], s_after[kKv4MaxSeqs], s_pages[kKv4MaxSeqs], s_held[kKv4MaxSeqs];
    const int b = threadIdx.x;
    int head, count;
    ring_state(a.state, a.n_pages, head, count);
    int len = 0, fresh = 0;
    bool valid = true;
    if (b < a.B) {
        len = a.len[b];
        fresh = a.n_new[b];
        valid = len >= 0 && fresh >= 0 && (int64_t)len + fresh <= ((int64_t)a.max_pages << a.shift);
    }
    const int round = (1 << a.shift) - 1;
    const int held = valid ? (int)(((int64_t)len + round) >> a.shift) : 0;
    const uint32_t need = valid ? (uint32_t)(((int64_t)len + fresh + round) >> a.shift) - held : 0;
    // A request is served if all pages and rows asked for up to it fit,
    // refused requests' included: those that need pages and are served are
    // then the first of the batch that need any.
    uint32_t pages = need, rows = valid ? (uint32_t)min(fresh, (int)kPlanCap) : 0;
    wg_scan2(pages, rows, s_w[0]);
    const int why = !valid ? 1 : need > 0 && pages > (uint32_t)count ? 2
                    : fresh > 0 && rows > (uint32_t)a.n_rows ? 3 : 0;
    if (__syncthreads_or(why)) {
        pages = why ? 0 : need;
        rows = why ? 0 : (uint32_t)fresh;
        wg_scan2(pages, rows, s_w[1]);
    }
    if (b < a.B) {
        const int after = why ? max(len, 0) : len + fresh;
        s_rows[b] = (int32_t)rows;
        s_after[b] = after;
        s_pages[b] = (int32_t)pages;
        s_held[b] = held;
        if (a.write && blockIdx.x == 0) {
            a.cu[b + 1] = (int32_t)rows;
            a.len_out[b] = after;
            a.refused[b] = (uint8_t)why;
            if (b == 0) a.cu[0] = 0;
            if (b == a.B - 1) {
                a.state_out[0] = ring_entry(head + (int)pages, a.n_pages);
                a.state_out[1] = count - (int32_t)pages;
            }
        }
    }
    __syncthreads();
    auto ring_page = [&](int e) { return a.ring[ring_entry(head + e, a.n_pages)]; };
    if (a.write && blockIdx.x == 0)
        for (int e = b; e < s_pages[a.B - 1]; e += blockDim.x) {
            const int q = find_request(s_pages, a.B, e);
            const int first = q ? s_pages[q - 1] : 0;
            a.table[(size_t)q * a.max_pages + s_held[q] + e - first] = ring_page(e);
        }
    // positions and slots, -1 behind the last request's rows
    for (int r = blockIdx.x * blockDim.x + b; a.map && r < a.n_rows; r += gridDim.x * blockDim.x) {
        int p = -1, slot = -1;
        if (r < s_rows[a.B - 1]) {
            const int q = find_request(s_rows, a.B, r);
            p = s_after[q] - (s_rows[q] - r);
            const int i = p >> a.shift;
            const int page = i < s_held[q] ? a.table[(size_t)q * a.max_pages + i]
                                           : ring_page((q ? s_pages[q - 1] : 0) + i - s_held[q]);
            // an entry that the pool does not have (a damaged table) maps nowhere
            if (page >= 0 && page < a.n_pages) slot = (page << a.shift) | (p & round);
        }
        a.pos[r] = p;
        a.slots[r] = slot;
    }
}

struct ReleaseArgs {
    const int32_t* len;
    const uint8_t* done;
    int32_t B, shift, max_pages, n_pages;
    const int32_t* table;
    int32_t* ring;
    const int32_t* state;
    int32_t *state_out, *len_out;
};

__global__ __launch_bounds__(1024) void release_kernel(ReleaseArgs a) {
    __shared__ uint32_t s_w[32];
    __shared__ int32_t s_pages[kKv4MaxSeqs];
    const int b = threadIdx.x;
    int head, count;
    ring_state(a.state, a.n_pages, head, count);
    int len = 0;
    bool done = false;
    if (b < a.B) {
        len = a.len[b];
        done = a.done[b] != 0;
    }
    const int round = (1 << a.shift) - 1;
    // a length that the table cannot hold gives nothing back
    const bool valid = len >= 0 && len <= ((int64_t)a.max_pages << a.shift);
    uint32_t pages = done && valid ? (uint32_t)(((int64_t)len + round) >> a.shift) : 0, none = 0;
    wg_scan2(pages, none, s_w);
    if (b < a.B) {
        s_pages[b] = (int32_t)pages;
        a.len_out[b] = done ? 0 : len;
        if (b == a.B - 1) {
            a.state_out[0] = head;
            a.state_out[1] = (int32_t)min((int64_t)count + pages, (int64_t)a.n_pages);
        }
    }
    __syncthreads();
    // never more than the ring holds: a page given back twice cannot pass it
    const int total = min(s_pages[a.B - 1], a.n_pages);
    for (int e = b; e < total; e += blockDim.x) {
        const int q = find_request(s_pages, a.B, e);
        const int i = e - (q ? s_pages[q - 1] : 0);
        a.ring[ring_entry(ring_entry(head + count, a.n_pages) + e, a.n_pages)] = a.table[(size_t)q * a.max_pages + i];
    }
}

// -------------------------------------------- head rows: norm, rotary, cache
//
// One pass over rows of heads.  Eight neighbouring elements a lane (one or
// two 16-byte loads), so a head is 8 or 16 lanes and a wavefront has one head
// of 8 or 4 consecutive rows at once.  A lane keeps its row and its columns
// over all heads, so the row's angles, position and slot and the norms'
// weights stay in registers; a workgroup computes its rows' angles once, one
// pair a thread, and passes them through LDS.  RMSNorm: y = x rsqrt(mean x^2 +
// eps) w in fp32, the root rounded once, the sum over the head's lanes by DPP.  Rotary: pairs (i, i + d / 2)
// or (2 i, 2 i + 1) of the first d elements turn by pos * theta^(-2 i / d); a
// partner half a head away comes from another lane, by DPP if d is the head.
// 4-bit groups are four lanes: their amax by DPP, then four
// v_cvt_scalef32_pk_fp4_f32 a lane give its dword of codes; consecutive rows
// of a page are adjacent, 128 to 256 bytes of codes and 4 to 8 of a scale
// array from each wavefront.
// With few rows several workgroups share a row's heads.  Bound: a launch for
// up to some 256 rows, then memory.  4096 rows of 40 + 40 heads of 128, bf16:
// norm and rotary 34.5 us (4.9 TB/s read and written, a large copy's rate),
// append 24.9 us (4.3 TB/s).  One row of four heads a wavefront, angles from
// LDS, took 10 and 40 % longer.  Streams that no later access of the call
// repeats bypass the caches: stores 4 us of rotary's 45, loads 5 of append's
// 28; rotary's loads do not (1 us slower, its lines are stored to as well).

enum RowsMode { ROWS_ROPE = 0, ROWS_ROPE_APPEND = 1, ROWS_APPEND = 2 };

struct RowsArgs {
    const char *q, *k, *v;              // rows of heads, strides in bytes
    int64_t q_stride, k_stride, v_stride;
    char *q_out, *k_out;
    int64_t q_out_stride, k_out_stride;
    const void *q_norm, *k_norm;
    const int32_t *pos, *slots;
    int32_t n_rows, nq, nkv, rope_dim, interleaved;
    float eps;
    Kv4Pool pool;
    double ratio;                       // theta^(-2 / d)
};

template <int CTRL>
__device__ __forceinline__ float dpp_mov(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;
constexpr int kDppRor8 = 0x128, kDppQuadMirror = 0x1B;

// Sum over the 8 or 16 lanes of a head, in every lane of it.
template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
    v += dpp_mov<kDppXor1>(v);
    v += dpp_mov<kDppXor2>(v);
    v += dpp_mov<kDppHalfMirror>(v);   // the other four lanes hold one sum each way round
    if (LPH == 16) v += dpp_mov<kDppMirror>(v);
    return v;
}

// The value of the lane half a head's lanes away.
template <int LPH>
__device__ __forceinline__ float half_head_away(float v) {
    if (LPH == 16) return dpp_mov<kDppRor8>(v);
    return dpp_mov<kDppQuadMirror>(dpp_mov<kDppHalfMirror>(v));   // 7 - i, then its quad reversed: i ^ 4
}

// 1 / sqrt(m) rounded once: v_rsq_f32 (off by up to a unit; subnormal numbers
// count as 0 there, hence the scaling) and a Newton step in fp64, which leaves
// 2e-14.
__device__ __forceinline__ float rsqrt_rounded(float m) {
    const bool tiny = m < 0x1p-100f;
    const float y = __builtin_amdgcn_rsqf(tiny ? m * 0x1p100f : m) * (tiny ? 0x1p50f : 1.f);
    const double r = y * (1.5 - 0.5 * m * ((double)y * y));
    return y > 0.f && y < INFINITY ? (float)r : y;     // zero, infinity, NaN as they come
}

// ratio^i / (2 pi), i < 64, by squaring: off by at most 70 roundings of 2^-53,
// less than 1e-8 radians at position 2^20.  (A table of them among the
// arguments, 512 bytes, made a launch 0.3 us longer.)
__device__ __forceinline__ double turns_per_position(double ratio, int i) {
    double f = 0.15915494309189535;
#pragma unroll
    for (int bit = 0; bit < 6; ++bit) {
        if (i >> bit & 1) f *= ratio;
        ratio *= ratio;
    }
    return f;
}

// cos and sin of 2 pi t, rounded once.  The turn t = pos * freq is reduced in
// fp64 (an fp32 product of a position near 2^20 is off by whole hundredths of
// a radian); the remaining angle of at most pi / 4 takes the Taylor series, in
// fp64 too, whose first omitted terms are below 3e-14: a pair's angle is
// computed once for all heads of a row, so its cost does not show, and a 4-bit
// code next to a border is decided by the value rather than by the series.
__device__ __forceinline__ float2 turn_cos_sin(double t) {
    const double quarters = rint(4.0 * t);
    const double x = (t - 0.25 * quarters) * 6.283185307179586;
    const int q = (int)((int64_t)quarters & 3);
    const double x2 = x * x;
    double s = fma(x2, 1.0 / 6227020800.0, -1.0 / 39916800.0);
    s = fma(x2, s, 1.0 / 362880.0);
    s = fma(x2, s, -1.0 / 5040.0);
    s = fma(x2, s, 1.0 / 120.0);
    s = fma(x2, s, -1.0 / 6.0);
    s = fma(x * x2, s, x);
    double c = fma(x2, -1.0 / 87178291200.0, 1.0 / 479001600.0);
    c = fma(x2, c, -1.0 / 3628800.0);
    c = fma(x2, c, 1.0 / 40320.0);
    c = fma(x2, c, -1.0 / 720.0);
    c = fma(x2, c, 1.0 / 24.0);
    c = fma(x2, c, -0.5);
    c = fma(x2, c, 1.0);
    const float a = (float)(q & 1 ? s : c), b = (float)(q & 1 ? c : s);   // |cos|, |sin| of the quadrant
    return make_float2(q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b);
}

template <typename T>
struct Eight;                           // eight elements as loaded
template <>
struct Eight<bf16_t> { uint4 a; };
template <>
struct Eight<float> { uint4 a, b; };

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void put16(char* p, u32x4_t w) {
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>(p));
}
template <bool NT>
__device__ __forceinline__ u32x4_t get16(const char* p) {
    if (NT) return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
    return *reinterpret_cast<const u32x4_t*>(p);
}
template <bool NT>
__device__ __forceinline__ void load8(const char* p, Eight<bf16_t>& r) { r.a = __builtin_bit_cast(uint4, get16<NT>(p)); }
template <bool NT>
__device__ __forceinline__ void load8(const char* p, Eight<float>& r) {
    r.a = __builtin_bit_cast(uint4, get16<NT>(p));
    r.b = __builtin_bit_cast(uint4, get16<NT>(p + 16));
}
__device__ __forceinline__ void floats8(const Eight<bf16_t>& r, float* x) { unpack<bf16_t>(r.a, x); }
__device__ __forceinline__ void floats8(const Eight<float>& r, float* x) {
    unpack<float>(r.a, x);
    unpack<float>(r.b, x + 4);
}
__device__ __forceinline__ void store8(char* p, const float* x, bf16_t) {
    u32x4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f2bf(x[2 * i]) | (uint32_t)f2bf(x[2 * i + 1]) << 16;
    put16(p, w);
}
__device__ __forceinline__ void store8(char* p, const float* x, float) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
        put16(p + 16 * h, u32x4_t{__float_as_uint(x[4 * h]), __float_as_uint(x[4 * h + 1]),
                                  __float_as_uint(x[4 * h + 2]), __float_as_uint(x[4 * h + 3])});
}

// A lane's eight elements as e2m1 codes of its group's scale (one group: the
// four lanes of a quad).
__device__ __forceinline__ uint32_t quantise8(const float* x, int* scale_code) {
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(x[i]) & 0x7fffffffu);   // NaN above all
    amax = max(amax, (uint32_t)__builtin_amdgcn_mov_dpp((int)amax, kDppXor1, 0xf, 0xf, true));
    amax = max(amax, (uint32_t)__builtin_amdgcn_mov_dpp((int)amax, kDppXor2, 0xf, 0xf, true));
    const int code = kv4_scale_code(amax);
    *scale_code = code;
    if (code == kKv4NanScale) return 0;
    const float s = __uint_as_float((uint32_t)code << 23);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
    return w;
}

template <typename T, int HD, int MODE>
__global__ __launch_bounds__(256) void rows_kernel(RowsArgs a) {
    constexpr int LPH = HD / 8;                         // lanes per head
    constexpr int R = kWave / LPH;                      // rows of a workgroup
    constexpr bool ROPE = MODE != ROWS_APPEND, APPEND = MODE != ROWS_ROPE;
    __shared__ __attribute__((aligned(16))) float s_cos[R][HD / 2], s_sin[R][HD / 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane / LPH, row = blockIdx.x * R + r;  // this lane's row
    const int e0 = (lane % LPH) * 8;                    // first of this lane's elements in its head
    const int n_head = (ROPE ? a.nq + a.nkv : a.nkv) + (APPEND ? a.nkv : 0);
    const int nq = ROPE ? a.nq : 0;
    const int step = gridDim.y * 4;
    const bool there = (uint32_t)row < (uint32_t)a.n_rows;

    auto source = [&](int h) -> const char* {
        if (ROPE && h < nq) return a.q + row * a.q_stride + (size_t)(h * HD + e0) * sizeof(T);
        h -= nq;
        if (h < a.nkv) return a.k + row * a.k_stride + (size_t)(h * HD + e0) * sizeof(T);
        return a.v + row * a.v_stride + (size_t)((h - a.nkv) * HD + e0) * sizeof(T);
    };
    int h = blockIdx.y * 4 + wave;
    Eight<T> next = {};
    if (h < n_head && there) load8<APPEND>(source(h), next);
    Eight<T> q_gain = {}, k_gain = {};
    if constexpr (ROPE) {
        if (a.q_norm) load8<false>((const char*)a.q_norm + e0 * sizeof(T), q_gain);
        if (a.k_norm) load8<false>((const char*)a.k_norm + e0 * sizeof(T), k_gain);
        const int tr = tid / (HD / 2), i = tid % (HD / 2);
        if (blockIdx.x * R + tr < a.n_rows && i < a.rope_dim / 2) {
            const float2 cs = turn_cos_sin((double)a.pos[blockIdx.x * R + tr] * turns_per_position(a.ratio, i));
            s_cos[tr][i] = cs.x;
            s_sin[tr][i] = cs.y;
        }
        __syncthreads();
    }
    float c[8], sn[8];                                  // this lane's angles, for all heads
    if constexpr (ROPE) {
        const int half = a.rope_dim / 2;
        const int p0 = e0 >= a.rope_dim ? 0 : a.interleaved ? e0 / 2 : e0 < half ? e0 : e0 - half;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = p0 + (a.interleaved ? i / 2 : i);
            c[i] = s_cos[r][p];
            sn[i] = s_sin[r][p];
        }
    }
    // rows of no request are left as they were
    const bool live = there && !(ROPE && a.pos[row] < 0);
    int page = 0, prow = 0;
    const bool kept = APPEND && live && kv4_slot(a.pool.d, a.slots[row], &page, &prow);
    for (; h < n_head; h += step) {
        const Eight<T> cur = next;
        if (h + step < n_head && there) load8<APPEND>(source(h + step), next);
        float x[8];
        floats8(cur, x);
        const bool is_q = h < nq, is_k = !is_q && h < nq + a.nkv;
        if constexpr (ROPE) {
            // every product and sum rounded by itself: a value is what its
            // formula gives in fp32 whichever way a caller evaluates it
#pragma clang fp contract(off)
            // squares by runs of 4 (or 2), then pairs of neighbouring sums: less
            // rounding than one run, and the order in which the torch build that
            // the calls were compared with adds a head of 128 (or 64)
            float sq[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) sq[i] = x[i] * x[i];
            const float lo = HD == 128 ? ((sq[0] + sq[1]) + sq[2]) + sq[3] : (sq[0] + sq[1]) + (sq[2] + sq[3]);
            const float hi = HD == 128 ? ((sq[4] + sq[5]) + sq[6]) + sq[7] : (sq[4] + sq[5]) + (sq[6] + sq[7]);
            const float ss = head_sum<LPH>(lo + hi);
            if (is_q ? a.q_norm != nullptr : is_k && a.k_norm) {
                const float inv = rsqrt_rounded(ss * (1.f / HD) + a.eps);
                float w[8];
                floats8(is_q ? q_gain : k_gain, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] * inv * w[i];
            }
            if (a.interleaved) {
                if ((is_q || is_k) && e0 < a.rope_dim) {
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const float u = x[i], v = x[i + 1];
                        x[i] = u * c[i] - v * sn[i];
                        x[i + 1] = v * c[i] + u * sn[i];
                    }
                }
            } else {
                const int half = a.rope_dim / 2;
                const bool low = e0 < half;
                // every lane takes part in the exchange; rope_dim is a
                // multiple of 16, so partners are whole lanes apart
                float y[8];
                if (half == HD / 2) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = half_head_away<LPH>(x[i]);
                } else {
                    const int other = low ? lane + half / 8 : lane - half / 8;
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], other, kWave);
                }
                if ((is_q || is_k) && e0 < a.rope_dim) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = low ? x[i] * c[i] - y[i] * sn[i] : x[i] * c[i] + y[i] * sn[i];
                }
            }
            if (is_q && live) store8(a.q_out + row * a.q_out_stride + (size_t)(h * HD + e0) * sizeof(T), x, T());
        }
        if constexpr (!APPEND) {
            if (is_k && live) store8(a.k_out + row * a.k_out_stride + (size_t)((h - nq) * HD + e0) * sizeof(T), x, T());
        } else {
            if (is_q) continue;
            int code;
            const uint32_t w = quantise8(x, &code);
            if (kept) {
                const int hk = is_k ? h - nq : h - nq - a.nkv;
                uint8_t* codes = is_k ? a.pool.k : a.pool.v;
                uint8_t* scales = is_k ? a.pool.ks : a.pool.vs;
                *reinterpret_cast<uint32_t*>(codes + kv4_code_offset(a.pool.d, page, hk, prow) + e0 / 2) = w;
                if (e0 % kKv4Group == 0)
                    scales[kv4_scale_offset(a.pool.d, page, hk, e0 / kKv4Group, prow)] = (uint8_t)code;
            }
        }
    }
}

struct ReadArgs {
    Kv4Pool pool;
    const int32_t* slots;
    int32_t n_rows;
    char *k, *v;
    int64_t k_stride, v_stride;
};

// Cache rows back as values: eight elements a lane, four conversions.  Bound:
// memory; 16001 rows of 8 + 8 heads of 128 to bf16 19 us, 4.4 TB/s.
template <typename T, int HD>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a) {
    constexpr int LPH = HD / 8;
    const int per_row = 2 * a.pool.d.n_kv * LPH;        // lanes that a row's K and V take
    const int64_t total = (int64_t)a.n_rows * per_row;
    for (int64_t t = blockIdx.x * (int64_t)256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int row = (int)(t / per_row), c = (int)(t - (int64_t)row * per_row);
        int page, prow;
        if (!kv4_slot(a.pool.d, a.slots[row], &page, &prow)) continue;
        const int e0 = (c % LPH) * 8;
        int h = c / LPH;
        const bool is_k = h < a.pool.d.n_kv;
        if (!is_k) h -= a.pool.d.n_kv;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(
            (is_k ? a.pool.k : a.pool.v) + kv4_code_offset(a.pool.d, page, h, prow) + e0 / 2);
        const uint32_t code =
            (is_k ? a.pool.ks : a.pool.vs)[kv4_scale_offset(a.pool.d, page, h, e0 / kKv4Group, prow)];
        const float s = __uint_as_float(code << 23);
        char* out = (is_k ? a.k + row * a.k_stride : a.v + row * a.v_stride) + (size_t)(h * HD + e0) * sizeof(T);
        if constexpr (sizeof(T) == 2) {
            // every value is a bf16 number: nothing is rounded
            const u32x4_t o = {
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))};
            put16(out, o);
        } else {
            float x[8];
            auto put = [&](auto pair, int i) { x[i] = pair[0]; x[i + 1] = pair[1]; };
            put(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), 0);
            put(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1), 2);
            put(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), 4);
            put(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3), 6);
            store8(out, x, float());
        }
    }
}

template <typename T, int MODE>
hipError_t launch_rows(const RowsArgs& a, int hd, hipStream_t s) {
    const int heads = (MODE != ROWS_APPEND ? a.nq + a.nkv : a.nkv) + (MODE != ROWS_ROPE ? a.nkv : 0);
    const int blocks = (int)(((int64_t)a.n_rows * hd + 511) / 512);
    // few rows: up to one head a wavefront, so that about four workgroups a
    // CU have work
    int parts = (1024 + blocks - 1) / blocks;
    if (parts > (heads + 3) / 4) parts = (heads + 3) / 4;
    const dim3 grid(blocks, parts), wg(256);
    if (hd == 128) hipLaunchKernelGGL((rows_kernel<T, 128, MODE>), grid, wg, 0, s, a);
    else hipLaunchKernelGGL((rows_kernel<T, 64, MODE>), grid, wg, 0, s, a);
    return hipGetLastError();
}

template <int MODE>
hipError_t launch_rows_dtype(const RowsArgs& a, int dtype, int hd, hipStream_t s) {
    return dtype == BUDDY_BF16 ? launch_rows<bf16_t, MODE>(a, hd, s) : launch_rows<float, MODE>(a, hd, s);
}

buddy_status kv4_check_pool(const buddy_kv4* c, Kv4Pool* out) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return BUDDY_EINVAL;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) || !aligned16(c->v_scale)) return BUDDY_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128) return BUDDY_ESHAPE;
    if (c->page_rows < 16 || c->page_rows > 256 || (c->page_rows & (c->page_rows - 1))) return BUDDY_ESHAPE;
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return BUDDY_ESHAPE;
    if (c->n_pages < 1) return BUDDY_EINVAL;
    if ((int64_t)c->n_pages * c->page_rows > INT32_MAX) return BUDDY_ECAPACITY;
    out->k = c->k; out->v = c->v; out->ks = c->k_scale; out->vs = c->v_scale;
    out->d = Kv4Dims{c->n_pages, __builtin_ctz((unsigned)c->page_rows), c->n_kv_heads, c->head_dim};
    return BUDDY_OK;
}

namespace {

// Rows of heads of `width` elements: whole 16-byte units apart.
bool rows_ok(const void* p, int64_t stride, int64_t width, int64_t n_rows, int size) {
    return p && aligned16(p) && stride >= 0 && stride <= INT64_MAX / 64 / (n_rows > 0 ? n_rows : 1) &&
           stride * size % 16 == 0 && (n_rows <= 1 || stride >= width);
}

bool overlap(const int32_t* x, const int32_t* y, int n) {
    return (uintptr_t)x < (uintptr_t)(y + n) && (uintptr_t)y < (uintptr_t)(x + n);
}

constexpr int kKv4MaxRows = 1 << 24;     // of a call: grids stay within 32 bits of threads

buddy_status check_paging(int32_t B, int32_t page_rows, int32_t max_pages, int32_t n_pages) {
    if (page_rows < 16 || page_rows > 256 || (page_rows & (page_rows - 1))) return BUDDY_ESHAPE;
    if (max_pages < 1 || n_pages < 1) return BUDDY_EINVAL;
    if (B > kKv4MaxSeqs) return BUDDY_ECAPACITY;
    if ((int64_t)n_pages * page_rows > INT32_MAX || (int64_t)max_pages * page_rows > INT32_MAX)
        return BUDDY_ECAPACITY;
    return BUDDY_OK;
}

// The head form and the rows' places, for the calls that norm and rotate.
buddy_status fill_rope(const buddy_qk_form* f, RowsArgs& a) {
    if (!f) return BUDDY_EINVAL;
    if (f->dtype != BUDDY_F32 && f->dtype != BUDDY_BF16) return BUDDY_EINVAL;
    if (f->head_dim != 64 && f->head_dim != 128) return BUDDY_ESHAPE;
    if (f->n_heads < 1 || f->n_kv_heads < 1 || f->n_heads > 1024 || f->n_kv_heads > 1024) return BUDDY_ESHAPE;
    if (f->rope_dim < 0 || f->rope_dim > f->head_dim || f->rope_dim % 16) return BUDDY_ESHAPE;
    if (!(f->rms_eps >= 0.f) || !(f->rope_theta > 0.f)) return BUDDY_EINVAL;
    if (!aligned16(f->q_norm) || !aligned16(f->k_norm)) return BUDDY_EINVAL;
    a.nq = f->n_heads;
    a.nkv = f->n_kv_heads;
    a.rope_dim = f->rope_dim;
    a.interleaved = f->interleaved != 0;
    a.eps = f->rms_eps;
    a.q_norm = f->q_norm;
    a.k_norm = f->k_norm;
    if (f->rope_dim > 0) a.ratio = pow((double)f->rope_theta, -2.0 / f->rope_dim);
    return BUDDY_OK;
}

}  // namespace
}  // namespace buddy

using namespace buddy;

extern "C" {

buddy_status buddy_plan_pages(const int32_t* len, const int32_t* n_new, int32_t B, int32_t page_rows, int32_t* table,
                              int32_t max_pages, const int32_t* ring, int32_t n_pages, const int32_t* ring_state,
                              int32_t* ring_state_out, int32_t* len_out, int32_t* cu_rows, int32_t* pos,
                              int32_t* slots, int32_t n_rows, uint8_t* refused, void* stream) {
    if (B == 0) return BUDDY_OK;
    if (B < 0 || n_rows < 0 || !len || !n_new || !table || !ring || !ring_state || !ring_state_out || !len_out ||
        !cu_rows || !refused || (n_rows > 0 && (!pos || !slots)))
        return BUDDY_EINVAL;
    const buddy_status st = check_paging(B, page_rows, max_pages, n_pages);
    if (st != BUDDY_OK) return st;
    if (n_rows >= (1 << 30)) return BUDDY_ECAPACITY;
    PlanArgs a{len, n_new, B, __builtin_ctz((unsigned)page_rows), max_pages, n_pages, n_rows, table, ring,
               ring_state, ring_state_out, len_out, cu_rows, pos, slots, refused, 1, 1};
    hipStream_t s = (hipStream_t)stream;
    const unsigned wg = B <= 256 ? 256 : 1024;
    const unsigned blocks = n_rows <= (int)wg ? 1 : (n_rows + wg - 1) / wg < 1024 ? (n_rows + wg - 1) / wg : 1024;
    const bool in_place = overlap(len, len_out, B) || overlap(ring_state, ring_state_out, 2);
    if (!in_place) {
        hipLaunchKernelGGL(plan_kernel, dim3(blocks), dim3(wg), 0, s, a);
    } else if (n_rows <= 4096) {                       // one workgroup's time for 4096 is that of a launch
        hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(wg), 0, s, a);
    } else {
        a.write = 0;
        hipLaunchKernelGGL(plan_kernel, dim3(blocks), dim3(wg), 0, s, a);
        a.write = 1; a.map = 0;
        hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(wg), 0, s, a);
    }
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

buddy_status buddy_release_pages(const int32_t* len, const uint8_t* done, int32_t B, int32_t page_rows,
                                 const int32_t* table, int32_t max_pages, int32_t* ring, int32_t n_pages,
                                 const int32_t* ring_state, int32_t* ring_state_out, int32_t* len_out, void* stream) {
    if (B == 0) return BUDDY_OK;
    if (B < 0 || !len || !done || !table || !ring || !ring_state || !ring_state_out || !len_out) return BUDDY_EINVAL;
    const buddy_status st = check_paging(B, page_rows, max_pages, n_pages);
    if (st != BUDDY_OK) return st;
    const ReleaseArgs a{len, done, B, __builtin_ctz((unsigned)page_rows), max_pages, n_pages, table, ring,
                        ring_state, ring_state_out, len_out};
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(B <= 256 ? 256 : 1024), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

buddy_status buddy_qk_norm_rope(const buddy_qk_form* f, const void* q, int64_t q_stride, const void* k,
                                int64_t k_stride, const int32_t* pos, int32_t n_rows, void* q_out,
                                int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
    RowsArgs a;
    memset(&a, 0, sizeof(a));
    const buddy_status st = fill_rope(f, a);
    if (st != BUDDY_OK) return st;
    if (n_rows == 0) return BUDDY_OK;
    const int size = f->dtype == BUDDY_BF16 ? 2 : 4;
    const int64_t qw = (int64_t)f->n_heads * f->head_dim, kw = (int64_t)f->n_kv_heads * f->head_dim;
    if (n_rows < 0 || !pos || !rows_ok(q, q_stride, qw, n_rows, size) || !rows_ok(k, k_stride, kw, n_rows, size) ||
        !rows_ok(q_out, q_out_stride, qw, n_rows, size) || !rows_ok(k_out, k_out_stride, kw, n_rows, size))
        return BUDDY_EINVAL;
    if (n_rows > kKv4MaxRows) return BUDDY_ECAPACITY;
    a.q = (const char*)q; a.q_stride = q_stride * size;
    a.k = (const char*)k; a.k_stride = k_stride * size;
    a.q_out = (char*)q_out; a.q_out_stride = q_out_stride * size;
    a.k_out = (char*)k_out; a.k_out_stride = k_out_stride * size;
    a.pos = pos; a.n_rows = n_rows;
    return launch_rows_dtype<ROWS_ROPE>(a, f->dtype, f->head_dim, (hipStream_t)stream) == hipSuccess ? BUDDY_OK
                                                                                                  : BUDDY_EDEVICE;
}

buddy_status buddy_kv4_append_qkv(const buddy_kv4* cache, const buddy_qk_form* f, const void* q, int64_t q_stride,
                                  const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                  const int32_t* pos, const int32_t* slots, int32_t n_rows, void* q_out,
                                  int64_t q_out_stride, void* stream) {
    RowsArgs a;
    memset(&a, 0, sizeof(a));
    buddy_status st = kv4_check_pool(cache, &a.pool);
    if (st != BUDDY_OK || (st = fill_rope(f, a)) != BUDDY_OK) return st;
    if (f->head_dim != cache->head_dim || f->n_kv_heads != cache->n_kv_heads) return BUDDY_EINVAL;
    if (n_rows == 0) return BUDDY_OK;
    const int size = f->dtype == BUDDY_BF16 ? 2 : 4;
    const int64_t qw = (int64_t)f->n_heads * f->head_dim, kw = (int64_t)f->n_kv_heads * f->head_dim;
    if (n_rows < 0 || !pos || !slots || !rows_ok(q, q_stride, qw, n_rows, size) ||
        !rows_ok(k, k_stride, kw, n_rows, size) || !rows_ok(v, v_stride, kw, n_rows, size) ||
        !rows_ok(q_out, q_out_stride, qw, n_rows, size))
        return BUDDY_EINVAL;
    if (n_rows > kKv4MaxRows) return BUDDY_ECAPACITY;
    a.q = (const char*)q; a.q_stride = q_stride * size;
    a.k = (const char*)k; a.k_stride = k_stride * size;
    a.v = (const char*)v; a.v_stride = v_stride * size;
    a.q_out = (char*)q_out; a.q_out_stride = q_out_stride * size;
    a.pos = pos; a.slots = slots; a.n_rows = n_rows;
    return launch_rows_dtype<ROWS_ROPE_APPEND>(a, f->dtype, f->head_dim, (hipStream_t)stream) == hipSuccess
               ? BUDDY_OK : BUDDY_EDEVICE;
}

buddy_status buddy_kv4_append(const buddy_kv4* cache, int32_t dtype, const void* k, int64_t k_stride, const void* v,
                              int64_t v_stride, const int32_t* slots, int32_t n_rows, void* stream) {
    RowsArgs a;
    memset(&a, 0, sizeof(a));
    const buddy_status st = kv4_check_pool(cache, &a.pool);
    if (st != BUDDY_OK) return st;
    if (dtype != BUDDY_F32 && dtype != BUDDY_BF16) return BUDDY_EINVAL;
    if (n_rows == 0) return BUDDY_OK;
    const int size = dtype == BUDDY_BF16 ? 2 : 4;
    const int64_t kw = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (n_rows < 0 || !slots || !rows_ok(k, k_stride, kw, n_rows, size) || !rows_ok(v, v_stride, kw, n_rows, size))
        return BUDDY_EINVAL;
    if (n_rows > kKv4MaxRows) return BUDDY_ECAPACITY;
    a.k = (const char*)k; a.k_stride = k_stride * size;
    a.v = (const char*)v; a.v_stride = v_stride * size;
    a.slots = slots; a.n_rows = n_rows; a.nkv = cache->n_kv_heads;
    return launch_rows_dtype<ROWS_APPEND>(a, dtype, cache->head_dim, (hipStream_t)stream) == hipSuccess
               ? BUDDY_OK : BUDDY_EDEVICE;
}

buddy_status buddy_kv4_read(const buddy_kv4* cache, const int32_t* slots, int32_t n_rows, int32_t dtype, void* k_out,
                            int64_t k_stride, void* v_out, int64_t v_stride, void* stream) {
    ReadArgs a;
    memset(&a, 0, sizeof(a));
    const buddy_status st = kv4_check_pool(cache, &a.pool);
    if (st != BUDDY_OK) return st;
    if (dtype != BUDDY_F32 && dtype != BUDDY_BF16) return BUDDY_EINVAL;
    if (n_rows == 0) return BUDDY_OK;
    const int size = dtype == BUDDY_BF16 ? 2 : 4;
    const int64_t kw = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (n_rows < 0 || !slots || !rows_ok(k_out, k_stride, kw, n_rows, size) ||
        !rows_ok(v_out, v_stride, kw, n_rows, size))
        return BUDDY_EINVAL;
    if (n_rows > kKv4MaxRows) return BUDDY_ECAPACITY;
    a.slots = slots; a.n_rows = n_rows;
    a.k = (char*)k_out; a.k_stride = k_stride * size;
    a.v = (char*)v_out; a.v_stride = v_stride * size;
    const int64_t lanes = (int64_t)n_rows * 2 * kw / 8;
    const int64_t blocks = (lanes + 255) / 256;
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)), wg(256);
    hipStream_t s = (hipStream_t)stream;
    const bool big = cache->head_dim == 128;
    if (dtype == BUDDY_BF16) {
        if (big) hipLaunchKernelGGL((read_kernel<bf16_t, 128>), grid, wg, 0, s, a);
        else hipLaunchKernelGGL((read_kernel<bf16_t, 64>), grid, wg, 0, s, a);
    } else {
        if (big) hipLaunchKernelGGL((read_kernel<float, 128>), grid, wg, 0, s, a);
        else hipLaunchKernelGGL((read_kernel<float, 64>), grid, wg, 0, s, a);
    }
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

}  // extern "C"
