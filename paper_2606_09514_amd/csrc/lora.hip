// Low-rank adapters of many requests beside a shared projection
// (buddy_lora_plan, buddy_lora_add): out[r] = y[r] + scale_i B_i (A_i x[r]) for
// the adapter i of row r.
//
// The plan sorts the rows by adapter and cuts each adapter's rows into tiles,
// so that a tile reads its adapter's weights once.  Two kernels then run over
// the tiles: shrink, t = A x, whose long sums are split over workgroups that
// leave fp32 parts in the workspace, and expand, which adds the parts in order,
// multiplies by B and adds to y.  Bound: memory (the adapters in use, x, y and
// out); few rows: two launches.
#include "mx8.h"

namespace buddy {

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kLoraMaxAdapters = 4096;
constexpr int kLoraMaxRank = 128;
constexpr int kPlanHead = 4;             // ints before the tiles: tiles, rows, adapters, rows of a tile
constexpr int kTileHead = 4;             // ints of a tile before its rows: adapter, how many
constexpr int kShrinkParts = 8;          // parts of a sum over d_in

// Rows of a tile, by the rows and adapters of the call alone, so that a plan and
// the calls that use it agree.  A tile of 64 reads the adapter's weights a quarter as
// often; filled by few rows it multiplies for nothing.  Five adapters of rank 128,
// 18944 -> 3584: 1200 rows 96 us with tiles of 16, 54 with 64, 800 rows 56 and 55;
// of rank 16 the two are within a tenth.  1000 rows of 40 adapters: 36 with 16.
inline int lora_tile_rows(int n_rows, int n_adapters) { return n_rows >= 1024 && n_rows / (n_adapters + 1) >= 32 ? 64 : 16; }
// Tiles at most: every group of rows (an adapter's or none's) ends in one that
// is not full.
inline int lora_max_tiles(int n_rows, int n_adapters) {
    const int groups = n_rows < n_adapters + 1 ? n_rows : n_adapters + 1;
    return n_rows / lora_tile_rows(n_rows, n_adapters) + groups;
}

// ------------------------------------------------------------------- plan
//
// One workgroup: rows of each adapter are counted in LDS, prefix sums give each
// adapter's first tile, then tiles and their rows are written.  A tile's rows
// stand beside it, so that a kernel reads both at once.  Rows of one
// adapter come in no fixed order: a row's result does not depend on it.
struct LoraPlanArgs { const int32_t* ids; int32_t n_rows, n_adapters, tile_rows; int32_t* plan; };

// A wavefront whose rows are all of one group, as those of a prompt are, counts
// them at once.  4099 rows of 5 adapters: 12.5 us with an atomic each.
__device__ __forceinline__ int add_to(int* s, int g) {
    const int first = __builtin_amdgcn_readfirstlane(g);
    const uint64_t here = __ballot(1), same = __ballot(g == first);
    if (first < 0 || same != here) return g >= 0 ? atomicAdd(&s[g], 1) : -1;
    const int place = __builtin_amdgcn_mbcnt_hi((uint32_t)(here >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)here, 0));
    int base = 0;
    if (place == 0) base = atomicAdd(&s[first], (int)__popcll(here));
    return __builtin_amdgcn_readfirstlane(base) + place;
}

template <int kPer>                       // groups of a thread
__global__ __launch_bounds__(1024) void lora_plan_kernel(LoraPlanArgs a) {
    __shared__ int s_n[kPer * 1024], s_tile[kPer * 1024], s_wave[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int T = a.tile_rows;
    for (int i = tid; i < kPer * 1024; i += 1024) s_n[i] = 0;
    __syncthreads();
    auto group = [&](int r) {             // -1 none is group 0; others no group
        const int id = a.ids[r];
        return id >= -1 && id < a.n_adapters ? id + 1 : -1;
    };
    for (int r = tid; r < a.n_rows; r += 1024) add_to(s_n, group(r));
    __syncthreads();
    int tiles = 0;                        // of this thread's groups
#pragma unroll
    for (int i = 0; i < kPer; ++i) tiles += (s_n[tid * kPer + i] + T - 1) / T;
    int end = tiles;                      // inclusive sums over the wavefront
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(end, d);
        if (lane >= d) end += v;
    }
    if (lane == 63) s_wave[wave] = end;
    __syncthreads();
    int tile = end - tiles, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        if (w < wave) tile += s_wave[w];
        all += s_wave[w];
    }
    int32_t* out = a.plan + kPlanHead;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int g = tid * kPer + i, n = s_n[g];
        s_tile[g] = tile;
        for (int at = 0; at < n; at += T, ++tile)
            *reinterpret_cast<int2*>(out + (int64_t)tile * (kTileHead + T)) = make_int2(g - 1, min(T, n - at));
        s_n[g] = 0;
    }
    if (tid == 0) *reinterpret_cast<int4*>(a.plan) = make_int4(all, a.n_rows, a.n_adapters, T);
    __syncthreads();
    for (int r = tid; r < a.n_rows; r += 1024) {
        const int g = group(r), at = add_to(s_n, g);
        if (at >= 0) out[(int64_t)(s_tile[g] + at / T) * (kTileHead + T) + kTileHead + at % T] = r;
    }
}

// ------------------------------------------------------------ shrink, expand

struct LoraArgs {
    const char *a, *b, *x, *y;
    const float* scale;
    char* out;
    int64_t x_stride, y_stride, out_stride;   // bytes
    const int32_t* plan;
    float* part;                              // [parts][n_rows][rank]
    int32_t n_rows, n_adapters, tile_rows, rank, d_in, d_out, parts, blocks, in_place;
};

// A tile of the plan: its adapter, and how many rows it has.  A plan that does
// not fit the call has no tiles.
struct Tile { int adapter, count; const int32_t* rows; };
__device__ __forceinline__ Tile tile_of(const LoraArgs& a, int t) {
    const int T = a.tile_rows;
    const int32_t* p = a.plan + kPlanHead + (int64_t)t * (kTileHead + T);
    const int4 head = *reinterpret_cast<const int4*>(a.plan);
    const int2 v = *reinterpret_cast<const int2*>(p);
    const bool fits = t < head.x && head.y == a.n_rows && head.z == a.n_adapters && head.w == T && v.x >= -1 && v.x < a.n_adapters &&
                      v.y >= 1 && v.y <= T;
    return Tile{fits ? v.x : -1, fits ? v.y : 0, p + kTileHead};
}
// Row i (of 0..tile_rows - 1) of a tile, -1 for one that it does not have.
__device__ __forceinline__ int row_of(const LoraArgs& a, const Tile& t, int i) {
    const int r = t.rows[i];              // without a branch: several are read at once
    return (i < t.count) & ((uint32_t)r < (uint32_t)a.n_rows) ? r : -1;
}

// A 16 x 32 operand, lane i + 16 g: row i, k = 8 g .. + 7.  For bf16 the matrix
// instruction of that size; for fp32 eight of 16 x 16 x 4, whose operands are
// one element a lane (k = g): any order of k serves as long as both sides have
// the same, so instruction e takes element e of every lane.
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { u32x4_t v; };
template <> struct Frag<float> { f32x4_t v[2]; };

__device__ __forceinline__ void load_frag(const char* p, Frag<bf16_t>& f) { f.v = *reinterpret_cast<const u32x4_t*>(p); }
__device__ __forceinline__ void load_frag(const char* p, Frag<float>& f) {
    f.v[0] = *reinterpret_cast<const f32x4_t*>(p);
    f.v[1] = *reinterpret_cast<const f32x4_t*>(p + 16);
}
__device__ __forceinline__ void clear_unless(bool keep, Frag<bf16_t>& f) {
#pragma unroll
    for (int e = 0; e < 4; ++e) f.v[e] = keep ? f.v[e] : 0;
}
__device__ __forceinline__ void clear_unless(bool keep, Frag<float>& f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e >> 2][e & 3] = keep ? f.v[e >> 2][e & 3] : 0.f;
}
__device__ __forceinline__ f32x4_t mfma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a.v), __builtin_bit_cast(bf16x8_t, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mfma(const Frag<float>& a, const Frag<float>& b, f32x4_t c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[e >> 2][e & 3], b.v[e >> 2][e & 3], c, 0, 0, 0);
    return c;
}

// t = A x for a part of d_in and 16 RT of the rank: a wavefront takes the RT tiles
// of 16 of the rank and the RG groups of 16 rows of the plan's tile, the workgroup's four wavefronts a
// quarter of the part each (their sums meet in LDS in order, a group at a time).
// Left in the workspace as [part][row][rank].  4099 rows of 3584 inputs, rank 64, five
// adapters: 19.8 us (29 MB of x); with one group of rows a wavefront, which reads A
// again for each, 22.
template <typename T, int RT, int RG>
__global__ __launch_bounds__(256) void shrink_kernel(LoraArgs a) {
    __shared__ __attribute__((aligned(16))) f32x4_t s_sum[4][RT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int r0 = blockIdx.z * 16 * RT;                                 // of the rank
    const Tile t = tile_of(a, blockIdx.x);
    int row[RG];                                                        // results of row 0 in place of none are dropped
#pragma unroll
    for (int u = 0; u < RG; ++u) row[u] = row_of(a, t, 16 * u + i);
    if (t.count == 0 || t.adapter < 0) return;
    // steps of 32 of d_in, the last may be short
    const int steps = (a.d_in + 31) / 32, whole = a.d_in / 32;
    const int slices = a.parts * 4, slice = blockIdx.y * 4 + wave;
    const int first = (int)((int64_t)steps * slice / slices), last = (int)((int64_t)steps * (slice + 1) / slices);
    const char* x[RG];
#pragma unroll
    for (int u = 0; u < RG; ++u) x[u] = a.x + max(row[u], 0) * a.x_stride + 8 * g * sizeof(T);
    const char* w[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
        w[r] = a.a + ((int64_t)t.adapter * a.rank + min(r0 + 16 * r + i, a.rank - 1)) * a.d_in * sizeof(T) + 8 * g * sizeof(T);
    f32x4_t acc[RG][RT] = {};
    constexpr int U = RT * RG <= 2 ? 4 : RT * RG <= 16 ? 2 : 1;          // steps in flight
    int k = first;
    for (; k + U <= min(last, whole); k += U) {
        Frag<T> fx[U][RG], fw[U][RT];
#pragma unroll
        for (int v = 0; v < U; ++v) {
#pragma unroll
            for (int u = 0; u < RG; ++u) load_frag(x[u] + (int64_t)(k + v) * 32 * sizeof(T), fx[v][u]);
#pragma unroll
            for (int r = 0; r < RT; ++r) load_frag(w[r] + (int64_t)(k + v) * 32 * sizeof(T), fw[v][r]);
        }
#pragma unroll
        for (int v = 0; v < U; ++v)
#pragma unroll
            for (int u = 0; u < RG; ++u)
#pragma unroll
                for (int r = 0; r < RT; ++r) acc[u][r] = mfma(fw[v][r], fx[v][u], acc[u][r]);
    }
    for (; k < last; ++k) {
        const bool there = k * 32 + 8 * g < a.d_in;                      // 8 of d_in are there or not
        Frag<T> fx[RG] = {}, fw;
#pragma unroll
        for (int u = 0; u < RG; ++u)
            if (there) load_frag(x[u] + (int64_t)k * 32 * sizeof(T), fx[u]);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            fw = {};
            if (there) load_frag(w[r] + (int64_t)k * 32 * sizeof(T), fw);
#pragma unroll
            for (int u = 0; u < RG; ++u) acc[u][r] = mfma(fw, fx[u], acc[u][r]);
        }
    }
#pragma unroll
    for (int u = 0; u < RG; ++u) {
        if (u > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) s_sum[wave][r][lane] = acc[u][r];
        __syncthreads();
        // element e of lane: rank 16 r + 4 (lane / 16) + e, row lane % 16
        for (int at = threadIdx.x; at < RT * 64; at += 256) {
            const int r = at >> 6, l = at & 63;
            const f32x4_t v = (s_sum[0][r][l] + s_sum[1][r][l]) + (s_sum[2][r][l] + s_sum[3][r][l]);
            const int j = r0 + 16 * r + 4 * (l >> 4), to = row_of(a, t, 16 * u + (l & 15));
            if (to >= 0 && j < a.rank)                                   // rank % 8 == 0
                *reinterpret_cast<f32x4_t*>(a.part + ((int64_t)blockIdx.y * a.n_rows + to) * a.rank + j) = v;
        }
    }
}

// out = y + scale B t for blocks of 64 outputs a wavefront and the rows of a
// tile.  t is the sum of its parts in order; for bf16 it enters the product as
// two bf16 parts, the second the rounding of the first, so that 16 of its bits
// count.  The products are of 16 rows by the 16 outputs 4 j + q (q < 4), so that a
// lane ends with four neighbouring outputs of four rows and sixteen lanes with a
// row's 64: y is read and out written in whole lines.  Neighbouring workgroups take
// neighbouring outputs of the same rows.  4099 rows of 37888 outputs, rank 64: 169 us
// (3.7 TB/s).  Measured on the way: the rows' tiles in neighbouring workgroups 187
// instead of 181, the next y asked for after the stores 184 instead of 178, one block
// of outputs a workgroup instead of four 240; t added up by each wavefront for itself,
// 16 bytes a row at a time, 178 (and 578 rows of rank 128 96 instead of 79).
template <typename T> struct Weight;                 // t as it enters the product
template <> struct Weight<float> { Frag<float> f; };
template <> struct Weight<bf16_t> { Frag<bf16_t> hi, lo; };

// Half (the first or second four) of a lane's eight elements.
__device__ __forceinline__ void put_half(f32x4_t x, int half, Weight<float>& w) { w.f.v[half] = x; }
__device__ __forceinline__ void put_half(f32x4_t x, int half, Weight<bf16_t>& w) {
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        hi[p] = pack_bf16x2(x[2 * p], x[2 * p + 1]);
        const float dx = x[2 * p] - __uint_as_float(hi[p] << 16), dy = x[2 * p + 1] - __uint_as_float(hi[p] & 0xffff0000u);
        lo[p] = pack_bf16x2(dx == dx ? dx : 0.f, dy == dy ? dy : 0.f);   // an infinity has no second part
    }
    reinterpret_cast<uint2*>(&w.hi)[half] = make_uint2(hi[0], hi[1]);
    reinterpret_cast<uint2*>(&w.lo)[half] = make_uint2(lo[0], lo[1]);
}
__device__ __forceinline__ f32x4_t mfma(const Weight<float>& a, const Frag<float>& b, f32x4_t c) { return mfma(a.f, b, c); }
__device__ __forceinline__ f32x4_t mfma(const Weight<bf16_t>& a, const Frag<bf16_t>& b, f32x4_t c) { return mfma(a.lo, b, mfma(a.hi, b, c)); }

// Four neighbouring values.
template <typename T> struct Four;
template <> struct Four<bf16_t> { uint2 v; };
template <> struct Four<float> { f32x4_t v; };
__device__ __forceinline__ void add4(char* out, const Four<bf16_t>& y, f32x4_t v) {
    const uint32_t a = f2bf(__uint_as_float(y.v.x << 16) + v[0]), b = f2bf(__uint_as_float(y.v.x & 0xffff0000u) + v[1]);
    const uint32_t c = f2bf(__uint_as_float(y.v.y << 16) + v[2]), d = f2bf(__uint_as_float(y.v.y & 0xffff0000u) + v[3]);
    *reinterpret_cast<uint2*>(out) = make_uint2(a | b << 16, c | d << 16);
}
__device__ __forceinline__ void add4(char* out, const Four<float>& y, f32x4_t v) { *reinterpret_cast<f32x4_t*>(out) = y.v + v; }

// KT: steps of 32 of the rank; RG: groups of 16 rows, a tile of 64 or half of one,
// whose t stays in LDS (of 16 rows: in registers) over a.blocks blocks of 256 outputs
// of the workgroup.
template <typename T, int KT, int RG>
__global__ __launch_bounds__(256) void expand_kernel(LoraArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    constexpr int kPieces = RG == 2 ? 2 : 1;                             // of a tile
    const Tile t = tile_of(a, blockIdx.y / kPieces);
    const int at0 = blockIdx.y % kPieces * 32;                           // first row of the piece
    int row[RG][4];                                                      // 4 g + e of each group
#pragma unroll
    for (int u = 0; u < RG; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) row[u][e] = row_of(a, t, at0 + 16 * u + 4 * g + e);
    if (t.count <= at0 || (t.adapter < 0 && a.in_place)) return;
    const int first = blockIdx.x * a.blocks * 256 + wave * 64, end = min(first + a.blocks * 256, a.d_out);
    // outputs n .. n + 3 (all there or none) of the lane's rows; others are read in
    // place of what is not there and not stored
    auto load = [&](int u, int n, Four<T>* y) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = *reinterpret_cast<const Four<T>*>(a.y + max(row[u][e], 0) * a.y_stride + (int64_t)min(n, a.d_out - 4) * sizeof(T));
    };
    auto store = [&](int u, int e, int n, const Four<T>& y, f32x4_t v) {
        if (row[u][e] >= 0 && n < a.d_out) add4(a.out + row[u][e] * a.out_stride + (int64_t)n * sizeof(T), y, v);
    };
    if (t.adapter < 0) {
        Four<T> y[4];
        const f32x4_t none = {-0.f, -0.f, -0.f, -0.f};                   // y + -0 is y
        for (int n0 = first; n0 < end; n0 += 256)
#pragma unroll
            for (int u = 0; u < RG; ++u) {
                load(u, n0 + 4 * i, y);
#pragma unroll
                for (int e = 0; e < 4; ++e) store(u, e, n0 + 4 * i, y[e], none);
            }
        return;
    }
    const float scale = a.scale[t.adapter];
    // y of the next outputs is asked for as soon as a group's are stored, B as soon
    // as the last group is done: one block's latency is hidden behind the other's work
    Four<T> y[RG][4];
    Frag<T> fb[4][KT];
    auto take_b = [&](int n) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t from = (int64_t)t.adapter * a.d_out + min(n + q, a.d_out - 1);
#pragma unroll
            for (int k = 0; k < KT; ++k)
                load_frag(a.b + (from * a.rank + min(32 * k + 8 * g, a.rank - 8)) * sizeof(T), fb[q][k]);
        }
    };
    if (first < end) {
        take_b(first + 4 * i);
#pragma unroll
        for (int u = 0; u < RG; ++u) load(u, first + 4 * i, y[u]);
    }
    // t as operands in LDS: the workgroup reads the parts once, in whole lines
    __shared__ Weight<T> s_w[RG * KT * 64];
    constexpr int kStep = 32 / KT, kTake = RG * 16 / kStep > 0 ? RG * 16 / kStep : 1;   // rows of the workgroup at a time
    constexpr int kAhead = kTake < 4 ? kTake : 4;
    const int c = threadIdx.x % (KT * 8), r = threadIdx.x / (KT * 8);    // four of the rank
    if (r < RG * 16)
        for (int q0 = 0; q0 < kTake; q0 += kAhead) {
            int of[kAhead];
            f32x4_t v[kAhead] = {};
#pragma unroll
            for (int q = 0; q < kAhead; ++q) of[q] = row_of(a, t, at0 + r + (q0 + q) * kStep);
            const bool there = 4 * c < a.rank;                           // rank % 8 == 0
            for (int p = 0; p < a.parts; ++p)
#pragma unroll
                for (int q = 0; q < kAhead; ++q)
                    v[q] += *reinterpret_cast<const f32x4_t*>(a.part + ((int64_t)p * a.n_rows + max(of[q], 0)) * a.rank + (there ? 4 * c : 0));
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                const int m = r + (q0 + q) * kStep;
                if (of[q] < 0 || !there) v[q] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
                put_half(v[q], c & 1, s_w[((m >> 4) * KT + (c >> 3)) * 64 + (c >> 1 & 3) * 16 + (m & 15)]);
            }
        }
    __syncthreads();
    Weight<T> w[KT];
    if constexpr (RG == 1)
#pragma unroll
        for (int k = 0; k < KT; ++k) w[k] = s_w[k * 64 + lane];
    for (int n0 = first; n0 < end; n0 += 256) {
        const int n = n0 + 4 * i;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < KT; ++k) clear_unless(32 * k + 8 * g < a.rank, fb[q][k]);
#pragma unroll
        for (int u = 0; u < RG; ++u) {
            f32x4_t acc[4] = {};
#pragma unroll
            for (int k = 0; k < KT; ++k) {
                if constexpr (RG > 1) w[k] = s_w[(u * KT + k) * 64 + lane];
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[q] = mfma(w[k], fb[q][k], acc[q]);
            }
            f32x4_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = (f32x4_t){scale * acc[0][e], scale * acc[1][e], scale * acc[2][e], scale * acc[3][e]};
            if (__ballot(((row[u][0] | row[u][1] | row[u][2] | row[u][3]) >= 0) & (n < a.d_out)) == ~0ull) {
#pragma unroll
                for (int e = 0; e < 4; ++e) add4(a.out + row[u][e] * a.out_stride + (int64_t)n * sizeof(T), y[u][e], v[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) store(u, e, n, y[u][e], v[e]);
            }
            if (n0 + 256 < end) load(u, n + 256, y[u]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (n0 + 256 < end) take_b(n + 256);
    }
}

// Blocks of the rank of the first kernel, in workgroups of their own.
static int lora_rank_blocks(int rank, int tile_rows) { return tile_rows == 16 ? (rank + 31) / 32 : (rank + 63) / 64; }
// Parts of the sums over d_in: about 256 workgroups (320 of the large tiles), each
// wavefront with four steps or more; at most 8, and 16 for all blocks of 32 of the
// rank, since every workgroup of the second kernel adds up the parts (14 rows, 5120
// -> 5120, rank 128: 27 us with 8 parts and the whole rank in one workgroup, 20 with
// 4; 64 rows, d_in 18944, rank 64: 30 and 28).
static int lora_parts(const buddy_lora* l, int n_rows) {
    const int T = lora_tile_rows(n_rows, l->n_adapters);
    const int groups = lora_max_tiles(n_rows, l->n_adapters) * lora_rank_blocks(l->rank, T);
    const int want = ((T == 16 ? 256 : 320) + groups - 1) / groups, steps = (l->d_in / 32 + 15) / 16, limit = 16 / ((l->rank + 31) / 32);
    const int most = limit < kShrinkParts ? limit : kShrinkParts, p = want < steps ? want : steps;
    return p < 1 ? 1 : p > most ? most : p;
}
// Rows of parts for n_rows rows or fewer: parts is at most 320 / groups + 1, and
// there are more than n_rows / 64 groups.
static int64_t lora_part_rows(int n_rows) {
    return (int64_t)n_rows * kShrinkParts < 65536 + (int64_t)n_rows ? (int64_t)n_rows * kShrinkParts : 65536 + (int64_t)n_rows;
}

template <typename T>
void launch_shrink(const LoraArgs& a, unsigned tiles, hipStream_t s) {
    const dim3 grid(tiles, a.parts, lora_rank_blocks(a.rank, a.tile_rows)), wg(256);
    if (a.tile_rows == 16) {
        if (a.rank <= 16) hipLaunchKernelGGL((shrink_kernel<T, 1, 1>), grid, wg, 0, s, a);
        else hipLaunchKernelGGL((shrink_kernel<T, 2, 1>), grid, wg, 0, s, a);
    } else if (a.rank <= 16) {
        hipLaunchKernelGGL((shrink_kernel<T, 1, 4>), grid, wg, 0, s, a);
    } else if (a.rank <= 32) {
        hipLaunchKernelGGL((shrink_kernel<T, 2, 4>), grid, wg, 0, s, a);
    } else {
        hipLaunchKernelGGL((shrink_kernel<T, 4, 4>), grid, wg, 0, s, a);
    }
}
template <typename T, int KT>
void launch_expand(LoraArgs& a, unsigned tiles, hipStream_t s) {
    // half a tile of 64 a workgroup, but of rank 64 (33..64), whose B would be read
    // twice as often: 4099 rows of 37888 outputs, whole and halves: rank 16 174 and
    // 172 us (of 3584 76 and 72), rank 64 194 and 209, rank 128 345 and 280.  All bf16:
    // fp32 adapters take the same tiles with up to 256 registers, from rank 33 on one
    // wavefront a SIMD: 1100 rows of 37888 outputs, rank 16, 64 and 128, 80, 152 and 206
    // us (bf16 49, 67 and 84)
    constexpr int RG = KT == 2 ? 4 : 2;
    const unsigned pieces = a.tile_rows == 16 ? tiles : tiles * (4 / RG);
    const int64_t work = (int64_t)pieces * ((a.d_out + 255) / 256);      // workgroups of one block each
    a.blocks = work >= 16384 ? 8 : work >= 8192 ? 4 : work >= 4096 ? 2 : 1;
    const dim3 grid((a.d_out + a.blocks * 256 - 1) / (a.blocks * 256), pieces);
    if (a.tile_rows == 16) hipLaunchKernelGGL((expand_kernel<T, KT, 1>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((expand_kernel<T, KT, RG>), grid, dim3(256), 0, s, a);
}

template <typename T>
hipError_t launch_lora(LoraArgs& a, hipStream_t s) {
    const unsigned tiles = lora_max_tiles(a.n_rows, a.n_adapters);
    launch_shrink<T>(a, tiles, s);
    if (a.rank <= 32) launch_expand<T, 1>(a, tiles, s);
    else if (a.rank <= 64) launch_expand<T, 2>(a, tiles, s);
    else launch_expand<T, 4>(a, tiles, s);
    return hipGetLastError();
}

static buddy_status lora_sizes(const buddy_lora* l, int32_t n_rows) {
    if (!l || n_rows < 0 || !is_dtype(l->dtype) || l->n_adapters < 1 || l->d_in < 1 || l->d_out < 1) return BUDDY_EINVAL;
    if (l->rank < 8 || l->rank > kLoraMaxRank || l->rank % 8 || l->d_in % 8 || l->d_out % 8) return BUDDY_ESHAPE;
    if (l->d_in > (1 << 20) || l->d_out > (1 << 20)) return BUDDY_ESHAPE;
    return l->n_adapters > kLoraMaxAdapters || n_rows > (1 << 20) ? BUDDY_ECAPACITY : BUDDY_OK;
}

}  // namespace buddy

using namespace buddy;

extern "C" {

int64_t buddy_lora_plan_size(int32_t n_rows, int32_t n_adapters) {
    if (n_rows < 0 || n_rows > (1 << 20) || n_adapters < 1 || n_adapters > kLoraMaxAdapters) return 0;
    return kPlanHead + (int64_t)lora_max_tiles(n_rows, n_adapters) * (kTileHead + lora_tile_rows(n_rows, n_adapters));
}

buddy_status buddy_lora_plan(const int32_t* ids, int32_t n_rows, int32_t n_adapters, int32_t* plan, void* stream) {
    if (n_rows < 0 || n_adapters < 1) return BUDDY_EINVAL;
    if (buddy_lora_plan_size(n_rows, n_adapters) == 0) return BUDDY_ECAPACITY;
    if (n_rows == 0) return BUDDY_OK;
    if (!ids || !plan || ((uintptr_t)plan & 15)) return BUDDY_EINVAL;
    const LoraPlanArgs a{ids, n_rows, n_adapters, lora_tile_rows(n_rows, n_adapters), plan};
    hipStream_t s = (hipStream_t)stream;
    if (n_adapters < 1024) hipLaunchKernelGGL((lora_plan_kernel<1>), dim3(1), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((lora_plan_kernel<kLoraMaxAdapters / 1024 + 1>), dim3(1), dim3(1024), 0, s, a);
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

size_t buddy_lora_workspace(const buddy_lora* l, int32_t n_rows) {
    if (lora_sizes(l, n_rows) != BUDDY_OK) return 0;
    return 16 + (size_t)lora_part_rows(n_rows) * l->rank * 4;
}

buddy_status buddy_lora_add(const buddy_lora* l, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                            void* out, int64_t out_stride, int32_t n_rows, const int32_t* plan, void* workspace,
                            size_t workspace_bytes, void* stream) {
    const buddy_status st = lora_sizes(l, n_rows);
    if (st != BUDDY_OK) return st;
    if (!l->a || !l->b || !l->scale || ((uintptr_t)l->a & 15) || ((uintptr_t)l->b & 15)) return BUDDY_EINVAL;
    if (n_rows == 0) return BUDDY_OK;
    const int size = l->dtype == BUDDY_BF16 ? 2 : 4;
    if (!plan || ((uintptr_t)plan & 15) || !rows16(x, x_stride, l->d_in, n_rows, size) ||
        !rows16(y, y_stride, l->d_out, n_rows, size) || !rows16(out, out_stride, l->d_out, n_rows, size) ||
        (y == out && y_stride != out_stride && n_rows > 1) || !workspace || ((uintptr_t)workspace & 15) ||
        workspace_bytes < buddy_lora_workspace(l, n_rows))
        return BUDDY_EINVAL;
    LoraArgs a = {};
    a.a = (const char*)l->a; a.b = (const char*)l->b; a.scale = l->scale;
    a.x = (const char*)x; a.x_stride = x_stride * size;
    a.y = (const char*)y; a.y_stride = y_stride * size;
    a.out = (char*)out; a.out_stride = out_stride * size;
    a.plan = plan; a.part = (float*)workspace;
    a.n_rows = n_rows; a.n_adapters = l->n_adapters; a.tile_rows = lora_tile_rows(n_rows, l->n_adapters); a.rank = l->rank; a.d_in = l->d_in; a.d_out = l->d_out;
    a.parts = lora_parts(l, n_rows); a.in_place = y == out;
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = size == 2 ? launch_lora<bf16_t>(a, s) : launch_lora<float>(a, s);
    return e == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

}  // extern "C"
