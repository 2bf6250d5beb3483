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
constexpr int kShrinkParts = 8;          // parts of a sum over d_in

// Rows of a tile, by the rows of the call alone, so that a plan and the calls
// that use it agree.
__host__ __device__ inline int lora_tile_rows(int n_rows) { return n_rows >= 1024 ? 64 : 16; }
// Tiles at most: every group of rows (an adapter's or none's) ends in one that
// is not full.
__host__ __device__ inline int lora_max_tiles(int n_rows, int n_adapters) {
    const int groups = n_rows < n_adapters + 1 ? n_rows : n_adapters + 1;
    return n_rows / lora_tile_rows(n_rows) + groups;
}

// ------------------------------------------------------------------- plan
//
// One workgroup: rows of each adapter are counted in LDS, prefix sums give each
// adapter's first row and tile, then rows and tiles are written.  Rows of one
// adapter come in no fixed order: a row's result does not depend on it.
struct LoraPlanArgs { const int32_t* ids; int32_t n_rows, n_adapters; int32_t* plan; };

__global__ __launch_bounds__(1024) void lora_plan_kernel(LoraPlanArgs a) {
    constexpr int kPer = (kLoraMaxAdapters + 1 + 1023) / 1024;   // groups of a thread
    __shared__ int s_n[kPer * 1024], s_first[kPer * 1024], s_wave[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int T = lora_tile_rows(a.n_rows);
    for (int i = tid; i < kPer * 1024; i += 1024) s_n[i] = 0;
    __syncthreads();
    auto group = [&](int r) {             // -1 none is group 0; others no group
        const int id = a.ids[r];
        return id >= -1 && id < a.n_adapters ? id + 1 : -1;
    };
    for (int r = tid; r < a.n_rows; r += 1024) {
        const int g = group(r);
        if (g >= 0) atomicAdd(&s_n[g], 1);
    }
    __syncthreads();
    int rows = 0, tiles = 0;              // of this thread's groups
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int n = s_n[tid * kPer + i];
        rows += n;
        tiles += (n + T - 1) / T;
    }
    int r_end = rows, t_end = tiles;      // inclusive sums over the wavefront
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(r_end, d), v = __shfl_up(t_end, d);
        if (lane >= d) { r_end += u; t_end += v; }
    }
    if (lane == 63) { s_wave[0][wave] = r_end; s_wave[1][wave] = t_end; }
    __syncthreads();
    int row = r_end - rows, tile = t_end - tiles, all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) { row += s_wave[0][w]; tile += s_wave[1][w]; }
        all += s_wave[1][w];
    }
    int4* out = reinterpret_cast<int4*>(a.plan + kPlanHead);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int g = tid * kPer + i, n = s_n[g];
        s_first[g] = row;
        for (int at = 0; at < n; at += T) out[tile++] = make_int4(g - 1, row + at, min(T, n - at), 0);
        row += n;
    }
    if (tid == 0) {
        a.plan[0] = all;
        a.plan[1] = a.n_rows;
        a.plan[2] = a.n_adapters;
        a.plan[3] = T;
    }
    __syncthreads();
    int32_t* order = a.plan + kPlanHead + 4 * lora_max_tiles(a.n_rows, a.n_adapters);
    for (int r = tid; r < a.n_rows; r += 1024) {
        const int g = group(r);
        if (g >= 0) order[atomicAdd(&s_first[g], 1)] = r;
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
    int32_t n_rows, n_adapters, rank, d_in, d_out, parts, in_place;
};

// A tile of the plan: its adapter, and its rows from `order` on.  A plan that
// does not fit the call has no tiles.
struct Tile { int adapter, count; const int32_t* order; };
__device__ __forceinline__ Tile tile_of(const LoraArgs& a, int t) {
    Tile none = {-1, 0, nullptr};
    if (a.plan[1] != a.n_rows || a.plan[2] != a.n_adapters || a.plan[3] != lora_tile_rows(a.n_rows)) return none;
    const int most = lora_max_tiles(a.n_rows, a.n_adapters);
    if (t >= a.plan[0] || t >= most) return none;
    const int4 v = reinterpret_cast<const int4*>(a.plan + kPlanHead)[t];
    if (v.x < -1 || v.x >= a.n_adapters || v.y < 0 || v.z < 1 || v.z > lora_tile_rows(a.n_rows) || v.y > a.n_rows - v.z) return none;
    return Tile{v.x, v.z, a.plan + kPlanHead + 4 * most + v.y};
}
// Row i of a tile, -1 for one that it does not have.
__device__ __forceinline__ int row_of(const LoraArgs& a, const Tile& t, int i) {
    if (i >= t.count) return -1;
    const int r = t.order[i];
    return (uint32_t)r < (uint32_t)a.n_rows ? r : -1;
}

__device__ __forceinline__ float dot8(const uint4& p, const uint4& q, float s, bf16_t) {
    float u[8], v[8];
    unpack<bf16_t>(p, u);
    unpack<bf16_t>(q, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(u[i], v[i], s);
    return s;
}
__device__ __forceinline__ float dot8(const uint4& p, const uint4& q, float s, float) {
    float u[4], v[4];
    unpack<float>(p, u);
    unpack<float>(q, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(u[i], v[i], s);
    return s;
}

// t[r][j] over a part of d_in: a wavefront a (row, j), its lanes over k.
template <typename T>
__global__ __launch_bounds__(256) void shrink_kernel(LoraArgs a) {
    const Tile t = tile_of(a, blockIdx.x);
    if (t.count == 0 || t.adapter < 0) return;
    constexpr int E = 16 / sizeof(T);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int units = a.d_in / E;
    const int first = (int)((int64_t)units * blockIdx.y / a.parts), last = (int)((int64_t)units * (blockIdx.y + 1) / a.parts);
    for (int at = wave; at < t.count * a.rank; at += 4) {
        const int i = at / a.rank, j = at - i * a.rank, r = row_of(a, t, i);
        if (r < 0) continue;
        const uint4* x = reinterpret_cast<const uint4*>(a.x + r * a.x_stride);
        const uint4* w = reinterpret_cast<const uint4*>(a.a + ((int64_t)t.adapter * a.rank + j) * a.d_in * sizeof(T));
        float s = 0.f;
        for (int k = first + lane; k < last; k += 64) s = dot8(x[k], w[k], s, T());
        s = wave_sum(s);
        if (lane == 0) a.part[((int64_t)blockIdx.y * a.n_rows + r) * a.rank + j] = s;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void expand_kernel(LoraArgs a) {
    __shared__ float s_t[kLoraMaxRank];
    const Tile t = tile_of(a, blockIdx.x);
    if (t.count == 0 || (t.adapter < 0 && a.in_place)) return;
    const int n = blockIdx.y * 256 + threadIdx.x;
    const float scale = t.adapter < 0 ? 0.f : a.scale[t.adapter];
    for (int i = 0; i < t.count; ++i) {
        const int r = row_of(a, t, i);
        __syncthreads();
        if (t.adapter >= 0 && r >= 0 && (int)threadIdx.x < a.rank) {
            float s = 0.f;
            for (int p = 0; p < a.parts; ++p) s += a.part[((int64_t)p * a.n_rows + r) * a.rank + threadIdx.x];
            s_t[threadIdx.x] = s;
        }
        __syncthreads();
        if (r < 0 || n >= a.d_out) continue;
        const T* y = (const T*)(a.y + r * a.y_stride);
        T* o = (T*)(a.out + r * a.out_stride);
        if (t.adapter < 0) {
            o[n] = y[n];
            continue;
        }
        const T* b = (const T*)a.b + ((int64_t)t.adapter * a.d_out + n) * a.rank;
        float s = 0.f;
        for (int j = 0; j < a.rank; ++j) s = fmaf(St<T>::get(b, j), s_t[j], s);
        St<T>::put(o, n, fmaf(scale, s, St<T>::get(y, n)));
    }
}

template <typename T>
hipError_t launch_lora(const LoraArgs& a, hipStream_t s) {
    const unsigned tiles = lora_max_tiles(a.n_rows, a.n_adapters);
    hipLaunchKernelGGL((shrink_kernel<T>), dim3(tiles, a.parts), dim3(256), 0, s, a);
    hipLaunchKernelGGL((expand_kernel<T>), dim3(tiles, (a.d_out + 255) / 256), dim3(256), 0, s, a);
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
    return kPlanHead + 4 * (int64_t)lora_max_tiles(n_rows, n_adapters) + n_rows;
}

buddy_status buddy_lora_plan(const int32_t* ids, int32_t n_rows, int32_t n_adapters, int32_t* plan, void* stream) {
    if (n_rows < 0 || n_adapters < 1) return BUDDY_EINVAL;
    if (buddy_lora_plan_size(n_rows, n_adapters) == 0) return BUDDY_ECAPACITY;
    if (n_rows == 0) return BUDDY_OK;
    if (!ids || !plan || ((uintptr_t)plan & 15)) return BUDDY_EINVAL;
    const LoraPlanArgs a{ids, n_rows, n_adapters, plan};
    hipLaunchKernelGGL(lora_plan_kernel, dim3(1), dim3(1024), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

size_t buddy_lora_workspace(const buddy_lora* l, int32_t n_rows) {
    if (lora_sizes(l, n_rows) != BUDDY_OK) return 0;
    return 16 + (size_t)kShrinkParts * n_rows * l->rank * 4;
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
    a.n_rows = n_rows; a.n_adapters = l->n_adapters; a.rank = l->rank; a.d_in = l->d_in; a.d_out = l->d_out;
    a.parts = kShrinkParts; a.in_place = y == out;
    hipStream_t s = (hipStream_t)stream;
    const hipError_t e = size == 2 ? launch_lora<bf16_t>(a, s) : launch_lora<float>(a, s);
    return e == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

}  // extern "C"
