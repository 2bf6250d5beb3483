// The residual's addition with its norm, and rows of 8-bit elements: written
// (of plain or gated values) and read back, with their C ABI.
#include "mx8.h"
#include "epilogue.h"

namespace buddy {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E;

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_mov_u(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}

__device__ __forceinline__ uint4 get16(const char* p) { return *reinterpret_cast<const uint4*>(p); }

// Eight elements.
__device__ __forceinline__ void load8(const char* p, float* x, bf16_t) { unpack<bf16_t>(get16(p), x); }
__device__ __forceinline__ void load8(const char* p, float* x, float) {
    unpack<float>(get16(p), x);
    unpack<float>(get16(p + 16), x + 4);
}
__device__ __forceinline__ void store8(char* p, const float* x, bf16_t) {
    uint4 w;
    w.x = f2bf(x[0]) | (uint32_t)f2bf(x[1]) << 16;
    w.y = f2bf(x[2]) | (uint32_t)f2bf(x[3]) << 16;
    w.z = f2bf(x[4]) | (uint32_t)f2bf(x[5]) << 16;
    w.w = f2bf(x[6]) | (uint32_t)f2bf(x[7]) << 16;
    *reinterpret_cast<uint4*>(p) = w;
}
__device__ __forceinline__ void store8(char* p, const float* x, float) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 16) = make_float4(x[4], x[5], x[6], x[7]);
}

// A lane's eight elements as e4m3 codes of its group's scale.  A group is the
// four lanes of a quad; lanes behind a row's end bring zeros.
__device__ __forceinline__ uint2 quantise8(const float* x, int* scale_code) {
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(x[i]) & 0x7fffffffu);   // NaN above all
    amax = max(amax, dpp_mov_u<kDppXor1>(amax));
    amax = max(amax, dpp_mov_u<kDppXor2>(amax));
    const int code = mx8_scale_code(amax);
    *scale_code = code;
    if (code == kMx8NanScale) return make_uint2(0, 0);
    // 2^-e: scaled values are at most 448, exact down to subnormal fp32
    // numbers, which are far below half of the least e4m3 value
    const float s = __uint_as_float((uint32_t)(254 - code) << 23);
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * s, x[1] * s, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * s, x[3] * s, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4] * s, x[5] * s, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6] * s, x[7] * s, hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// ------------------------------------------------------- addition and norm
//
// y = h' rsqrt(mean h'^2 + eps) w of h' = h + delta.  A workgroup takes a row
// and holds it in registers, eight elements of each 8-element piece a lane, so
// everything is read and written once; the sum of squares crosses the
// wavefronts through LDS.  Bound: memory (few rows: a launch).  8192 rows of 5120,
// fp32 residual, bf16 delta, 8-bit rows: 81 us, 5.1 TB/s; one row 3.4.
struct NormArgs {
    const char *h, *delta, *w;
    char *h_out, *y;
    uint8_t *codes, *scales;
    int64_t h_stride, delta_stride, h_out_stride, y_stride, code_stride, scale_stride;   // bytes
    const int32_t* pos;
    int32_t n_rows, width;
    float eps;
};

// H: type of h, T: type of the rest; N pieces a lane.
template <typename H, typename T, int N>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a) {
    __shared__ float s_sum[2][16];
    const int tid = threadIdx.x, threads = blockDim.x;
    const int pieces = a.width / 8;
    int turn = 0;                        // half of s_sum, by turns over the rows that are not padding
    for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
        if (a.pos && a.pos[row] < 0) continue;
        float x[N][8], w[N][8];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = tid + i * threads;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = w[i][e] = 0.f;
            if (p >= pieces) continue;
            load8(a.h + row * a.h_stride + (int64_t)p * 8 * sizeof(H), x[i], H());
            load8(a.w + (int64_t)p * 8 * sizeof(T), w[i], T());
            if (a.delta) {
                float d[8];
                load8(a.delta + row * a.delta_stride + (int64_t)p * 8 * sizeof(T), d, T());
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] += d[e];
                if (sizeof(H) == 2) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[i][e] = bf2f(f2bf(x[i][e]));
                }
                store8(a.h_out + row * a.h_out_stride + (int64_t)p * 8 * sizeof(H), x[i], H());
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float t[4];                                  // squares added pair by pair
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = x[i][e] * x[i][e] + x[i][e + 4] * x[i][e + 4];
            sum += (t[0] + t[1]) + (t[2] + t[3]);
        }
        sum = wave_sum(sum);
        if (threads > kWave) {
            if ((tid & 63) == 0) s_sum[turn][tid >> 6] = sum;
            // the next live row's sums go into the other half, whose barrier keeps
            // those of the row after it from here
            __syncthreads();
            sum = 0.f;
            for (int i = 0; i < threads / kWave; ++i) sum += s_sum[turn][i];
            turn ^= 1;
        }
        const float r = 1.0f / sqrtf(sum / (float)a.width + a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = tid + i * threads;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = p < pieces ? x[i][e] * r * w[i][e] : 0.f;
            if (a.y && p < pieces) store8(a.y + row * a.y_stride + (int64_t)p * 8 * sizeof(T), y, T());
            if (a.codes) {
                int code;
                const uint2 c = quantise8(y, &code);
                if (p < pieces) {
                    *reinterpret_cast<uint2*>(a.codes + row * a.code_stride + (int64_t)p * 8) = c;
                    if ((p & 3) == 0) a.scales[row * a.scale_stride + (p >> 2)] = (uint8_t)code;
                }
            }
        }
    }
}

template <typename H, typename T>
hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
    // pieces a lane: the row over at least a wavefront and at most 1024 lanes
    const int pieces = a.width / 8;
    const int n = pieces <= 256 ? 1 : pieces <= 1024 ? 2 : 4;
    const int lanes = ((pieces + n - 1) / n + 63) / 64 * 64;
    const dim3 grid(a.n_rows < (1 << 20) ? a.n_rows : 1 << 20), wg(lanes);
    if (n == 1) hipLaunchKernelGGL((norm_kernel<H, T, 1>), grid, wg, 0, s, a);
    else if (n == 2) hipLaunchKernelGGL((norm_kernel<H, T, 2>), grid, wg, 0, s, a);
    else hipLaunchKernelGGL((norm_kernel<H, T, 4>), grid, wg, 0, s, a);
    return hipGetLastError();
}

// ------------------------------------------------------------- 8-bit rows
//
// A lane takes eight elements, four lanes a group, whole groups of the rows
// one behind another.  Bound: memory.  8195 rows of 4096, bf16: 24.7 us written and
// 20.4 read back (4.1 and 5.0 TB/s); 64 gated rows of 18944 4.4.
struct Rows8Args {
    uint8_t *codes, *scales;
    const char *x, *gate;                // quantise
    char* out;                           // read
    int64_t code_stride, scale_stride, x_stride, gate_stride, out_stride;   // bytes
    const int32_t* pos;
    int32_t n_rows, width, row_lanes;    // lanes of a row, whole groups
};

template <typename T, bool GATE>
__global__ __launch_bounds__(256) void quantise_kernel(Rows8Args a) {
    const int64_t step = (int64_t)gridDim.x * 256, end = (int64_t)a.n_rows * a.row_lanes;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < end; at += step) {   // quads stay whole
        const int64_t row = at / a.row_lanes;
        const int p = (int)(at - row * a.row_lanes);
        if (a.pos && a.pos[row] < 0) continue;
        const bool there = p * 8 < a.width;
        float x[8] = {};
        if (there) {
            load8(a.x + row * a.x_stride + (int64_t)p * 8 * sizeof(T), x, T());
            if (GATE) {
                float g[8];
                load8(a.gate + row * a.gate_stride + (int64_t)p * 8 * sizeof(T), g, T());
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = swiglu(g[e], x[e]);
            }
        }
        int code;
        const uint2 c = quantise8(x, &code);
        if (!there) continue;
        *reinterpret_cast<uint2*>(a.codes + row * a.code_stride + (int64_t)p * 8) = c;
        if ((p & 3) == 0) a.scales[row * a.scale_stride + (p >> 2)] = (uint8_t)code;
    }
}

template <typename T>
__global__ __launch_bounds__(256) void read8_kernel(Rows8Args a) {
    const int64_t step = (int64_t)gridDim.x * 256, end = (int64_t)a.n_rows * a.row_lanes;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < end; at += step) {
        const int64_t row = at / a.row_lanes;
        const int p = (int)(at - row * a.row_lanes);
        const uint2 c = *reinterpret_cast<const uint2*>(a.codes + row * a.code_stride + (int64_t)p * 8);
        const int code = a.scales[row * a.scale_stride + (p >> 2)];
        const float s = code == kMx8NanScale ? __uint_as_float(0x7fc00000u)
                        : code == 0          ? 0x1p-127f
                                             : __uint_as_float((uint32_t)code << 23);
        float x[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t word = h ? c.y : c.x;
            const f32x2_t u = __builtin_amdgcn_cvt_pk_f32_fp8(word, false), v = __builtin_amdgcn_cvt_pk_f32_fp8(word, true);
            x[4 * h] = u[0] * s;
            x[4 * h + 1] = u[1] * s;
            x[4 * h + 2] = v[0] * s;
            x[4 * h + 3] = v[1] * s;
        }
        store8(a.out + row * a.out_stride + (int64_t)p * 8 * sizeof(T), x, T());
    }
}

inline dim3 rows8_grid(const Rows8Args& a) {
    const int64_t blocks = ((int64_t)a.n_rows * a.row_lanes + 255) / 256;
    return dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20));
}

}  // namespace buddy

using namespace buddy;

extern "C" {

buddy_status buddy_add_rmsnorm(const buddy_norm* n, void* stream) {
    if (!n || n->n_rows < 0 || n->width < 1) return BUDDY_EINVAL;
    if (!is_dtype(n->hidden_dtype) || !is_dtype(n->dtype) || !(n->rms_eps >= 0.f)) return BUDDY_EINVAL;
    if (n->width % 16 || n->width > 32768) return BUDDY_ESHAPE;
    if (n->n_rows > kMaxRows) return BUDDY_ECAPACITY;
    if ((!n->y && !n->y_mx8) || (n->delta ? !n->h_out : n->h_out != nullptr)) return BUDDY_EINVAL;
    const int hs = n->hidden_dtype == BUDDY_BF16 ? 2 : 4, ts = n->dtype == BUDDY_BF16 ? 2 : 4;
    if (n->y_mx8) {
        if (n->y_mx8->n_rows != n->n_rows || n->y_mx8->width != n->width) return BUDDY_EINVAL;
        const buddy_status st = mx8_check(n->y_mx8);
        if (st != BUDDY_OK) return st;
    }
    if (n->n_rows == 0) return BUDDY_OK;
    if (!n->weight || ((uintptr_t)n->weight & 15) || !rows16(n->h, n->h_stride, n->width, n->n_rows, hs) ||
        (n->delta && (!rows16(n->delta, n->delta_stride, n->width, n->n_rows, ts) ||
                      !rows16(n->h_out, n->h_out_stride, n->width, n->n_rows, hs) ||
                      (n->h_out == n->h && n->h_out_stride != n->h_stride && n->n_rows > 1))) ||
        (n->y && !rows16(n->y, n->y_stride, n->width, n->n_rows, ts)))
        return BUDDY_EINVAL;
    NormArgs a = {};
    a.h = (const char*)n->h; a.h_stride = n->h_stride * hs;
    a.delta = (const char*)n->delta; a.delta_stride = n->delta_stride * ts;
    a.w = (const char*)n->weight;
    a.h_out = (char*)n->h_out; a.h_out_stride = n->h_out_stride * hs;
    a.y = (char*)n->y; a.y_stride = n->y_stride * ts;
    if (n->y_mx8) {
        a.codes = n->y_mx8->codes; a.code_stride = n->y_mx8->code_stride;
        a.scales = n->y_mx8->scales; a.scale_stride = n->y_mx8->scale_stride;
    }
    a.pos = n->pos; a.n_rows = n->n_rows; a.width = n->width; a.eps = n->rms_eps;
    hipStream_t s = (hipStream_t)stream;
    hipError_t e;
    if (hs == 4) e = ts == 4 ? launch_norm<float, float>(a, s) : launch_norm<float, bf16_t>(a, s);
    else e = ts == 4 ? launch_norm<bf16_t, float>(a, s) : launch_norm<bf16_t, bf16_t>(a, s);
    return e == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

buddy_status buddy_mx8_quantize(const buddy_mx8* out, int32_t dtype, const void* x, int64_t x_stride, const void* gate,
                                int64_t gate_stride, const int32_t* pos, void* stream) {
    const buddy_status st = mx8_check(out);
    if (st != BUDDY_OK) return st;
    if (!is_dtype(dtype)) return BUDDY_EINVAL;
    if (out->n_rows == 0) return BUDDY_OK;
    const int size = dtype == BUDDY_BF16 ? 2 : 4;
    if (!rows16(x, x_stride, out->width, out->n_rows, size) ||
        (gate && !rows16(gate, gate_stride, out->width, out->n_rows, size)))
        return BUDDY_EINVAL;
    Rows8Args a = {};
    a.codes = out->codes; a.code_stride = out->code_stride;
    a.scales = out->scales; a.scale_stride = out->scale_stride;
    a.x = (const char*)x; a.x_stride = x_stride * size;
    a.gate = (const char*)gate; a.gate_stride = gate_stride * size;
    a.pos = pos; a.n_rows = out->n_rows; a.width = out->width;
    a.row_lanes = (out->width + kMx8Group - 1) / kMx8Group * 4;
    const dim3 grid = rows8_grid(a), wg(256);
    hipStream_t s = (hipStream_t)stream;
    if (size == 2) {
        if (gate) hipLaunchKernelGGL((quantise_kernel<bf16_t, true>), grid, wg, 0, s, a);
        else hipLaunchKernelGGL((quantise_kernel<bf16_t, false>), grid, wg, 0, s, a);
    } else {
        if (gate) hipLaunchKernelGGL((quantise_kernel<float, true>), grid, wg, 0, s, a);
        else hipLaunchKernelGGL((quantise_kernel<float, false>), grid, wg, 0, s, a);
    }
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

buddy_status buddy_mx8_read(const buddy_mx8* m, int32_t dtype, void* out, int64_t out_stride, void* stream) {
    const buddy_status st = mx8_check(m);
    if (st != BUDDY_OK) return st;
    if (!is_dtype(dtype)) return BUDDY_EINVAL;
    if (m->n_rows == 0) return BUDDY_OK;
    const int size = dtype == BUDDY_BF16 ? 2 : 4;
    if (!rows16(out, out_stride, m->width, m->n_rows, size)) return BUDDY_EINVAL;
    Rows8Args a = {};
    a.codes = m->codes; a.code_stride = m->code_stride;
    a.scales = m->scales; a.scale_stride = m->scale_stride;
    a.out = (char*)out; a.out_stride = out_stride * size;
    a.n_rows = m->n_rows; a.width = m->width;
    a.row_lanes = m->width / 8;
    const dim3 grid = rows8_grid(a), wg(256);
    hipStream_t s = (hipStream_t)stream;
    if (size == 2) hipLaunchKernelGGL((read8_kernel<bf16_t>), grid, wg, 0, s, a);
    else hipLaunchKernelGGL((read8_kernel<float>), grid, wg, 0, s, a);
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

}  // extern "C"
