// A token for each row of logits by temperature, top-k, min-p, top-p and a given
// random number (buddy_sample).
//
// Weights are whole numbers, exp((l - max) / T) in units of 2^-40, so sums of
// them are exact in 64 bits and neither atomics nor the split of a row decide
// anything.  Every criterion keeps a prefix of the tokens by falling logit, so
// nothing is sorted: a histogram over the distance from the largest logit gives
// the bin in which a criterion ends, and histograms over the keys (the logits'
// bits, ordered as whole numbers) within that bin give the last key and how
// many of the tokens with that key still belong.
#include "mx8.h"

namespace buddy {

constexpr int kSampleThreads = 1024;
constexpr int kBins = 2048;
constexpr int kListed = 4096;            // tokens of a bin that are kept in LDS
constexpr int kMaxVocab = 1 << 20;
constexpr double kReach = 28.5;          // exp(-28.5) < 2^-41: weight 0
constexpr uint64_t kUnit = 1ull << 40;   // the largest logit's weight

struct SampleArgs {
    const char* logits;
    int64_t stride;                      // bytes
    int32_t B, vocab;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* token;
};

// Logits as whole numbers of the same order; both zeros are one, NaN counts as -inf.
constexpr uint32_t kNegInfKey = 0x007fffffu;
__device__ __forceinline__ uint32_t key_of(float l) {
    uint32_t u = __float_as_uint(l);
    if ((u & 0x7fffffffu) > 0x7f800000u) return kNegInfKey;
    if (u == 0x80000000u) u = 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// A row's weights: rint(2^40 exp((l - max) / T)).  exp by reduction to
// |r| <= ln 2 / 2 and the Taylor series to r^12, off by about 2e-16 of its value.
struct Weights {
    float max;
    double inv_t;
    float per_bin;                       // bins for each unit of distance
    __device__ uint64_t weight(float l) const {
        if (l == max) return kUnit;
        const double z = ((double)l - (double)max) * inv_t;
        if (!(z > -kReach)) return 0;
        const double n = rint(z * 1.4426950408889634);
        const double r = fma(n, -2.3190468138462996e-17, fma(n, -0.6931471805599453, z));   // ln 2 in two parts
        double p = 1.0 / 479001600.0;
        p = fma(p, r, 1.0 / 39916800.0);
        p = fma(p, r, 1.0 / 3628800.0);
        p = fma(p, r, 1.0 / 362880.0);
        p = fma(p, r, 1.0 / 40320.0);
        p = fma(p, r, 1.0 / 5040.0);
        p = fma(p, r, 1.0 / 720.0);
        p = fma(p, r, 1.0 / 120.0);
        p = fma(p, r, 1.0 / 24.0);
        p = fma(p, r, 1.0 / 6.0);
        p = fma(p, r, 0.5);
        p = fma(p, r, 1.0);
        p = fma(p, r, 1.0);
        const double scale = __longlong_as_double((int64_t)((int)n + 40 + 1023) << 52);
        return (uint64_t)rint(p * scale);
    }
    // rises with falling l
    __device__ int bin(float l) const {
        if (l == max) return 0;
        return (int)fminf((max - l) * per_bin, (float)(kBins - 1));
    }
};

// A row in 16-byte units, from the aligned unit that its first element is in;
// elements outside the row are skipped, and not read.
template <typename T>
struct Row {
    static constexpr int E = 16 / sizeof(T);
    const T* base;                       // aligned, at most E - 1 elements before the row
    int skip, end, units;                // elements before the row, before its end, units
    __device__ Row(const char* p, int vocab) {
        skip = (int)(((uintptr_t)p & 15) / sizeof(T));
        base = (const T*)p - skip;
        end = skip + vocab;
        units = (end + E - 1) / E;
    }
    // f(index, logit) for the elements of unit q in order
    template <typename F>
    __device__ void unit(int q, F f) const {
        const int at = q * E;
        if (at >= skip && at + E <= end) {
            float v[E];
            unpack<T>(*reinterpret_cast<const uint4*>(base + at), v);
#pragma unroll
            for (int e = 0; e < E; ++e) f(at - skip + e, v[e]);
        } else {
            for (int e = 0; e < E; ++e)
                if (at + e >= skip && at + e < end) f(at - skip + e, St<T>::get(base, at + e));
        }
    }
    template <typename F>
    __device__ void all(F f) const {
        for (int q = threadIdx.x; q < units; q += kSampleThreads) unit(q, f);
    }
};

__device__ __forceinline__ uint64_t shfl_up64(uint64_t v, int d) { return __shfl_up((unsigned long long)v, d); }

struct SampleShared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t wave_mass[16];
    uint32_t wave_count[16];
    uint32_t list[kListed];              // keys
    uint64_t block_mass[kMaxVocab / 256 + 1];   // of 64 units each
    uint32_t block_ties[kMaxVocab / 256 + 1];
    uint32_t listed, key_min, key_max;
    uint64_t red;
    // what a search found
    uint64_t found_mass;
    uint32_t found_count, found_at;
};

// Inclusive prefix sums over the workgroup.
__device__ __forceinline__ void scan(SampleShared& s, uint64_t& m, uint32_t& c) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t um = shfl_up64(m, d);
        const uint32_t uc = __shfl_up(c, d);
        if (lane >= d) { m += um; c += uc; }
    }
    __syncthreads();
    if (lane == 63) { s.wave_mass[wave] = m; s.wave_count[wave] = c; }
    __syncthreads();
    for (int w = 0; w < wave; ++w) { m += s.wave_mass[w]; c += s.wave_count[w]; }
}

// The first bin of the histogram at which the running count (by mass: the
// running mass) reaches target, and what lies before it: found_*.
__device__ void find(SampleShared& s, bool by_mass, uint64_t target) {
    __syncthreads();
    const int b = threadIdx.x * 2;
    const uint64_t m0 = s.mass[b], m1 = s.mass[b + 1];
    const uint32_t c0 = s.count[b], c1 = s.count[b + 1];
    uint64_t m = m0 + m1;
    uint32_t c = c0 + c1;
    scan(s, m, c);
    const uint64_t v = by_mass ? m : c, before = v - (by_mass ? m0 + m1 : c0 + c1), half = before + (by_mass ? m0 : c0);
    if (before < target && target <= v) {
        const bool second = half < target;
        s.found_at = b + second;
        s.found_mass = m - m1 - (second ? 0 : m0);
        s.found_count = c - c1 - (second ? 0 : c0);
    }
    __syncthreads();
}

// Kept: tokens of a key above `key`, and the first `ties` of those with it.
struct Cut { uint32_t key, ties; uint64_t mass; };

// The end of the prefix that reaches target (a count or a mass, at least 1 and
// at most all there is), inside the given bin, before which lie mass and count.
template <typename T>
__device__ Cut cut_in_bin(SampleShared& s, const Row<T>& row, const Weights& w, int bin, uint64_t mass, uint64_t count, bool by_mass, uint64_t target) {
    if (threadIdx.x == 0) { s.listed = 0; s.key_min = 0xffffffffu; s.key_max = 0; }
    __syncthreads();
    row.all([&](int, float l) {
        if (l != l || w.bin(l) != bin || w.weight(l) == 0) return;
        const uint32_t k = key_of(l), at = atomicAdd(&s.listed, 1u);
        if (at < kListed) s.list[at] = k;
        atomicMin(&s.key_min, k);
        atomicMax(&s.key_max, k);
    });
    __syncthreads();
    const int n = (int)s.listed;
    uint32_t lo = s.key_min, hi = s.key_max;
    for (;;) {
        const int bits = hi > lo ? 32 - __clz(hi - lo) : 0, shift = bits > 11 ? bits - 11 : 0;
        for (int i = threadIdx.x; i < kBins; i += kSampleThreads) { s.mass[i] = 0; s.count[i] = 0; }
        __syncthreads();
        auto add = [&](uint32_t k) {
            if (k < lo || k > hi) return;
            const uint32_t d = (hi - k) >> shift;
            atomicAdd(&s.count[d], 1u);
            atomicAdd((unsigned long long*)&s.mass[d], (unsigned long long)w.weight(logit_of(k)));
        };
        if (n <= kListed) {
            for (int i = threadIdx.x; i < n; i += kSampleThreads) add(s.list[i]);
        } else {
            row.all([&](int, float l) {
                if (l == l && w.bin(l) == bin && w.weight(l) != 0) add(key_of(l));
            });
        }
        find(s, by_mass, target - (by_mass ? mass : count));
        mass += s.found_mass;
        count += s.found_count;
        const uint32_t d = s.found_at;
        const uint32_t top = hi - (d << shift);
        if (shift == 0) {
            const uint64_t each = w.weight(logit_of(top));
            const uint64_t ties = by_mass ? (target - mass + each - 1) / each : target - count;
            __syncthreads();
            return Cut{top, (uint32_t)ties, mass + ties * each};
        }
        const uint32_t span = (1u << shift) - 1;
        hi = top;
        lo = max(lo, top > span ? top - span : 0u);
        __syncthreads();
    }
}

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleArgs a) {
    __shared__ SampleShared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x;
    const Row<T> row(a.logits + b * a.stride, a.vocab);

    // the largest logit, the lowest token that has it
    uint64_t best = 0;
    row.all([&](int i, float l) { best = max(best, (uint64_t)key_of(l) << 32 | (uint32_t)~i); });
    if (tid == 0) s.red = 0;
    __syncthreads();
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, d));
    if (lane == 0) atomicMax((unsigned long long*)&s.red, (unsigned long long)best);
    __syncthreads();
    best = s.red;
    const uint32_t top = (uint32_t)(best >> 32);
    const float temperature = a.temperature[b];
    if (top <= kNegInfKey || !(temperature > 0.f)) {
        if (tid == 0) a.token[b] = top <= kNegInfKey ? -1 : (int)~(uint32_t)best;
        return;
    }
    Weights w;
    w.max = logit_of(top);
    w.inv_t = 1.0 / (double)temperature;
    w.per_bin = (float)(kBins / kReach * w.inv_t);

    // tokens and weight by distance, and the tokens that min_p leaves
    for (int i = tid; i < kBins; i += kSampleThreads) { s.mass[i] = 0; s.count[i] = 0; }
    if (tid == 0) s.red = 0;
    __syncthreads();
    const double least_p = a.min_p ? fmin((double)a.min_p[b], 1.0) * (double)kUnit : 0.0;   // fmin(NaN, 1) = 1: below
    const uint64_t least = a.min_p && a.min_p[b] == a.min_p[b] && least_p > 0.0 ? (uint64_t)ceil(least_p) : 0;
    uint32_t near = 0;
    row.all([&](int, float l) {
        if (l != l) return;
        const uint64_t v = w.weight(l);
        if (v == 0) return;
        near += v >= least;
        const int d = w.bin(l);
        atomicAdd(&s.count[d], 1u);
        atomicAdd((unsigned long long*)&s.mass[d], (unsigned long long)v);
    });
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) near += __shfl_xor(near, d);
    if (lane == 0) atomicAdd((unsigned long long*)&s.red, (unsigned long long)near);
    __syncthreads();
    uint64_t n = s.red;                  // at least the largest logit's
    uint64_t m = s.mass[tid * 2] + s.mass[tid * 2 + 1];
    uint32_t c = s.count[tid * 2] + s.count[tid * 2 + 1];
    scan(s, m, c);
    if (tid == kSampleThreads - 1) { s.found_mass = m; s.found_count = c; }
    __syncthreads();
    const uint64_t all_mass = s.found_mass, all_count = s.found_count;
    const int32_t top_k = a.top_k ? a.top_k[b] : 0;
    if (top_k > 0 && (uint64_t)top_k < n) n = (uint64_t)top_k;

    // both searches start from the same histogram: the second one's bin is
    // found before the first search inside a bin overwrites it
    Cut cut{0, 0, all_mass};             // all
    const float top_p = a.top_p ? a.top_p[b] : 1.f;
    const bool share = top_p < 1.f;
    if (n < all_count) {
        find(s, false, n);
        const int bin = (int)s.found_at;
        const uint64_t before_mass = s.found_mass, before = s.found_count;
        __syncthreads();
        uint64_t kept_mass[2] = {s.mass[tid * 2], s.mass[tid * 2 + 1]};
        uint32_t kept_count[2] = {s.count[tid * 2], s.count[tid * 2 + 1]};
        cut = cut_in_bin(s, row, w, bin, before_mass, before, false, n);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) { s.mass[tid * 2 + i] = kept_mass[i]; s.count[tid * 2 + i] = kept_count[i]; }
        __syncthreads();
    }
    if (share) {
        double need = ceil((double)top_p * (double)cut.mass);
        uint64_t target = need > 1.0 ? (uint64_t)need : 1;
        if (target < cut.mass) {
            find(s, true, target);
            const int bin = (int)s.found_at;
            const uint64_t before_mass = s.found_mass, before = s.found_count;
            __syncthreads();
            cut = cut_in_bin(s, row, w, bin, before_mass, before, true, target);
        }
    }

    // weight and ties of blocks of 64 units, in the order of the vocabulary
    const uint64_t each = cut.ties ? w.weight(logit_of(cut.key)) : 0;
    const int blocks = (row.units + 63) / 64;
    for (int k = wave; k < blocks; k += 16) {
        uint64_t sum = 0;
        uint32_t ties = 0;
        const int q = k * 64 + lane;
        if (q < row.units)
            row.unit(q, [&](int, float l) {
                if (l != l) return;
                const uint32_t key = key_of(l);
                if (key > cut.key) sum += w.weight(l);
                else ties += key == cut.key;
            });
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            sum += (uint64_t)__shfl_xor((unsigned long long)sum, d);
            ties += __shfl_xor(ties, d);
        }
        if (lane == 0) { s.block_mass[k] = sum; s.block_ties[k] = ties; }
    }
    __syncthreads();
    // the block in which the running weight passes floor(u * mass)
    double x = floor((double)a.u[b] * (double)cut.mass);
    uint64_t target = x > 0.0 ? (uint64_t)fmin(x, 0x1p62) : 0;
    if (target >= cut.mass) target = cut.mass - 1;
    const int per = (blocks + kSampleThreads - 1) / kSampleThreads;
    uint64_t sum = 0;
    uint32_t ties = 0;
    for (int k = tid * per; k < min(blocks, (tid + 1) * per); ++k) { sum += s.block_mass[k]; ties += s.block_ties[k]; }
    uint64_t end = sum;
    uint32_t ties_end = ties;
    scan(s, end, ties_end);
    uint64_t at = end - sum;
    uint32_t seen = ties_end - ties;
    auto passed = [&](uint64_t mass, uint32_t t) { return mass + (uint64_t)min(t, cut.ties) * each > target; };
    if (!passed(at, seen) && passed(end, ties_end)) {
        int k = tid * per;
        while (!passed(at + s.block_mass[k], seen + s.block_ties[k])) { at += s.block_mass[k]; seen += s.block_ties[k]; ++k; }
        s.found_at = k;
        s.found_mass = at;
        s.found_count = seen;
    }
    __syncthreads();
    if (wave != 0) return;
    // then the token in it
    const int q = (int)s.found_at * 64 + lane;
    sum = 0;
    ties = 0;
    auto add = [&](float l) {
        const uint32_t key = l == l ? key_of(l) : 0;
        if (key > cut.key) sum += w.weight(l);
        else ties += key == cut.key && cut.ties;
    };
    if (q < row.units) row.unit(q, [&](int, float l) { add(l); });
    at = sum;
    seen = ties;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t um = shfl_up64(at, d);
        const uint32_t uc = __shfl_up(seen, d);
        if (lane >= d) { at += um; seen += uc; }
    }
    const uint64_t mass_end = at + s.found_mass;
    const uint32_t seen_end = seen + s.found_count;
    sum = mass_end - sum;
    ties = seen_end - ties;
    if (!passed(sum, ties) && passed(mass_end, seen_end))
        row.unit(q, [&](int i, float l) {
            if (passed(sum, ties)) return;
            add(l);
            if (passed(sum, ties)) a.token[b] = i;
        });
}

}  // namespace buddy

using namespace buddy;

extern "C" {

size_t buddy_sample_workspace(int32_t B, int32_t vocab) {
    return B < 0 || B > 65535 || vocab < 1 || vocab > kMaxVocab ? 0 : 16;
}

buddy_status buddy_sample(const buddy_sampling* p, void* stream) {
    if (!p || p->B < 0 || p->vocab < 1 || !is_dtype(p->dtype)) return BUDDY_EINVAL;
    if (p->B > 65535 || p->vocab > kMaxVocab) return BUDDY_ECAPACITY;
    if (p->B == 0) return BUDDY_OK;
    const int size = p->dtype == BUDDY_BF16 ? 2 : 4;
    if (!p->logits || (uintptr_t)p->logits % size || p->stride < 0 || p->stride > INT64_MAX / 64 / p->B ||
        (p->B > 1 && p->stride < p->vocab) || !p->temperature || !p->u || !p->token || !p->workspace ||
        ((uintptr_t)p->workspace & 15) || p->workspace_bytes < buddy_sample_workspace(p->B, p->vocab))
        return BUDDY_EINVAL;
    SampleArgs a = {};
    a.logits = (const char*)p->logits; a.stride = p->stride * size; a.B = p->B; a.vocab = p->vocab;
    a.temperature = p->temperature; a.top_k = p->top_k; a.top_p = p->top_p; a.min_p = p->min_p; a.u = p->u; a.token = p->token;
    hipStream_t s = (hipStream_t)stream;
    if (size == 2) hipLaunchKernelGGL((sample_kernel<bf16_t>), dim3(p->B), dim3(kSampleThreads), 0, s, a);
    else hipLaunchKernelGGL((sample_kernel<float>), dim3(p->B), dim3(kSampleThreads), 0, s, a);
    return hipGetLastError() == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

}  // extern "C"
