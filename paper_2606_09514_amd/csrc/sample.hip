// A token for each row of logits by temperature, top-k, min-p, top-p and a given
// random number (buddy_sample).
//
// Weights are whole numbers, exp((l - max) / T) in units of 2^-40, so sums of
// them are exact in 64 bits and neither atomics nor the split of a row decide
// anything.  Every criterion keeps a prefix of the tokens by falling logit, so
// nothing is sorted: a histogram over the distance from the largest logit gives
// the bin in which a criterion ends, and histograms over the keys (the logits'
// bits, ordered as whole numbers) of few tokens give the last key and how many
// of the tokens with that key still belong.
//
// Rows are split into chunks for three kernels that read them: the largest
// logit; the histogram (of counts where top_k limits the tokens, of weights where
// top_p does without it, none and the weights' sums over blocks where neither
// does); a list of the tokens that can hold the end of the prefix (and, without
// top_k, the sums over blocks of what lies before them).  A fourth, a workgroup a
// row, finds the end in the list and then the token.  min_p is a least logit, found
// by search among the keys.  Where the list overflows (a top_k of thousands,
// thousands of equal or nearly equal logits, or a low temperature with fewer than
// top_k tokens within 28.5 T of the largest logit and no min_p, which lists every
// finite one) the fourth reads the whole row, several times.
// Bound: memory for the first reading, then the weights' arithmetic in 64 bits.
// 256 rows of 151001 fp32 logits: 31, 36, 35 and 28 us (5.0 to 4.3 TB/s of the three
// readings); one of 128000: 5, 7, 9 and 15, each a chain of dependent steps.  With
// top_k 40 the fourth takes 13 us for 256 rows and 11.5 for one at a temperature of 1;
// at 0.1 their lists overflow, and it takes 115 and 91, with a top_p 187 and 150.
#include <float.h>

#include "mx8.h"

namespace buddy {

constexpr int kChunkThreads = 512, kChunkWaves = kChunkThreads / 64;
constexpr int kRowThreads = 512, kRowWaves = kRowThreads / 64;
constexpr int kBins = 2048;
constexpr int kListed = 4096;            // tokens of a list
constexpr int kShort = 192;              // tokens that are compared with each other
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxChunks = 64;
constexpr int kBlockUnits = 256;         // 16-byte units of a block
constexpr int kMaxBlocks = kMaxVocab / (4 * kBlockUnits) + 1;
constexpr double kReach = 28.5;          // exp(-28.5) < 2^-41: weight 0
constexpr uint64_t kUnit = 1ull << 40;   // the largest logit's weight

typedef unsigned long long ull;

struct SampleArgs {
    const char* logits;
    int64_t stride;                      // bytes
    int32_t B, vocab, chunks, list, blocks;   // of a row: chunks, places of the list, blocks
    const float *temperature, *top_p, *min_p, *u;
    const int32_t* top_k;
    int32_t* token;
    char* space;
    int64_t row_bytes;
};

// What a row keeps in the workspace.
struct RowSpace {
    uint64_t* hist;                      // [kBins] counts or weights
    uint64_t* best;                      // [kMaxChunks] key and ~token of a chunk's largest logit
    uint64_t* head;                      // before_mass, target (top_p alone); tokens that the list should hold
    uint64_t* blocks;
    uint2* list;                         // key, token
    __device__ RowSpace(const SampleArgs& a, int b) {
        hist = (uint64_t*)(a.space + b * a.row_bytes);
        best = hist + kBins;
        head = best + kMaxChunks;
        blocks = head + 4;
        list = (uint2*)(blocks + a.blocks);
    }
};
inline int64_t row_space_bytes(int list, int blocks) { return ((kBins + kMaxChunks + 4 + (int64_t)blocks + list) * 8 + 15) / 16 * 16; }

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

// A row's weights: rint(2^40 2^y), y = (l - max) / (T ln 2), by 2^f of the rest
// |f| <= 1/2 as the exponential series to the twelfth power (off by 2e-16 of its
// value).  NaN and -inf come out as 0.
struct Weights {
    float max;
    double per_nat;                      // 1 / (T ln 2)
    float per_bin;                       // bins for each unit of distance
    __device__ __forceinline__ uint64_t weight(float l) const {
        const double y = fmax(((double)l - (double)max) * per_nat, -100.0);
        const double n = rint(y), f = y - n;
        double p = 2.5678435993488196e-11;                // ln(2)^k / k!, k = 12 .. 0
        p = fma(p, f, 4.44553827187081e-10);
        p = fma(p, f, 7.054911620801121e-09);
        p = fma(p, f, 1.0178086009239696e-07);
        p = fma(p, f, 1.3215486790144305e-06);
        p = fma(p, f, 1.5252733804059838e-05);
        p = fma(p, f, 0.00015403530393381606);
        p = fma(p, f, 0.0013333558146428441);
        p = fma(p, f, 0.009618129107628477);
        p = fma(p, f, 0.055504108664821576);
        p = fma(p, f, 0.2402265069591007);
        p = fma(p, f, 0.6931471805599453);
        p = fma(p, f, 1.0);
        // at most 2^40: added to 2^52 it is rounded and stands in the low bits
        const double scale = __longlong_as_double((int64_t)((int)n + 40 + 1023) << 52);
        const uint64_t w = (uint64_t)__double_as_longlong(fma(p, scale, 0x1p52)) & ((1ull << 52) - 1);
        return l == max ? kUnit : w;                     // an infinite one too
    }
    // rises with falling l
    __device__ __forceinline__ int bin(float l) const {
        return l == max ? 0 : (int)fminf((max - l) * per_bin, (float)(kBins - 1));
    }
};

// A row in 16-byte units, from the aligned unit that its first element is in;
// elements outside the row are -inf, and not read.  Blocks of 256 units, four to
// a lane of the wavefront that takes one: unit 64 u + lane.
template <typename T>
struct Row {
    static constexpr int E = 16 / sizeof(T);
    const T* base;                       // aligned, at most E - 1 elements before the row
    int skip, end, blocks;               // elements before the row, before its end; blocks
    __device__ Row(const char* p, int vocab) {
        skip = (int)(((uintptr_t)p & 15) / sizeof(T));
        base = (const T*)p - skip;
        end = skip + vocab;
        blocks = (end + E * kBlockUnits - 1) / (E * kBlockUnits);
    }
    __device__ __forceinline__ void unit(int q, float* v) const {
        const int at = q * E;
        if (at >= skip && at + E <= end) {
            unpack<T>(*reinterpret_cast<const uint4*>(base + at), v);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = at + e >= skip && at + e < end ? St<T>::get(base, at + e) : -INFINITY;
        }
    }
    __device__ __forceinline__ int token(int q, int e) const { return q * E + e - skip; }
    // f(unit's token, its E logits) for the four units of a lane, then g(block),
    // over blocks first, first + step ..
    template <typename F, typename G>
    __device__ __forceinline__ void all(int first, int last, int step, F f, G g) const {
        const int lane = threadIdx.x & 63;
        for (int k = first; k < last; k += step) {
            float v[4][E];
#pragma unroll
            for (int u = 0; u < 4; ++u) unit(k * kBlockUnits + 64 * u + lane, v[u]);
#pragma unroll
            for (int u = 0; u < 4; ++u) f(token(k * kBlockUnits + 64 * u + lane, 0), v[u]);
            g(k);
        }
    }
    template <typename F>
    __device__ __forceinline__ void all(int first, int last, int step, F f) const {
        all(first, last, step, f, [](int) {});
    }
};

// ------------------------------------------------------------- reductions

// A value from another lane by DPP, 0 where the row mask or the row's end
// leaves a lane out.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t dpp_or_0(uint64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
    return (uint64_t)hi << 32 | lo;
}
// Inclusive prefix over a wavefront: rows of 16 by shifts of 1, 2, 4 and 8, then
// each row's last lane to the next row and lane 31 to the upper half.
template <typename F>
__device__ __forceinline__ uint64_t wave_prefix(uint64_t v, F f) {
    v = f(v, dpp_or_0<0x111, 0xf>(v));
    v = f(v, dpp_or_0<0x112, 0xf>(v));
    v = f(v, dpp_or_0<0x114, 0xf>(v));
    v = f(v, dpp_or_0<0x118, 0xf>(v));
    v = f(v, dpp_or_0<0x142, 0xa>(v));
    return f(v, dpp_or_0<0x143, 0xc>(v));
}
__device__ __forceinline__ uint64_t last_lane(uint64_t v) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
    return wave_prefix(v, [](uint64_t x, uint64_t y) { return x + y; });
}
__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
    return last_lane(wave_prefix(v, [](uint64_t x, uint64_t y) { return max(x, y); }));
}
__device__ __forceinline__ uint64_t wave_sum64(uint64_t v) {
    if (__ballot(v != 0) == 0) return 0;             // most blocks hold nothing that counts
    return last_lane(wave_scan(v));
}

// What the kernels know of a row once its largest logit is known.
enum SampleMode { MODE_NONE, MODE_LIST, MODE_SHARE, MODE_ALL };
struct RowRule {
    int mode;
    uint64_t best;
    Weights w;
    int64_t top_k;                       // 0: all
    uint32_t floor_key;                  // least key that min_p leaves, 0: all
    float floor;                         // its logit
    double top_p;                        // 1: all
};
// The least key with at least this weight, which that of hi has: 64 places at
// a time.
__device__ __forceinline__ uint32_t least_key(const Weights& w, uint64_t weight, uint32_t hi) {
    const int lane = threadIdx.x & 63;
    uint32_t lo = kNegInfKey;            // weight 0
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + 63) / 64, rest = hi - lo, mine = step * (uint32_t)(lane + 1);
        const uint32_t at = mine < rest ? lo + mine : hi;                // up to 64 steps more than rest: no overflow below 2^26 * 64
        const int first = __builtin_ctzll(__ballot(w.weight(logit_of(at)) >= weight));
        const uint32_t below = first > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)at, first > 0 ? first - 1 : 0) : lo;
        hi = (uint32_t)__builtin_amdgcn_readlane((int)at, first);
        lo = below;
    }
    return hi;
}
__device__ __forceinline__ RowRule rule_of(const SampleArgs& a, const RowSpace& sp, int b) {
    RowRule r = {};
    const int lane = threadIdx.x & 63;
    r.best = wave_max64(lane < a.chunks ? sp.best[lane] : 0);
    const uint32_t top = (uint32_t)(r.best >> 32);
    const float temperature = a.temperature[b], p = a.top_p ? a.top_p[b] : 1.f, m = a.min_p ? a.min_p[b] : 0.f;
    const int32_t k = a.top_k ? a.top_k[b] : 0;
    r.w.max = logit_of(top);
    r.w.per_nat = 1.4426950408889634 / (double)temperature;
    r.w.per_bin = (float)(kBins / kReach / (double)temperature);
    r.top_k = k > 0 && k < a.vocab ? k : 0;
    r.floor = -INFINITY;
    r.top_p = p < 1.f ? (double)p : 1.0;
    r.mode = top <= kNegInfKey || !(temperature > 0.f) ? MODE_NONE : r.top_k ? MODE_LIST : r.top_p < 1.0 ? MODE_SHARE : MODE_ALL;
    if (r.mode != MODE_NONE && m > 0.f) {
        r.floor_key = least_key(r.w, (uint64_t)ceil(fmin((double)m, 1.0) * (double)kUnit), top);
        r.floor = logit_of(r.floor_key);
    }
    return r;
}
// The weight that the tokens kept have to reach.
__device__ __forceinline__ uint64_t share_of(double top_p, uint64_t mass) {
    const double need = ceil(top_p * (double)mass);
    return need > 1.0 ? (uint64_t)need : 1;
}

// ------------------------------------------------------- kernels by chunks

__device__ __forceinline__ void chunk_of(const SampleArgs& a, int blocks, int* first, int* last) {
    *first = (int)((int64_t)blocks * blockIdx.x / a.chunks);
    *last = (int)((int64_t)blocks * (blockIdx.x + 1) / a.chunks);
}

template <typename T>
__global__ __launch_bounds__(kChunkThreads) void sample_max_kernel(SampleArgs a) {
    __shared__ uint64_t s_best[kChunkWaves];
    const int b = blockIdx.y, tid = threadIdx.x, wave = tid >> 6;
    const RowSpace sp(a, b);
    const Row<T> row(a.logits + b * a.stride, a.vocab);
    int first, last;
    chunk_of(a, row.blocks, &first, &last);
    // the largest, and the lowest token that has it
    uint32_t key = 0;
    int token = 0;
    row.all(first + wave, last, kChunkWaves, [&](int t, const float* v) {
#pragma unroll
        for (int e = 0; e < Row<T>::E; ++e) {
            const uint32_t k = key_of(v[e]);
            if (k > key) { key = k; token = t + e; }     // a lane's tokens rise
        }
    });
    const uint64_t best = wave_max64((uint64_t)key << 32 | (uint32_t)~token);
    if ((tid & 63) == 0) s_best[wave] = best;
    for (int i = blockIdx.x * kChunkThreads + tid; i < kBins; i += a.chunks * kChunkThreads) sp.hist[i] = 0;
    if (blockIdx.x == 0 && tid < 4) sp.head[tid] = 0;
    __syncthreads();
    if (tid == 0) {
        uint64_t m = s_best[0];
#pragma unroll
        for (int i = 1; i < kChunkWaves; ++i) m = max(m, s_best[i]);
        sp.best[blockIdx.x] = m;
    }
}

template <typename T>
__global__ __launch_bounds__(kChunkThreads) void sample_hist_kernel(SampleArgs a) {
    __shared__ uint64_t s_hist[kBins];
    const int b = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const RowSpace sp(a, b);
    const RowRule r = rule_of(a, sp, b);
    if (r.mode == MODE_NONE) return;
    const Row<T> row(a.logits + b * a.stride, a.vocab);
    const Weights w = r.w;
    int first, last;
    chunk_of(a, row.blocks, &first, &last);
    if (r.mode == MODE_ALL) {
        uint64_t sum = 0;
        row.all(first + wave, last, kChunkWaves,
                [&](int, const float* v) {
#pragma unroll
                    for (int e = 0; e < Row<T>::E; ++e) sum += v[e] >= r.floor ? w.weight(v[e]) : 0;
                },
                [&](int k) {
                    sum = wave_sum64(sum);
                    if (lane == 0) sp.blocks[k] = sum;
                    sum = 0;
                });
        return;
    }
    for (int i = tid; i < kBins; i += kChunkThreads) s_hist[i] = 0;
    __syncthreads();
    if (r.mode == MODE_LIST)
        row.all(first + wave, last, kChunkWaves, [&](int, const float* v) {
#pragma unroll
            for (int e = 0; e < Row<T>::E; ++e) {
                const int d = w.bin(v[e]);
                if (d < kBins - 1) atomicAdd((uint32_t*)&s_hist[d], 1u);    // the last one's are not asked for
            }
        });
    else
        row.all(first + wave, last, kChunkWaves, [&](int, const float* v) {
#pragma unroll
            for (int e = 0; e < Row<T>::E; ++e) {
                const uint64_t m = v[e] >= r.floor ? w.weight(v[e]) : 0;
                if (m) atomicAdd((ull*)&s_hist[w.bin(v[e])], (ull)m);
            }
        });
    __syncthreads();
    for (int i = tid; i < kBins; i += kChunkThreads)
        if (s_hist[i]) atomicAdd((ull*)&sp.hist[i], (ull)s_hist[i]);
}

// Inclusive prefix sums over the workgroup of N numbers a thread; s_w: one for
// each wavefront and number.
template <int WAVES, int N>
__device__ __forceinline__ void scan(uint64_t (&v)[N], uint64_t (*s_w)[N]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = wave_scan(v[j]);
    __syncthreads();
    if (lane == 63)
#pragma unroll
        for (int j = 0; j < N; ++j) s_w[wave][j] = v[j];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (i < wave) v[j] += s_w[i][j];
}

template <typename T>
__global__ __launch_bounds__(kChunkThreads) void sample_list_kernel(SampleArgs a) {
    __shared__ uint64_t s_w[kChunkWaves][1], s_before, s_target;
    __shared__ int s_bin;
    __shared__ uint2 s_list[kListed];
    __shared__ uint32_t s_n, s_place;
    const int b = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const RowSpace sp(a, b);
    const RowRule r = rule_of(a, sp, b);
    if (r.mode != MODE_LIST && r.mode != MODE_SHARE) return;
    if (tid == 0) s_n = 0;               // before the barriers of the scan
    const Row<T> row(a.logits + b * a.stride, a.vocab);
    const Weights w = r.w;
    constexpr int kPer = kBins / kChunkThreads;
    // the bin in which the running sum reaches the target
    uint64_t h[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum += h[i] = sp.hist[tid * kPer + i];
    uint64_t ends[1] = {sum};
    scan<kChunkWaves>(ends, s_w);
    const uint64_t end = ends[0];
    if (tid == kChunkThreads - 1) {
        s_target = r.mode == MODE_SHARE ? share_of(r.top_p, end) : (uint64_t)r.top_k;
        s_bin = kBins - 1;               // fewer than top_k: all that are finite, tokens of weight 0 too
    }
    __syncthreads();
    uint64_t at = end - sum;
    if (at < s_target && s_target <= end) {
        int i = 0;
        while (at + h[i] < s_target) at += h[i++];
        s_bin = tid * kPer + i;
        s_before = at;
    }
    __syncthreads();
    const int bin = s_bin;
    if (r.mode == MODE_SHARE && blockIdx.x == 0 && tid == 0) {
        sp.head[0] = s_before;
        sp.head[1] = s_target;
    }
    const bool from = r.mode == MODE_LIST;   // the list holds the bins before, too
    int first, last;
    chunk_of(a, row.blocks, &first, &last);
    const float floor = fmaxf(r.floor, -FLT_MAX);        // -inf is not listed
    sum = 0;
    row.all(first + wave, last, kChunkWaves,
            [&](int t, const float* v) {
#pragma unroll
                for (int e = 0; e < Row<T>::E; ++e) {
                    const int d = w.bin(v[e]);
                    if ((d == bin || (from && d < bin)) && v[e] >= floor) {
                        const uint32_t place = atomicAdd(&s_n, 1u);
                        if (place < (uint32_t)a.list) s_list[place] = make_uint2(key_of(v[e]), (uint32_t)(t + e));
                    }
                    if (!from && d < bin) sum += w.weight(v[e]);
                }
            },
            [&](int k) {
                if (from) return;
                sum = wave_sum64(sum);
                if (lane == 0) sp.blocks[k] = sum;
                sum = 0;
            });
    // into the row's list at once: a place in it for each token was an atomic to
    // memory and back, 45 us for 1000 tokens
    __syncthreads();
    const uint32_t n = s_n;
    if (tid == 0 && n) s_place = atomicAdd((uint32_t*)&sp.head[2], n);
    __syncthreads();
    for (uint32_t i = tid; i < min(n, (uint32_t)a.list); i += kChunkThreads)
        if (s_place + i < (uint32_t)a.list) sp.list[s_place + i] = s_list[i];
}

// --------------------------------------------------------- kernel by rows

// Kept: tokens of a key above `key`, and the first `ties` of those with it.
struct Cut { uint32_t key, ties; uint64_t mass; };

struct SampleShared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint2 list[kListed];                 // key, token
    uint64_t block_mass[kMaxBlocks + 1];
    uint32_t block_ties[kMaxBlocks + 1];
    uint64_t w_sum[kRowWaves][2];
    uint32_t key_min, key_max, listed;
    uint64_t red;
    uint64_t found_mass, found_count;
    uint32_t found_at, found_here, found_key;
};

__device__ __forceinline__ void clear_hist(SampleShared& s) {
    for (int i = threadIdx.x; i < kBins; i += kRowThreads) { s.mass[i] = 0; s.count[i] = 0; }
}
// The first bin of the histogram at which the running count (by mass: the
// running mass) reaches target, what lies before it and how many it holds: found_*.
__device__ void find(SampleShared& s, bool by_mass, uint64_t target) {
    constexpr int kPer = kBins / kRowThreads;
    __syncthreads();
    const int b = threadIdx.x * kPer;
    uint64_t m[kPer], v[2] = {0, 0};
    uint32_t c[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        v[0] += m[i] = s.mass[b + i];
        v[1] += c[i] = s.count[b + i];
    }
    uint64_t mass = v[0], count = v[1];
    scan<kRowWaves>(v, s.w_sum);
    const uint64_t end = by_mass ? v[0] : v[1];
    mass = v[0] - mass;
    count = v[1] - count;
    if ((by_mass ? mass : count) < target && target <= end) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if ((by_mass ? mass : count) < target && target <= (by_mass ? mass + m[i] : count + c[i])) {
                s.found_at = b + i;
                s.found_mass = mass;
                s.found_count = count;
                s.found_here = c[i];
            }
            mass += m[i];
            count += c[i];
        }
    }
    __syncthreads();
}

// The end of the prefix that reaches target (a count or a mass, at least 1 and
// at most all there is) among the tokens that each(f) calls f(key) for, before
// which lie mass and count; keys lo .. hi occur.
template <typename F>
__device__ Cut cut_among(SampleShared& s, const Weights& w, uint32_t lo, uint32_t hi, uint64_t mass, uint64_t count, bool by_mass,
                         uint64_t target, F each) {
    for (;;) {
        const int bits = hi > lo ? 32 - __clz(hi - lo) : 0, shift = bits > 11 ? bits - 11 : 0;
        __syncthreads();
        clear_hist(s);
        __syncthreads();
        each([&](uint32_t k) {
            if (k < lo || k > hi) return;
            const uint64_t m = w.weight(logit_of(k));
            if (m == 0) return;
            const uint32_t d = (hi - k) >> shift;
            atomicAdd(&s.count[d], 1u);
            atomicAdd((ull*)&s.mass[d], (ull)m);
        });
        find(s, by_mass, target - (by_mass ? mass : count));
        mass += s.found_mass;
        count += s.found_count;
        uint32_t top = hi - (s.found_at << shift);
        if (shift != 0 && s.found_here == 1) {   // a bin of one token: it
            const uint32_t bottom = top - min(top, (1u << shift) - 1);
            each([&](uint32_t k) {
                if (k <= top && k >= bottom && k >= lo && w.weight(logit_of(k)) != 0) s.found_key = k;
            });
            __syncthreads();
            top = s.found_key;
        }
        if (shift == 0 || s.found_here == 1) {
            const uint64_t one = w.weight(logit_of(top));
            const uint64_t ties = by_mass ? (target - mass + one - 1) / one : target - count;
            __syncthreads();
            return Cut{top, (uint32_t)ties, mass + ties * one};
        }
        const uint32_t span = (1u << shift) - 1;
        hi = top;
        lo = max(lo, top > span ? top - span : 0u);
    }
}

// top_k and top_p among the tokens that each(f) calls f(key) for: everything that
// can be kept.
template <typename F>
__device__ Cut cut_all(SampleShared& s, const RowRule& r, F each) {
    if (threadIdx.x == 0) { s.key_min = 0xffffffffu; s.key_max = 0; s.red = 0; s.found_count = 0; }
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0;
    uint64_t mass = 0, count = 0;
    each([&](uint32_t k) {
        const uint64_t m = r.w.weight(logit_of(k));
        if (m == 0) return;
        lo = min(lo, k);
        hi = max(hi, k);
        mass += m;
        ++count;
    });
    if (count) {
        atomicMin(&s.key_min, lo);
        atomicMax(&s.key_max, hi);
        atomicAdd((ull*)&s.red, (ull)mass);
        atomicAdd((ull*)&s.found_count, (ull)count);
    }
    __syncthreads();
    lo = s.key_min;
    hi = s.key_max;
    const uint64_t there = s.found_count;                // at least the largest logit's
    Cut cut{lo - 1, 0, s.red};           // all of these, not what the list leaves out
    if (r.top_k && (uint64_t)r.top_k < there) cut = cut_among(s, r.w, lo, hi, 0, 0, false, (uint64_t)r.top_k, each);
    if (r.top_p < 1.0) {
        const uint64_t target = share_of(r.top_p, cut.mass);
        if (target < cut.mass) cut = cut_among(s, r.w, lo, hi, 0, 0, true, target, each);
    }
    __syncthreads();
    return cut;
}

// The same of a short list, a token a thread: its place and the weight ahead of it
// by comparison with each other token, where cut_among takes a histogram and two
// scans for each 11 bits of the keys, for top_k and for top_p.  25 rows of 1999
// bf16 logits, top_k 40: 45 us with that, 40 with this, with a top_p 46.5 and 39; the
// short lists of top_p alone gained 1 and are left to cut_among.
__device__ Cut cut_short(SampleShared& s, const RowRule& r, int n) {
    const int tid = threadIdx.x;
    uint4* all = reinterpret_cast<uint4*>(s.mass);       // key, token, weight
    uint64_t one = 0;
    uint2 t = make_uint2(0, 0);
    if (tid < n) {
        t = s.list[tid];
        one = r.w.weight(logit_of(t.x));
        all[tid] = make_uint4(t.x, t.y, (uint32_t)one, (uint32_t)(one >> 32));
    }
    if (tid == 0) { s.red = s.found_mass = 0; s.key_min = 0xffffffffu; s.listed = 0; }
    __syncthreads();
    uint64_t ahead = 0;
    int64_t place = 0;
    if (tid < n) {
        const uint64_t mine = (uint64_t)t.x << 32 | (uint32_t)~t.y;
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
            const uint4 o = all[j];
            const bool before = ((uint64_t)o.x << 32 | (uint32_t)~o.y) > mine;
            ahead += before ? (uint64_t)o.w << 32 | o.z : 0;
            place += before;
        }
    }
    bool kept = tid < n && place < r.top_k;
    if (r.top_p < 1.0) {
        const uint64_t sum = wave_sum64(kept ? one : 0);
        if ((tid & 63) == 0 && sum) atomicAdd((ull*)&s.found_mass, (ull)sum);
        __syncthreads();
        kept = kept && ahead < share_of(r.top_p, s.found_mass);
    }
    const uint64_t sum = wave_sum64(kept ? one : 0);
    if ((tid & 63) == 0 && sum) atomicAdd((ull*)&s.red, (ull)sum);
    if (kept) atomicMin(&s.key_min, t.x);
    __syncthreads();
    if (kept && t.x == s.key_min) atomicAdd(&s.listed, 1u);
    __syncthreads();
    return Cut{s.key_min, s.listed, s.red};
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void sample_token_kernel(SampleArgs a) {
    __shared__ SampleShared s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int b = blockIdx.x;
    const RowSpace sp(a, b);
    const RowRule r = rule_of(a, sp, b);
    if (r.mode == MODE_NONE) {
        if (tid == 0) a.token[b] = (uint32_t)(r.best >> 32) <= kNegInfKey ? -1 : (int)~(uint32_t)r.best;
        return;
    }
    const Row<T> row(a.logits + b * a.stride, a.vocab);
    const Weights w = r.w;
    const int blocks = row.blocks;
    const uint64_t listed = r.mode == MODE_ALL ? 0 : (uint32_t)sp.head[2];
    const bool whole = listed > (uint64_t)a.list;        // more than the list holds: read the row
    const int n = whole ? 0 : (int)listed;
    for (int i = tid; i < n; i += kRowThreads) s.list[i] = sp.list[i];
    for (int k = tid; k < blocks; k += kRowThreads) {
        s.block_mass[k] = r.mode == MODE_ALL || (r.mode == MODE_SHARE && !whole) ? sp.blocks[k] : 0;
        s.block_ties[k] = 0;
    }
    __syncthreads();
    auto each_listed = [&](auto f) {
        for (int i = tid; i < n; i += kRowThreads) f(s.list[i].x);
    };
    Cut cut;
    if (whole) {
        cut = cut_all(s, r, [&](auto f) {
            row.all(wave, blocks, kRowWaves, [&](int, const float* v) {
#pragma unroll 1
                for (int e = 0; e < Row<T>::E; ++e)
                    if (v[e] >= r.floor) f(key_of(v[e]));
            });
        });
        uint64_t sum = 0;
        uint32_t ties = 0;
        row.all(wave, blocks, kRowWaves,
                [&](int, const float* v) {
#pragma unroll
                    for (int e = 0; e < Row<T>::E; ++e) {
                        const uint32_t key = key_of(v[e]);
                        if (key > cut.key) sum += w.weight(v[e]);
                        ties += key == cut.key;
                    }
                },
                [&](int k) {
                    sum = wave_sum64(sum);
                    const uint64_t all_ties = wave_sum64(ties);
                    if (lane == 0) { s.block_mass[k] = sum; s.block_ties[k] = (uint32_t)all_ties; }
                    sum = 0;
                    ties = 0;
                });
    } else if (r.mode == MODE_ALL) {
        uint64_t sum = 0;
        for (int k = tid; k < blocks; k += kRowThreads) sum += s.block_mass[k];
        uint64_t v[2] = {sum, 0};
        scan<kRowWaves>(v, s.w_sum);
        if (tid == kRowThreads - 1) s.red = v[0];
        __syncthreads();
        cut = Cut{r.floor_key ? r.floor_key - 1 : 0, 0, s.red};
    } else {
        if (r.mode == MODE_LIST) {
            cut = n <= kShort ? cut_short(s, r, n) : cut_all(s, r, each_listed);
        } else {
            if (tid == 0) { s.key_min = 0xffffffffu; s.key_max = 0; }
            __syncthreads();
            each_listed([&](uint32_t k) { atomicMin(&s.key_min, k); atomicMax(&s.key_max, k); });
            __syncthreads();
            cut = cut_among(s, w, s.key_min, s.key_max, sp.head[0], 0, true, sp.head[1], each_listed);
        }
        for (int i = tid; i < n; i += kRowThreads) {
            const uint2 t = s.list[i];
            const int k = (int)(t.y + row.skip) / (Row<T>::E * kBlockUnits);
            if (t.x > cut.key) atomicAdd((ull*)&s.block_mass[k], (ull)w.weight(logit_of(t.x)));
            else if (t.x == cut.key) atomicAdd(&s.block_ties[k], 1u);
        }
    }
    __syncthreads();

    // the block in which the running weight passes floor(u * mass)
    const uint64_t one = cut.ties ? w.weight(logit_of(cut.key)) : 0;
    const double place = floor((double)a.u[b] * (double)cut.mass);
    uint64_t target = place > 0.0 ? (uint64_t)fmin(place, 0x1p62) : 0;
    if (target >= cut.mass) target = cut.mass - 1;
    const int per = (blocks + kRowThreads - 1) / kRowThreads;
    uint64_t sum = 0, ties = 0;
    for (int k = tid * per; k < min(blocks, (tid + 1) * per); ++k) { sum += s.block_mass[k]; ties += s.block_ties[k]; }
    uint64_t v[2] = {sum, ties};
    scan<kRowWaves>(v, s.w_sum);
    const uint64_t end = v[0], ties_end = v[1];
    uint64_t at = end - sum, seen = ties_end - ties;
    auto passed = [&](uint64_t mass, uint64_t t) { return mass + min(t, (uint64_t)cut.ties) * one > target; };
    if (!passed(at, seen) && passed(end, ties_end)) {
        int k = tid * per;
        while (!passed(at + s.block_mass[k], seen + s.block_ties[k])) { at += s.block_mass[k]; seen += s.block_ties[k]; ++k; }
        s.found_at = k;
        s.found_mass = at;
        s.found_count = seen;
    }
    __syncthreads();
    if (wave != 0) return;
    // then the token in it, four neighbouring units a lane
    constexpr int E = Row<T>::E;
    const int q = (int)s.found_at * kBlockUnits + 4 * lane;
    float l[4][E];
#pragma unroll
    for (int u = 0; u < 4; ++u) row.unit(q + u, l[u]);
    sum = 0;
    ties = 0;
    auto add = [&](float x) {
        const uint32_t key = key_of(x);
        if (key > cut.key) sum += w.weight(x);
        else ties += key == cut.key && cut.ties;
    };
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) add(l[u][e]);
    const uint64_t mass_end = s.found_mass + wave_scan(sum), seen_end = s.found_count + wave_scan(ties);
    sum = mass_end - sum;
    ties = seen_end - ties;
    if (!passed(sum, ties) && passed(mass_end, seen_end)) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool was = passed(sum, ties);
                add(l[u][e]);
                if (!was && passed(sum, ties)) a.token[b] = row.token(q + u, e);
            }
    }
}

template <typename T>
hipError_t launch_sample(SampleArgs& a, hipStream_t s) {
    // chunks of a row: about four workgroups a CU, each of a block a wavefront or more
    const int most = (a.vocab + 4 * kBlockUnits * kChunkWaves - 1) / (4 * kBlockUnits * kChunkWaves);
    const int want = (1024 + a.B - 1) / a.B;
    a.chunks = want < most ? want : most;
    if (a.chunks > kMaxChunks) a.chunks = kMaxChunks;
    const dim3 grid(a.chunks, a.B), wg(kChunkThreads);
    hipLaunchKernelGGL((sample_max_kernel<T>), grid, wg, 0, s, a);
    hipLaunchKernelGGL((sample_hist_kernel<T>), grid, wg, 0, s, a);
    hipLaunchKernelGGL((sample_list_kernel<T>), grid, wg, 0, s, a);
    hipLaunchKernelGGL((sample_token_kernel<T>), dim3(a.B), dim3(kRowThreads), 0, s, a);
    return hipGetLastError();
}

// Places of a list and blocks of a row of fp32 (of bf16: fewer).
static int sample_list(int vocab) { return vocab < kListed ? vocab : kListed; }
static int sample_blocks(int vocab) { return (vocab + 3 + 4 * kBlockUnits - 1) / (4 * kBlockUnits); }

}  // namespace buddy

using namespace buddy;

extern "C" {

size_t buddy_sample_workspace(int32_t B, int32_t vocab) {
    if (B < 0 || B > 65535 || vocab < 1 || vocab > kMaxVocab) return 0;
    return 16 + (size_t)B * row_space_bytes(sample_list(vocab), sample_blocks(vocab));
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
    a.list = sample_list(p->vocab); a.blocks = sample_blocks(p->vocab);
    a.space = (char*)p->workspace; a.row_bytes = row_space_bytes(a.list, a.blocks);
    const hipError_t e = size == 2 ? launch_sample<bf16_t>(a, (hipStream_t)stream) : launch_sample<float>(a, (hipStream_t)stream);
    return e == hipSuccess ? BUDDY_OK : BUDDY_EDEVICE;
}

}  // extern "C"
