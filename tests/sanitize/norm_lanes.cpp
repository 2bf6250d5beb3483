// The norm's kernel on the host, a thread a lane (test infrastructure only):
// rows that one workgroup takes one behind another, padding among them in every
// pattern.  Each access of its LDS array is kept with the wavefront that made it
// and the barriers that it had passed; a write and another wavefront's access of
// one element with no barrier between them end the run with status 1, as does a
// wrong row.  norm_kernel.inc is the kernel's text out of rows8.hip, its LDS array
// a static one of Cells.
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <barrier>
#include <map>
#include <mutex>
#include <set>
#include <thread>
#include <vector>

#define __global__
#define __launch_bounds__(n)

typedef uint16_t bf16_t;
struct uint2 { uint32_t x, y; };
struct Dim { int x; };
constexpr int kWave = 64;
static Dim blockIdx{0}, gridDim{1}, blockDim{0};
static thread_local Dim threadIdx{0};
static thread_local int barriers = 0;
static std::barrier<>* workgroup;
static std::vector<std::barrier<>*> wavefront;
static std::vector<float> lanes;

static void __syncthreads() {
    workgroup->arrive_and_wait();
    ++barriers;
}
static float wave_sum(float v) {
    const int tid = threadIdx.x, wave = tid / kWave;
    lanes[tid] = v;
    wavefront[wave]->arrive_and_wait();
    float sum = 0.f;
    for (int i = 0; i < kWave; ++i) sum += lanes[wave * kWave + i];
    wavefront[wave]->arrive_and_wait();
    return sum;
}

struct Cell;
static std::mutex mutex;
struct Interval { std::set<int> readers, writers; };
static std::map<std::pair<const Cell*, int>, Interval> accesses;                // element, barriers passed
struct Cell {
    float v;
    static void note(const Cell* c, bool write) {
        Interval& i = accesses[{c, barriers}];
        (write ? i.writers : i.readers).insert(threadIdx.x / kWave);
    }
    Cell& operator=(float x) {
        std::lock_guard<std::mutex> hold(mutex);
        note(this, true);
        v = x;
        return *this;
    }
    operator float() const {
        std::lock_guard<std::mutex> hold(mutex);
        note(this, false);
        return v;
    }
};

static void load8(const char* p, float* x, float) { memcpy(x, p, 32); }
static void store8(char* p, const float* x, float) { memcpy(p, x, 32); }
static float bf2f(bf16_t v) { const uint32_t u = (uint32_t)v << 16; float f; memcpy(&f, &u, 4); return f; }
static bf16_t f2bf(float v) { uint32_t u; memcpy(&u, &v, 4); return (bf16_t)(u >> 16); }
static uint2 quantise8(const float*, int* code) { *code = 0; return uint2{0, 0}; }

#include "norm_kernel.inc"

template <int N>
static int run(int threads, int rows, int padding) {
    const int width = threads * 8 * N;
    std::vector<float> h(rows * width), w(width), y(rows * width, 9.f);
    std::vector<int32_t> pos(rows);
    for (int r = 0; r < rows; ++r) {
        pos[r] = padding >> r & 1 ? -1 : r;
        for (int i = 0; i < width; ++i) h[r * width + i] = (float)((i * 7 + r * 13) % 31 - 15) * (float)(1 << r);
    }
    for (int i = 0; i < width; ++i) w[i] = 1.f + (float)(i % 5);
    NormArgs a = {};
    a.h = (const char*)h.data(); a.h_stride = width * 4;
    a.w = (const char*)w.data();
    a.y = (char*)y.data(); a.y_stride = width * 4;
    a.pos = pos.data(); a.n_rows = rows; a.width = width; a.eps = 1e-6f;
    blockDim.x = threads;
    std::barrier<> all(threads);
    workgroup = &all;
    lanes.assign(threads, 0.f);
    wavefront.clear();
    for (int i = 0; i < threads / kWave; ++i) wavefront.push_back(new std::barrier<>(kWave));
    accesses.clear();
    std::vector<std::thread> lane;
    for (int t = 0; t < threads; ++t)
        lane.emplace_back([t, &a] {
            threadIdx.x = t;
            barriers = 0;
            norm_kernel<float, float, N>(a);
        });
    for (auto& t : lane) t.join();
    for (auto* b : wavefront) delete b;

    int bad = 0;
    for (const auto& entry : accesses) {
        const Interval& i = entry.second;
        std::set<int> both = i.readers;
        both.insert(i.writers.begin(), i.writers.end());
        if (!i.writers.empty() && both.size() > 1) bad = 1;
    }
    if (bad) fprintf(stderr, "padding %#x of %d rows: an element is written while another wavefront may read it\n", padding, rows);
    for (int r = 0; r < rows; ++r) {
        double sum = 0;
        for (int i = 0; i < width; ++i) sum += (double)h[r * width + i] * h[r * width + i];
        const double scale = 1 / sqrt(sum / width + 1e-6);
        for (int i = 0; i < width; ++i) {
            const double want = pos[r] < 0 ? 9.0 : h[r * width + i] * scale * w[i], got = y[r * width + i];
            // N pieces of three additions, 64 lanes and the wavefronts: fewer than 80
            // roundings of 2^-24 each, halved by the root, and four behind it
            if (!(fabs(got - want) <= 44 * ldexp(1, -24) * fabs(want))) {
                fprintf(stderr, "padding %#x, row %d, element %d: %g, not %g\n", padding, r, i, got, want);
                return 1;
            }
        }
    }
    return bad;
}

int main() {
    int bad = 0;
    for (int padding = 0; padding < 32; ++padding) bad |= run<1>(128, 5, padding);
    for (int padding : {0, 1, 2, 3, 5, 6}) bad |= run<2>(320, 3, padding);
    if (bad) return 1;
    printf("norm lanes ok\n");
    return 0;
}
