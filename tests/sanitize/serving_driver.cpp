// Test driver for the host code of the operators around attention under
// AddressSanitizer and UndefinedBehaviorSanitizer (test infrastructure only):
// every refusal of their entry points, none of which reaches the device, the
// scale of a group against its definition, and workspaces against what the
// calls lay out in them.  The projection's source is part of this file, so
// that its plans can be read.  Exit status 0 means that every check held.
#include <float.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "../../paper_2606_09514_amd/csrc/linear8.hip"

using namespace buddy;

static int failures = 0;
#define EXPECT(cond, what)                                                                             \
    do {                                                                                               \
        if (!(cond)) { fprintf(stderr, "FAILED: %s (line %d)\n", what, __LINE__); ++failures; }        \
    } while (0)
// What a refused call returns with one thing changed.
#define WITH(call, change, status)                                                                     \
    do { auto k = base; change; EXPECT(call == status, #change); } while (0)

static char* const P = (char*)0x10000;                                   // never followed
static void* at(int n) { return P + n; }

static buddy_mx8 rows_of(int32_t rows, int32_t width) {
    return buddy_mx8{(uint8_t*)P, (uint8_t*)P, width, 16 * ((width + 511) / 512), rows, width};
}

static void scales() {
    // least e with amax <= 448 * 2^e, within the codes that are written
    for (uint32_t e = 0; e < 255; ++e)
        for (uint32_t m : {0u, 1u, 0x5fffffu, 0x600000u, 0x600001u, 0x7fffffu}) {
            const uint32_t bits = e << 23 | m;
            float v;
            memcpy(&v, &bits, 4);
            int want = kMx8MinScale;
            while (want < kMx8MaxScale && (double)v > ldexp(448.0, want - 127)) ++want;
            EXPECT(mx8_scale_code(bits) == want, "scale");
        }
    for (uint32_t bits : {0x7f800000u, 0x7f800001u, 0x7fc00000u, 0x7fffffffu}) EXPECT(mx8_scale_code(bits) == kMx8NanScale, "nan scale");
}

static void mx8_refusals(buddy_status (*call)(const buddy_mx8*)) {
    const buddy_mx8 base = rows_of(3, 48);
    EXPECT(call(nullptr) == BUDDY_EINVAL, "no rows");
    WITH(call(&k), k.n_rows = -1, BUDDY_EINVAL);
    WITH(call(&k), k.width = 0, BUDDY_EINVAL);
    WITH(call(&k), k.width = -16, BUDDY_EINVAL);
    WITH(call(&k), k.width = 40, BUDDY_ESHAPE);
    WITH(call(&k), k.width = (1 << 20) + 16, BUDDY_ESHAPE);
    WITH(call(&k), k.n_rows = (1 << 24) + 1, BUDDY_ECAPACITY);
    WITH(call(&k), k.codes = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.scales = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.codes = (uint8_t*)at(8), BUDDY_EINVAL);
    WITH(call(&k), k.scales = (uint8_t*)at(4), BUDDY_EINVAL);
    WITH(call(&k), k.code_stride = 32, BUDDY_EINVAL);
    WITH(call(&k), k.code_stride = 56, BUDDY_EINVAL);
    WITH(call(&k), k.code_stride = -48, BUDDY_EINVAL);
    WITH(call(&k), k.code_stride = INT64_MAX - 15, BUDDY_EINVAL);
    WITH(call(&k), k.scale_stride = 0, BUDDY_EINVAL);
    WITH(call(&k), k.scale_stride = 24, BUDDY_EINVAL);
    WITH(call(&k), (k.width = 528, k.code_stride = 528, k.scale_stride = 16), BUDDY_EINVAL);
}

static void norm() {
    buddy_norm base = {};
    base.n_rows = 3; base.width = 48; base.hidden_dtype = BUDDY_F32; base.dtype = BUDDY_BF16;
    base.h = base.delta = base.weight = P; base.h_out = base.y = P;
    base.h_stride = base.delta_stride = base.h_out_stride = base.y_stride = 48;
    base.rms_eps = 1e-6f;
    const buddy_mx8 m = rows_of(3, 48), other = rows_of(2, 48), wide = rows_of(3, 64);
    buddy_mx8 torn = m;
    torn.code_stride = 32;
    auto call = [](const buddy_norm* k) { return buddy_add_rmsnorm(k, nullptr); };
    EXPECT(call(nullptr) == BUDDY_EINVAL, "null");
    WITH(call(&k), k.n_rows = -1, BUDDY_EINVAL);
    WITH(call(&k), k.width = 0, BUDDY_EINVAL);
    WITH(call(&k), k.width = 40, BUDDY_ESHAPE);
    WITH(call(&k), k.width = 32784, BUDDY_ESHAPE);
    WITH(call(&k), k.n_rows = (1 << 24) + 1, BUDDY_ECAPACITY);
    WITH(call(&k), k.hidden_dtype = 2, BUDDY_EINVAL);
    WITH(call(&k), k.dtype = -1, BUDDY_EINVAL);
    WITH(call(&k), k.rms_eps = -1e-6f, BUDDY_EINVAL);
    WITH(call(&k), k.rms_eps = NAN, BUDDY_EINVAL);
    WITH(call(&k), k.h = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.h = at(4), BUDDY_EINVAL);
    WITH(call(&k), k.weight = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.weight = at(2), BUDDY_EINVAL);
    WITH(call(&k), k.h_out = nullptr, BUDDY_EINVAL);                     // a sum without its place
    WITH(call(&k), k.delta = nullptr, BUDDY_EINVAL);                     // a place without a sum
    WITH(call(&k), k.y = nullptr, BUDDY_EINVAL);                         // nothing to write
    WITH(call(&k), k.delta = at(8), BUDDY_EINVAL);
    WITH(call(&k), k.y = at(8), BUDDY_EINVAL);
    WITH(call(&k), k.h_stride = 47, BUDDY_EINVAL);
    WITH(call(&k), k.h_stride = 50, BUDDY_EINVAL);                       // 200 bytes
    WITH(call(&k), k.delta_stride = 52, BUDDY_EINVAL);                   // 104 bytes
    WITH(call(&k), k.h_out_stride = 0, BUDDY_EINVAL);
    WITH(call(&k), k.y_stride = -48, BUDDY_EINVAL);
    WITH(call(&k), k.y_mx8 = &other, BUDDY_EINVAL);
    WITH(call(&k), k.y_mx8 = &wide, BUDDY_EINVAL);
    WITH(call(&k), k.y_mx8 = &torn, BUDDY_EINVAL);
    const buddy_mx8 none = rows_of(0, 48);
    WITH(call(&k), k.n_rows = 0, BUDDY_OK);
    WITH(call(&k), (k.n_rows = 0, k.y_mx8 = &none, k.h = k.delta = k.weight = nullptr, k.y = nullptr, k.delta = P), BUDDY_OK);
}

static void quantise_and_read() {
    mx8_refusals([](const buddy_mx8* m) { return buddy_mx8_quantize(m, BUDDY_F32, P, 1024, nullptr, 0, nullptr, nullptr); });
    mx8_refusals([](const buddy_mx8* m) { return buddy_mx8_read(m, BUDDY_F32, P, 1024, nullptr); });
    const buddy_mx8 m = rows_of(3, 48), none = rows_of(0, 48);
    EXPECT(buddy_mx8_quantize(&m, 7, P, 48, nullptr, 0, nullptr, nullptr) == BUDDY_EINVAL, "type");
    EXPECT(buddy_mx8_quantize(&m, BUDDY_BF16, nullptr, 48, nullptr, 0, nullptr, nullptr) == BUDDY_EINVAL, "x");
    EXPECT(buddy_mx8_quantize(&m, BUDDY_BF16, at(2), 48, nullptr, 0, nullptr, nullptr) == BUDDY_EINVAL, "x start");
    EXPECT(buddy_mx8_quantize(&m, BUDDY_BF16, P, 52, nullptr, 0, nullptr, nullptr) == BUDDY_EINVAL, "x stride");
    EXPECT(buddy_mx8_quantize(&m, BUDDY_BF16, P, 48, P, 40, nullptr, nullptr) == BUDDY_EINVAL, "gate stride");
    EXPECT(buddy_mx8_quantize(&m, BUDDY_BF16, P, 48, at(8), 48, nullptr, nullptr) == BUDDY_EINVAL, "gate start");
    EXPECT(buddy_mx8_quantize(&none, BUDDY_BF16, nullptr, 0, nullptr, 0, nullptr, nullptr) == BUDDY_OK, "none");
    EXPECT(buddy_mx8_read(&m, 3, P, 48, nullptr) == BUDDY_EINVAL, "type");
    EXPECT(buddy_mx8_read(&m, BUDDY_F32, P, 40, nullptr) == BUDDY_EINVAL, "out stride");
    EXPECT(buddy_mx8_read(&m, BUDDY_F32, at(8), 48, nullptr) == BUDDY_EINVAL, "out start");
    EXPECT(buddy_mx8_read(&none, BUDDY_F32, nullptr, 0, nullptr) == BUDDY_OK, "none");
}

static void linear() {
    static buddy_mx8 x, w;
    x = rows_of(3, 48);
    w = rows_of(5, 48);
    mx8_refusals([](const buddy_mx8* m) { return buddy_mx8_linear(m, &w, BUDDY_F32, P, 8, P, 1 << 30, nullptr); });
    mx8_refusals([](const buddy_mx8* m) { return buddy_mx8_linear(&x, m, BUDDY_F32, P, 8, P, 1 << 30, nullptr); });
    const size_t need = buddy_mx8_linear_workspace(&x, &w);
    EXPECT(need >= 16, "workspace");
    struct Call { buddy_mx8 x, w; int32_t t; void* out; int64_t os; void* ws; size_t n; } base{x, w, BUDDY_BF16, P, 5, P, need};
    auto call = [](const Call* k) { return buddy_mx8_linear(&k->x, &k->w, k->t, k->out, k->os, k->ws, k->n, nullptr); };
    WITH(call(&k), k.t = 2, BUDDY_EINVAL);
    WITH(call(&k), k.w = rows_of(5, 64), BUDDY_EINVAL);
    WITH(call(&k), k.w.n_rows = 0, BUDDY_EINVAL);
    WITH(call(&k), k.w.n_rows = (1 << 20) + 1, BUDDY_ECAPACITY);
    WITH(call(&k), k.x.n_rows = (1 << 20) + 1, BUDDY_ECAPACITY);
    WITH(call(&k), k.out = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.out = at(1), BUDDY_EINVAL);
    WITH(call(&k), k.os = 4, BUDDY_EINVAL);
    WITH(call(&k), k.os = -5, BUDDY_EINVAL);
    WITH(call(&k), k.os = INT64_MAX / 4, BUDDY_EINVAL);
    WITH(call(&k), k.ws = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.ws = at(8), BUDDY_EINVAL);
    WITH(call(&k), k.n = need - 1, BUDDY_EINVAL);
    WITH(call(&k), (k.x.n_rows = 0, k.out = nullptr, k.ws = nullptr, k.n = 0), BUDDY_OK);

    // plans stay in their workspace, at most the kernels' shapes, for every count
    // up to the one that the workspace was asked for
    uint64_t s = 1;
    auto next = [&](int n) { s = s * 6364136223846793005ull + 1442695040888963407ull; return (int)((s >> 33) % n); };
    for (int t = 0; t < 4000; ++t) {
        const int shift = next(17), K = 16 * (1 + next(1 << (4 + next(8)))), n = 1 + next(1 << shift), rows = 1 + next(1 << next(15));
        const size_t space = linear8_space(rows, n, K);
        EXPECT(space % 16 == 0 && space >= 16, "space");
        for (int r : {1, 1 + next(rows), 1 + next(rows < 300 ? rows : 300), rows}) {
            if (r > rows) continue;
            EXPECT(linear8_space(r, n, K) <= space, "fewer rows, less space");
            for (bool wide : {false, true}) {
                const Linear8Plan p = linear8_plan(r, n, K, wide);
                const int steps = up(K, kStepK);
                if (p.form == Linear8Plan::STREAM) { EXPECT(r <= 16, "stream"); continue; }
                EXPECT(p.splits >= 1 && p.splits <= steps, "splits");
                const size_t sums = p.splits > 1 ? (size_t)p.splits * r * up(n, 16) * 64 : 0;
                EXPECT(4 * (size_t)(p.pw + p.px) + sums <= space, "plan in its space");
                if (p.form == Linear8Plan::TILE) {
                    EXPECT(!wide && K % kStepK == 0 && steps / p.splits >= 4, "tile");
                    EXPECT(p.pw == (int64_t)up(n, kTile) * 4 * steps * 64 && p.px == (int64_t)up(r, kTile) * 4 * steps * 64, "scales");
                } else {
                    EXPECT(p.tj == 1 || p.tj == 2 || p.tj == 4 || p.tj == 6 || p.tj == 8, "row tiles");
                    EXPECT(p.parts == 1 || p.parts == 2 || (p.parts == 4 && p.tj <= 4) || (p.parts == 8 && p.tj == 1), "parts");
                    EXPECT(p.per >= 1 && p.per * p.parts <= 8, "wavefronts");
                    EXPECT((int64_t)p.chunks * p.tj * 16 >= r && (int64_t)(p.chunks - 1) * p.tj * 16 < r, "chunks");
                }
            }
        }
    }
    EXPECT(buddy_mx8_linear_workspace(nullptr, &w) == 0 && buddy_mx8_linear_workspace(&x, nullptr) == 0, "no sizes");
    buddy_mx8 sizes = x;
    sizes.codes = sizes.scales = nullptr;
    sizes.code_stride = 0;
    EXPECT(buddy_mx8_linear_workspace(&sizes, &w) == need, "pointers are not read");
    sizes.width = 64;
    EXPECT(buddy_mx8_linear_workspace(&sizes, &w) == 0, "other widths");
}

static void lora() {
    EXPECT(buddy_lora_plan_size(-1, 3) == 0 && buddy_lora_plan_size(3, 0) == 0 && buddy_lora_plan_size(3, 4097) == 0 &&
           buddy_lora_plan_size((1 << 20) + 1, 3) == 0, "plan sizes that are refused");
    for (int rows : {0, 1, 15, 16, 1023, 1024, 1025, 4099, 1 << 20})
        for (int n : {1, 2, 31, 1023, 1024, 4096}) {
            // the worst of ids: every group ends in a tile of one row
            const int T = rows >= 1024 && rows / (n + 1) >= 32 ? 64 : 16, groups = rows < n + 1 ? rows : n + 1;
            const int64_t tiles = groups + (rows - groups) / T;
            EXPECT(buddy_lora_plan_size(rows, n) >= 4 + tiles * (4 + T), "plan size");
        }
    EXPECT(buddy_lora_plan(nullptr, -1, 3, (int32_t*)P, nullptr) == BUDDY_EINVAL, "rows");
    EXPECT(buddy_lora_plan((int32_t*)P, 3, 0, (int32_t*)P, nullptr) == BUDDY_EINVAL, "adapters");
    EXPECT(buddy_lora_plan((int32_t*)P, 3, 4097, (int32_t*)P, nullptr) == BUDDY_ECAPACITY, "many adapters");
    EXPECT(buddy_lora_plan((int32_t*)P, (1 << 20) + 1, 3, (int32_t*)P, nullptr) == BUDDY_ECAPACITY, "many rows");
    EXPECT(buddy_lora_plan(nullptr, 3, 3, (int32_t*)P, nullptr) == BUDDY_EINVAL, "ids");
    EXPECT(buddy_lora_plan((int32_t*)P, 3, 3, nullptr, nullptr) == BUDDY_EINVAL, "plan");
    EXPECT(buddy_lora_plan((int32_t*)P, 3, 3, (int32_t*)at(4), nullptr) == BUDDY_EINVAL, "plan start");
    EXPECT(buddy_lora_plan(nullptr, 0, 3, nullptr, nullptr) == BUDDY_OK, "no rows");

    const buddy_lora l = {P, P, (float*)P, BUDDY_BF16, 3, 16, 40, 24};
    const size_t need = buddy_lora_workspace(&l, 5);
    EXPECT(need >= 16 + 5 * 16 * 4, "workspace");
    struct Call { buddy_lora l; void *x, *y, *out; int64_t xs, ys, os; int32_t rows; int32_t* plan; void* ws; size_t n; }
        base{l, P, P, P, 40, 24, 24, 5, (int32_t*)P, P, need};
    auto call = [](const Call* k) {
        return buddy_lora_add(&k->l, k->x, k->xs, k->y, k->ys, k->out, k->os, k->rows, k->plan, k->ws, k->n, nullptr);
    };
    EXPECT(buddy_lora_add(nullptr, P, 40, P, 24, P, 24, 5, (int32_t*)P, P, need, nullptr) == BUDDY_EINVAL, "null");
    WITH(call(&k), k.l.a = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.l.b = at(8), BUDDY_EINVAL);
    WITH(call(&k), k.l.scale = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.l.dtype = 5, BUDDY_EINVAL);
    WITH(call(&k), k.l.n_adapters = 0, BUDDY_EINVAL);
    WITH(call(&k), k.l.n_adapters = 4097, BUDDY_ECAPACITY);
    WITH(call(&k), k.rows = -1, BUDDY_EINVAL);
    WITH(call(&k), k.rows = (1 << 20) + 1, BUDDY_ECAPACITY);
    WITH(call(&k), k.l.rank = 0, BUDDY_ESHAPE);
    WITH(call(&k), k.l.rank = 12, BUDDY_ESHAPE);
    WITH(call(&k), k.l.rank = 136, BUDDY_ESHAPE);
    WITH(call(&k), k.l.d_in = 36, BUDDY_ESHAPE);
    WITH(call(&k), k.l.d_out = 20, BUDDY_ESHAPE);
    WITH(call(&k), k.l.d_in = 0, BUDDY_EINVAL);
    WITH(call(&k), k.l.d_out = (1 << 20) + 8, BUDDY_ESHAPE);
    WITH(call(&k), k.x = at(8), BUDDY_EINVAL);
    WITH(call(&k), k.y = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.out = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.xs = 32, BUDDY_EINVAL);
    WITH(call(&k), k.ys = 28, BUDDY_EINVAL);
    WITH(call(&k), k.os = 16, BUDDY_EINVAL);
    WITH(call(&k), k.os = 32, BUDDY_EINVAL);                             // in place, rows elsewhere
    WITH(call(&k), k.plan = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.plan = (int32_t*)at(8), BUDDY_EINVAL);
    WITH(call(&k), k.ws = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.ws = at(4), BUDDY_EINVAL);
    WITH(call(&k), k.n = need - 1, BUDDY_EINVAL);
    WITH(call(&k), (k.rows = 0, k.x = k.y = k.out = k.ws = nullptr, k.plan = nullptr), BUDDY_OK);
    size_t last = 0;
    for (int rows = 0; rows <= 1 << 20; rows += 1 + rows / 7) {
        const size_t n = buddy_lora_workspace(&l, rows);
        EXPECT(n >= last, "fewer rows, less space");
        last = n;
    }
    buddy_lora bad = l;
    bad.rank = 9;
    EXPECT(buddy_lora_workspace(&bad, 5) == 0 && buddy_lora_workspace(nullptr, 5) == 0 && buddy_lora_workspace(&l, -1) == 0, "no sizes");
}

static void sample() {
    EXPECT(buddy_sample_workspace(-1, 5) == 0 && buddy_sample_workspace(65536, 5) == 0 && buddy_sample_workspace(2, 0) == 0 &&
           buddy_sample_workspace(2, (1 << 20) + 1) == 0, "no sizes");
    EXPECT(buddy_sample_workspace(3, 1000) > buddy_sample_workspace(2, 1000) && buddy_sample_workspace(0, 1000) >= 16, "sizes");
    buddy_sampling base = {};
    base.logits = P; base.stride = 1000; base.dtype = BUDDY_BF16; base.B = 3; base.vocab = 1000;
    base.temperature = base.u = (float*)P; base.token = (int32_t*)P; base.workspace = P;
    base.workspace_bytes = buddy_sample_workspace(3, 1000);
    auto call = [](const buddy_sampling* k) { return buddy_sample(k, nullptr); };
    EXPECT(call(nullptr) == BUDDY_EINVAL, "null");
    WITH(call(&k), k.B = -1, BUDDY_EINVAL);
    WITH(call(&k), k.B = 65536, BUDDY_ECAPACITY);
    WITH(call(&k), k.vocab = 0, BUDDY_EINVAL);
    WITH(call(&k), k.vocab = (1 << 20) + 1, BUDDY_ECAPACITY);
    WITH(call(&k), k.dtype = 2, BUDDY_EINVAL);
    WITH(call(&k), k.logits = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.logits = at(1), BUDDY_EINVAL);
    WITH(call(&k), k.stride = 999, BUDDY_EINVAL);
    WITH(call(&k), k.stride = -1000, BUDDY_EINVAL);
    WITH(call(&k), k.stride = INT64_MAX / 8, BUDDY_EINVAL);
    WITH(call(&k), k.temperature = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.u = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.token = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.workspace = nullptr, BUDDY_EINVAL);
    WITH(call(&k), k.workspace = at(8), BUDDY_EINVAL);
    WITH(call(&k), k.workspace_bytes -= 1, BUDDY_EINVAL);
    WITH(call(&k), (k.B = 0, k.logits = nullptr, k.workspace = nullptr), BUDDY_OK);
}

int main() {
    scales();
    norm();
    quantise_and_read();
    linear();
    lora();
    sample();
    if (failures) return 1;
    printf("serving driver ok\n");
    return 0;
}
