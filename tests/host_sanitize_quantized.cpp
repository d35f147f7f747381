// Host-side exerciser of the entry points of the 8-bit projections and the 4-bit paged cache, for a build with AddressSanitizer and
// UndefinedBehaviorSanitizer on the host code (tests/test_host_sanitizers_quantized.py).  Nothing is launched: every call is one that its
// checks must refuse, and the queries only compute.
#include <limits.h>
#include <math.h>
#include <stdio.h>

#include "koala.h"

static int failures = 0;
#define EXPECT(cond)                                                         \
    do {                                                                     \
        if (!(cond)) { printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); ++failures; } \
    } while (0)

alignas(256) static char mem[4096];   // stands for device memory: addresses that are looked at, never followed

static void quantizer() {
    struct Case {
        int form = KOALA_ROWS_PLAIN, dt = KOALA_BF16, rows = 3, cols = 100;
        void *x = mem;
        int64_t xs = 104;
        void *gain = mem;
        int gdt = KOALA_FP32;
        float eps = 1e-6f;
        int8_t *q = (int8_t *)mem;
        int64_t qs = 112;
        float *scale = (float *)mem;
        koala_status run() const { return koala_quantize_rows(nullptr, form, dt, rows, cols, x, xs, gain, gdt, eps, q, qs, scale); }
    };
    { Case c; c.x = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    { Case c; c.q = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    { Case c; c.scale = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    { Case c; c.form = KOALA_ROWS_NORM; c.gain = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    for (int f : {-1, 3, INT_MAX, INT_MIN}) { Case c; c.form = f; EXPECT(c.run() == KOALA_E_UNSUPPORTED); }
    for (int d : {-1, 2, 7, INT_MAX}) { Case c; c.dt = d; EXPECT(c.run() == KOALA_E_UNSUPPORTED); }
    for (int d : {-1, 2, 7, INT_MAX}) { Case c; c.form = KOALA_ROWS_NORM; c.gdt = d; EXPECT(c.run() == KOALA_E_UNSUPPORTED); }
    for (int n : {0, -1, INT_MIN}) {
        { Case c; c.rows = n; EXPECT(c.run() == KOALA_E_SHAPE); }
        { Case c; c.cols = n; EXPECT(c.run() == KOALA_E_SHAPE); }
    }
    { Case c; c.cols = INT_MAX; c.xs = c.qs = LLONG_MAX; EXPECT(c.run() == KOALA_E_SHAPE); }
    for (int64_t n : {(int64_t)96, (int64_t)0, (int64_t)-8, (int64_t)LLONG_MIN}) { Case c; c.xs = n; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.form = KOALA_ROWS_SWIGLU; c.xs = 192; EXPECT(c.run() == KOALA_E_SHAPE); }
    for (int64_t n : {(int64_t)104, (int64_t)0, (int64_t)LLONG_MIN}) { Case c; c.qs = n; EXPECT(c.run() == KOALA_E_SHAPE); }
    for (float e : {-1.f, NAN}) { Case c; c.form = KOALA_ROWS_NORM; c.eps = e; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.x = mem + 8; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.q = (int8_t *)mem + 4; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.scale = (float *)(mem + 2); EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.xs = 101; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.xs = LLONG_MAX; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.qs = 120; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.form = KOALA_ROWS_NORM; c.gain = mem + 4; EXPECT(c.run() == KOALA_E_ALIGN); }
}

static void product() {
    size_t need = 1;
    EXPECT(koala_linear_workspace_bytes(1, 4096, 4096, nullptr) == KOALA_E_NULL);
    for (int n : {0, -1, INT_MIN}) {
        EXPECT(koala_linear_workspace_bytes(n, 16, 16, &need) == KOALA_E_SHAPE);
        EXPECT(koala_linear_workspace_bytes(1, n, 16, &need) == KOALA_E_SHAPE);
        EXPECT(koala_linear_workspace_bytes(1, 16, n, &need) == KOALA_E_SHAPE);
    }
    for (int n : {8, 17, 131072, INT_MAX}) EXPECT(koala_linear_workspace_bytes(1, 16, n, &need) == KOALA_E_SHAPE);
    // every plan is one that can be made, at the sizes' ends too
    for (int rows : {1, 16, 17, 64, 65, 128, 2000, 1 << 20, INT_MAX})
        for (int out : {1, 15, 4096, 151936, INT_MAX})
            for (int in : {16, 1040, 17920, 131056}) {
                const bool fits = rows <= 1 << 26 && out <= 1 << 26 && (long)rows * out <= 1l << 37;
                EXPECT(koala_linear_workspace_bytes(rows, out, in, &need) == (fits ? KOALA_OK : KOALA_E_SHAPE));
                if (fits) EXPECT(need % 16 == 0 && (rows > 64 || need == 0));
            }
    struct Case {
        int rows = 480, out = 6656, in = 17920;
        int8_t *q = (int8_t *)mem, *w = (int8_t *)mem;
        int64_t qs = 17920, ws = 17920, ys = 6656;
        float *qsc = (float *)mem, *wsc = (float *)mem;
        int dt = KOALA_BF16;
        void *add = nullptr, *y = mem, *work = mem;
        size_t bytes = 0;
        koala_status run() const { return koala_linear_quantized(nullptr, rows, out, in, q, qs, qsc, w, ws, wsc, dt, add, y, ys, work, bytes); }
    };
    { Case c; c.q = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    { Case c; c.w = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    { Case c; c.qsc = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    { Case c; c.wsc = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    { Case c; c.y = nullptr; EXPECT(c.run() == KOALA_E_NULL); }
    for (int d : {-1, 2, INT_MAX}) { Case c; c.dt = d; EXPECT(c.run() == KOALA_E_UNSUPPORTED); }
    for (int n : {0, -5}) { Case c; c.rows = n; EXPECT(c.run() == KOALA_E_SHAPE); }
    for (int n : {0, 24, 131072}) { Case c; c.in = n; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.qs = 17904; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.ws = -16; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.ys = 6655; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.qs = (1 << 22) + 16; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.ws = 1ll << 40; EXPECT(c.run() == KOALA_E_SHAPE); }
    { Case c; c.q = (int8_t *)mem + 8; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.w = (int8_t *)mem + 1; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.qs = 17921; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.qsc = (float *)(mem + 1); EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.wsc = (float *)(mem + 2); EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.y = mem + 1; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.add = mem + 1; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.work = mem + 4; EXPECT(c.run() == KOALA_E_ALIGN); }
    { Case c; c.bytes = 16; EXPECT(c.run() == KOALA_E_WORKSPACE); }
    { Case c; c.work = nullptr; c.bytes = (size_t)-1; EXPECT(c.run() == KOALA_E_WORKSPACE); }
}

static koala_paged_kv cache() {
    koala_paged_kv kv = {};
    kv.k = kv.v = kv.k_scale = kv.v_scale = (uint8_t *)mem;
    kv.n_layers = 2; kv.n_pages = 10; kv.page_size = 64; kv.n_kv_heads = 4; kv.head_dim = 128; kv.max_batch = 3; kv.pages_per_seq = 5;
    kv.page_table = (int32_t *)mem;
    kv.ctx_len = (int32_t *)mem;
    return kv;
}
static koala_status append(const koala_paged_kv *kv, int layer = 0, int batch = 1, int rows = 2, int dt = KOALA_BF16, int heads = 8, void *q = mem,
                           int64_t qs = 1024, void *k = mem, int64_t ks = 512, void *v = mem, int64_t vs = 512, float *cos = (float *)mem,
                           float *sin = (float *)mem, int rope_rows = 100, void *q_out = mem) {
    return koala_paged_append(kv, nullptr, layer, batch, rows, dt, heads, q, qs, k, ks, v, vs, nullptr, nullptr, cos, sin, rope_rows, q_out);
}
static koala_status attend(const koala_paged_kv *kv, int layer = 0, int batch = 1, int rows = 2, int dt = KOALA_BF16, int heads = 8, void *q = mem,
                           int64_t qs = 1024, uint64_t *mask = nullptr, int64_t ms = 0, float scale = 0.1f, int max_len = 0, void *out = mem,
                           void *work = mem, size_t bytes = (size_t)-1) {
    return koala_paged_attend(kv, nullptr, layer, batch, rows, dt, heads, q, qs, mask, ms, scale, max_len, out, work, bytes);
}
static koala_status read(const koala_paged_kv *kv, int layer = 0, int layers = 1, int batch = 1, int n = 5, int dt = KOALA_BF16, void *k = mem, void *v = mem) {
    return koala_paged_read(kv, nullptr, layer, layers, batch, nullptr, n, dt, k, v);
}
static koala_status commit(const koala_paged_kv *kv, int batch = 1, int32_t *len = (int32_t *)mem, int32_t *path = (int32_t *)mem, int stride = 5,
                           int32_t *out = (int32_t *)mem) {
    return koala_paged_commit(kv, nullptr, batch, len, path, stride, out);
}

static void paged() {
    // a cache that is none: refused by every entry point alike
    auto all = [](const koala_paged_kv *kv, koala_status want) {
        EXPECT(append(kv) == want);
        EXPECT(attend(kv) == want);
        EXPECT(read(kv) == want);
        EXPECT(commit(kv) == want);
    };
    all(nullptr, KOALA_E_NULL);
    { auto c = cache(); c.k = nullptr; all(&c, KOALA_E_NULL); }
    { auto c = cache(); c.v = nullptr; all(&c, KOALA_E_NULL); }
    { auto c = cache(); c.k_scale = nullptr; all(&c, KOALA_E_NULL); }
    { auto c = cache(); c.v_scale = nullptr; all(&c, KOALA_E_NULL); }
    { auto c = cache(); c.page_table = nullptr; all(&c, KOALA_E_NULL); }
    { auto c = cache(); c.ctx_len = nullptr; all(&c, KOALA_E_NULL); }
    for (int n : {0, -1, INT_MIN}) {
        { auto c = cache(); c.n_layers = n; all(&c, KOALA_E_SHAPE); }
        { auto c = cache(); c.n_pages = n; all(&c, KOALA_E_SHAPE); }
        { auto c = cache(); c.n_kv_heads = n; all(&c, KOALA_E_SHAPE); }
        { auto c = cache(); c.pages_per_seq = n; all(&c, KOALA_E_SHAPE); }
        { auto c = cache(); c.max_batch = n; all(&c, KOALA_E_SHAPE); }
    }
    { auto c = cache(); c.n_kv_heads = 4097; all(&c, KOALA_E_SHAPE); }
    { auto c = cache(); c.pages_per_seq = INT_MAX; all(&c, KOALA_E_SHAPE); }
    for (int d : {0, 32, 96, 256, INT_MAX, -128}) { auto c = cache(); c.head_dim = d; all(&c, KOALA_E_UNSUPPORTED); }
    for (int p : {0, 8, 48, 512, INT_MAX, INT_MIN}) { auto c = cache(); c.page_size = p; all(&c, KOALA_E_UNSUPPORTED); }
    { auto c = cache(); c.k = (uint8_t *)mem + 8; all(&c, KOALA_E_ALIGN); }
    { auto c = cache(); c.v_scale = (uint8_t *)mem + 2; all(&c, KOALA_E_ALIGN); }

    const auto kv = cache();
    for (int b : {0, -1, 4, INT_MAX}) {
        EXPECT(append(&kv, 0, b) == KOALA_E_SHAPE);
        EXPECT(attend(&kv, 0, b) == KOALA_E_SHAPE);
        EXPECT(read(&kv, 0, 1, b) == KOALA_E_SHAPE);
        EXPECT(commit(&kv, b) == KOALA_E_SHAPE);
    }
    for (int l : {-1, 2, INT_MAX, INT_MIN}) {
        EXPECT(append(&kv, l) == KOALA_E_SHAPE);
        EXPECT(attend(&kv, l) == KOALA_E_SHAPE);
        EXPECT(read(&kv, l) == KOALA_E_SHAPE);
    }
    EXPECT(read(&kv, 1, 2) == KOALA_E_SHAPE && read(&kv, 0, INT_MAX) == KOALA_E_SHAPE && read(&kv, 0, 0) == KOALA_E_SHAPE);
    EXPECT(read(&kv, 0, 1, 1, 0) == KOALA_E_SHAPE && read(&kv, 0, 2, 3, INT_MAX) == KOALA_E_SHAPE);
    EXPECT(read(&kv, 0, 1, 1, 5, 9) == KOALA_E_UNSUPPORTED);
    EXPECT(read(&kv, 0, 1, 1, 5, KOALA_FP32, nullptr) == KOALA_E_NULL && read(&kv, 0, 1, 1, 5, KOALA_FP32, mem, mem + 4) == KOALA_E_ALIGN);

    EXPECT(append(&kv, 0, 1, 0) == KOALA_E_SHAPE && append(&kv, 0, 3, INT_MAX) == KOALA_E_SHAPE);
    EXPECT(append(&kv, 0, 1, 2, 5) == KOALA_E_UNSUPPORTED);
    EXPECT(append(&kv, 0, 1, 2, KOALA_BF16, -1) == KOALA_E_SHAPE && append(&kv, 0, 1, 2, KOALA_BF16, 4097) == KOALA_E_SHAPE);
    EXPECT(append(&kv, 0, 1, 2, KOALA_BF16, 8, nullptr) == KOALA_E_NULL);
    EXPECT(append(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1016) == KOALA_E_SHAPE && append(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1028) == KOALA_E_ALIGN);
    EXPECT(append(&kv, 0, 1, 2, KOALA_BF16, 8, mem + 8) == KOALA_E_ALIGN);
    EXPECT(append(&kv, 0, 1, 2, KOALA_BF16, 0, nullptr, 0, nullptr) == KOALA_E_NULL);
    EXPECT(append(&kv, 0, 1, 2, KOALA_FP32, 0, nullptr, 0, mem, 511) == KOALA_E_SHAPE);
    EXPECT(append(&kv, 0, 1, 2, KOALA_FP32, 0, nullptr, 0, mem, 514) == KOALA_E_ALIGN);
    EXPECT(append(&kv, 0, 1, 2, KOALA_FP32, 0, nullptr, 0, mem, 512, mem, LLONG_MIN) == KOALA_E_SHAPE);
    EXPECT(append(&kv, 0, 1, 2, KOALA_FP32, 0, nullptr, 0, mem, 512, mem, 512, nullptr) == KOALA_E_NULL);
    EXPECT(append(&kv, 0, 1, 2, KOALA_FP32, 0, nullptr, 0, mem, 512, mem, 512, (float *)(mem + 4)) == KOALA_E_ALIGN);
    EXPECT(append(&kv, 0, 1, 2, KOALA_FP32, 0, nullptr, 0, mem, 512, mem, 512, (float *)mem, (float *)mem, 0) == KOALA_E_SHAPE);
    EXPECT(append(&kv, 0, 3, INT_MAX / 3, KOALA_FP32, 4096, mem, 4096 * 128) == KOALA_E_SHAPE);   // more lanes than can be counted

    for (int r : {0, -1, KOALA_MAX_NODES + 1, INT_MAX}) EXPECT(attend(&kv, 0, 1, r) == KOALA_E_SHAPE);
    EXPECT(attend(&kv, 0, 1, 2, 3) == KOALA_E_UNSUPPORTED);
    for (int h : {0, 6, -4, 4100, INT_MAX}) EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, h) == KOALA_E_SHAPE);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, nullptr) == KOALA_E_NULL);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1023) == KOALA_E_SHAPE && attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1025) == KOALA_E_ALIGN);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, (uint64_t *)mem, 1) == KOALA_E_SHAPE);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, nullptr, -1) == KOALA_E_SHAPE);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, (uint64_t *)(mem + 4)) == KOALA_E_ALIGN);
    for (float s : {0.f, -1.f, NAN, INFINITY}) EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, nullptr, 0, s) == KOALA_E_SHAPE);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, nullptr, 0, 1.f, -1) == KOALA_E_SHAPE);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, nullptr, 0, 1.f, 0, mem + 8) == KOALA_E_ALIGN);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, nullptr, 0, 1.f, 0, mem, nullptr) == KOALA_E_NULL);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, nullptr, 0, 1.f, 0, mem, mem + 4) == KOALA_E_ALIGN);
    size_t need = 0;
    EXPECT(koala_paged_workspace_bytes(&kv, nullptr) == KOALA_E_NULL && koala_paged_workspace_bytes(nullptr, &need) == KOALA_E_NULL);
    EXPECT(koala_paged_workspace_bytes(&kv, &need) == KOALA_OK && need > 0);
    EXPECT(attend(&kv, 0, 1, 2, KOALA_BF16, 8, mem, 1024, nullptr, 0, 1.f, 0, mem, mem, need - 1) == KOALA_E_WORKSPACE);
    { auto c = cache(); c.head_dim = 7; EXPECT(koala_paged_workspace_bytes(&c, &need) == KOALA_E_UNSUPPORTED); }
    {   // steps are counted in 32 bits
        auto c = cache();
        c.max_batch = 1 << 20;
        c.n_kv_heads = 64;
        c.pages_per_seq = (INT_MAX - 65536) / 64;
        EXPECT(attend(&c, 0, 1 << 20, 64, KOALA_BF16, 64, mem, 64 * 128) == KOALA_E_SHAPE);
    }

    EXPECT(commit(&kv, 1, nullptr) == KOALA_E_NULL && commit(&kv, 1, (int32_t *)mem, nullptr) == KOALA_E_NULL);
    EXPECT(commit(&kv, 1, (int32_t *)mem, (int32_t *)mem, 5, nullptr) == KOALA_E_NULL);
    for (int s : {0, -1, INT_MIN}) EXPECT(commit(&kv, 1, (int32_t *)mem, (int32_t *)mem, s) == KOALA_E_SHAPE);
    {   // more lanes than can be counted, in 64 bits either
        auto c = cache();
        c.n_layers = INT_MAX;
        EXPECT(commit(&c, 3) == KOALA_E_SHAPE);
        c.max_batch = INT_MAX;
        c.n_kv_heads = 4096;
        EXPECT(commit(&c, INT_MAX) == KOALA_E_SHAPE && read(&c, 0, INT_MAX, INT_MAX, INT_MAX) == KOALA_E_SHAPE);
    }
}

int main() {
    quantizer();
    product();
    paged();
    if (failures) return 1;
    printf("host sanitize quantized: ok\n");
    return 0;
}
