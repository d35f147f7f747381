// Projections in 8-bit integers with a scale for each token and each output channel (koala.h, "Projections in 8-bit integers").
#include "koala_internal.h"

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;

__device__ __forceinline__ float bf_lo(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float bf_hi(uint32_t p) { return __uint_as_float(p & 0xFFFF0000u); }

// ---------------------------------------------------------------------------------------------
// Rows to 8 bits.  A workgroup a row; a thread holds chunks of eight values (thread, thread + threads, ...) in registers, so the
// row is read once for the sum of squares, the largest magnitude and the rounding.  Rows wider than CH chunks a thread (CH = 0) are
// read again for each of them.
// ---------------------------------------------------------------------------------------------
struct QuantArgs {
    const void *x, *gain;
    size_t ldx, ldq;
    int cols;
    float eps;
    int8_t *q;
    float *scale;
    bool gain_f32;
};

// eight consecutive elements from i on (i a multiple of 8), those at and past n zero
template <bool F32> __device__ __forceinline__ void load8(const void *src, size_t row, int i, int n, float *x) {
    if (i + 8 <= n) {
        if (F32) {
            const f32x4 *p = (const f32x4 *)((const float *)src + row + i);
            const f32x4 a = p[0], b = p[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
        } else {
            const u32x4 a = *(const u32x4 *)((const bf16_t *)src + row + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[2 * e] = bf_lo(a[e]); x[2 * e + 1] = bf_hi(a[e]); }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = i + e >= n ? 0.f : F32 ? ((const float *)src)[row + i + e] : bf_lo(((const bf16_t *)src)[row + i + e]);
    }
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
__device__ __forceinline__ unsigned wave_max(unsigned x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = max(x, (unsigned)__shfl_xor((int)x, o));
    return x;
}

template <int FORM, bool F32, int CH>
__global__ __launch_bounds__(1024) void k_quantize_rows(QuantArgs a) {
    __shared__ float s_sum[16];
    __shared__ unsigned s_top[16];
    const int tid = threadIdx.x, nt = blockDim.x, wave = tid >> 6, nw = nt >> 6, cols = a.cols;
    const size_t row = blockIdx.x, from = row * a.ldx;
    const int nch = (cols + 7) / 8;
    constexpr int HELD = CH > 0 ? CH : 1;
    float v[HELD][8];
    // the chunk's values, the norm's row factor not yet applied
    auto take = [&](int c, float *x) {
        if (FORM == KOALA_ROWS_SWIGLU) {
            float p[16];
            load8<F32>(a.x, from, 16 * c, 2 * cols, p);
            load8<F32>(a.x, from, 16 * c + 8, 2 * cols, p + 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = p[2 * e] / (1.f + expf(-p[2 * e])) * p[2 * e + 1];
        } else {
            load8<F32>(a.x, from, 8 * c, cols, x);
        }
    };
    auto gains = [&](int c, float *g) {
        if (a.gain_f32) load8<true>(a.gain, 0, 8 * c, cols, g);
        else load8<false>(a.gain, 0, 8 * c, cols, g);
    };
    if (CH > 0)
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = tid + i * nt;
            if (c < nch) take(c, v[i]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    float r = 1.f;
    if (FORM == KOALA_ROWS_NORM) {
        float sum = 0.f;
        auto add = [&](const float *x) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
        };
        if (CH > 0)
#pragma unroll
            for (int i = 0; i < HELD; ++i) add(v[i]);
        else
            for (int c = tid; c < nch; c += nt) {
                take(c, v[0]);
                add(v[0]);
            }
        sum = wave_sum(sum);
        if ((tid & 63) == 0) s_sum[wave] = sum;
        __syncthreads();
        sum = 0.f;
        for (int w = 0; w < nw; ++w) sum += s_sum[w];
        r = 1.f / sqrtf(sum / (float)cols + a.eps);
    }
    auto scaled = [&](int c, float *x) {
        if (FORM != KOALA_ROWS_NORM) return;
        float g[8];
        gains(c, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * r * g[e];
    };
    // the largest magnitude by its bits: an infinity or not-a-number is larger than any number
    unsigned top = 0;
    auto look = [&](const float *x) {
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    };
    if (CH > 0)
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = tid + i * nt;
            if (c < nch) scaled(c, v[i]);
            look(v[i]);
        }
    else
        for (int c = tid; c < nch; c += nt) {
            take(c, v[0]);
            scaled(c, v[0]);
            look(v[0]);
        }
    top = wave_max(top);
    if ((tid & 63) == 0) s_top[wave] = top;
    __syncthreads();
    top = 0;
    for (int w = 0; w < nw; ++w) top = max(top, s_top[w]);
    const bool bad = top >= 0x7F800000u;
    float scale = __uint_as_float(top) / 127.f;
    if (!(scale > 0.f)) scale = 1.f;   // all zero (or so small that a scale would be): whole numbers are zero
    if (tid == 0) a.scale[row] = bad ? __builtin_nanf("") : scale;
    auto put = [&](int c, const float *x) {
        uint32_t w[2] = {0, 0};
        if (!bad)
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e >> 2] |= ((uint32_t)(int)rintf(x[e] / scale) & 0xFFu) << (8 * (e & 3));
        *(u32x2 *)(a.q + row * a.ldq + 8 * c) = (u32x2){w[0], w[1]};
    };
    if (CH > 0)
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = tid + i * nt;
            if (c < nch) put(c, v[i]);
        }
    else
        for (int c = tid; c < nch; c += nt) {
            take(c, v[0]);
            scaled(c, v[0]);
            put(c, v[0]);
        }
    if (tid == 0 && (nch & 1)) *(u32x2 *)(a.q + row * a.ldq + 8 * nch) = (u32x2){0u, 0u};
}

// ---------------------------------------------------------------------------------------------
// Products.  The matrix pipe multiplies 16 output channels by 16 rows over 64 terms: a lane holds 16 consecutive terms of one
// channel or row, which is 16 bytes of the row-major matrix as it lies in memory.
// ---------------------------------------------------------------------------------------------
struct LinearArgs {
    const int8_t *q, *w;
    size_t ldq, ldw, ldy;
    const float *q_scale, *w_scale;
    const void *add;
    void *y;
    int rows, out, in;
    int splits;
    int *part;     // [splits][rows][out] where splits > 1
};

// the four consecutive outputs n .. n + 3 of row m from their sums
template <bool F32> __device__ __forceinline__ void finish4(const LinearArgs &a, int m, int n, i32x4 s) {
    if (m >= a.rows || n >= a.out) return;
    const float qs = a.q_scale[m];
    const size_t at = (size_t)m * a.ldy + n;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = n + e < a.out ? (float)s[e] * qs * a.w_scale[n + e] : 0.f;
    if (F32) {
        const float *add = a.add ? (const float *)a.add + at : nullptr;
        float *y = (float *)a.y + at;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.out) y[e] = v[e] + (add ? add[e] : 0.f);
    } else {
        const bf16_t *add = a.add ? (const bf16_t *)a.add + at : nullptr;
        bf16_t *y = (bf16_t *)a.y + at;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.out)
                y[e] = (bf16_t)__builtin_bit_cast(uint16_t, (__bf16)(v[e] + (add ? bf_lo(add[e]) : 0.f)));
    }
}

// Row groups: a workgroup owns 16 U output channels and MT row tiles, its waves take the 64-term steps in turn, both operands
// straight from memory into registers, and meet in LDS.
template <int U, int MT, int NW, bool F32>
__global__ __launch_bounds__(64 * NW) void k_linear_rows(LinearArgs a) {
    __shared__ i32x4 red[NW][U * MT][64];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63, li = l & 15, lg = l >> 4;
    const int n0 = blockIdx.x * (16 * U), m0 = blockIdx.y * (16 * MT);
    const int8_t *wp[U], *xp[MT];
#pragma unroll
    for (int u = 0; u < U; ++u) wp[u] = a.w + (size_t)min(n0 + 16 * u + li, a.out - 1) * a.ldw;
#pragma unroll
    for (int m = 0; m < MT; ++m) xp[m] = a.q + (size_t)min(m0 + 16 * m + li, a.rows - 1) * a.ldq;
    i32x4 acc[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[u][m] = (i32x4){0, 0, 0, 0};
    for (int k0 = wave * 64; k0 < a.in; k0 += NW * 64) {
        const int k = k0 + 16 * lg;
        const bool in = k < a.in;         // past the end: any weights, times zero
        const int kk = in ? k : 0;
        i32x4 x[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            x[m] = *(const i32x4 *)(xp[m] + kk);
            if (!in) x[m] = (i32x4){0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const i32x4 w = *(const i32x4 *)(wp[u] + kk);
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[u][m] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x[m], acc[u][m], 0, 0, 0);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int m = 0; m < MT; ++m) red[wave][u * MT + m][l] = acc[u][m];
    __syncthreads();
    for (int p = wave; p < U * MT; p += NW) {
        i32x4 s = red[0][p][l];
        for (int v = 1; v < NW; ++v) s += red[v][p][l];
        finish4<F32>(a, m0 + 16 * (p % MT) + li, n0 + 16 * (p / MT) + 4 * lg, s);
    }
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }
koala_status launched() { return hipGetLastError() == hipSuccess ? KOALA_OK : KOALA_E_DEVICE; }

template <int FORM, bool F32> void quantize(hipStream_t st, const QuantArgs &a, int rows) {
    const int nch = (a.cols + 7) / 8;
    const int threads = nch >= 1024 ? 1024 : (nch + 63) / 64 * 64;
    if (nch <= threads) k_quantize_rows<FORM, F32, 1><<<rows, threads, 0, st>>>(a);
    else if (nch <= 2 * threads) k_quantize_rows<FORM, F32, 2><<<rows, threads, 0, st>>>(a);
    else if (nch <= 4 * threads) k_quantize_rows<FORM, F32, 4><<<rows, threads, 0, st>>>(a);
    else k_quantize_rows<FORM, F32, 0><<<rows, threads, 0, st>>>(a);
}

}  // namespace

extern "C" {

koala_status koala_quantize_rows(void *hip_stream, int form, int x_dtype, int rows, int cols, const void *x, int64_t x_stride,
                                 const void *gain, int gain_dtype, float eps, int8_t *q, int64_t q_stride, float *scale) {
    if (!x || !q || !scale || (form == KOALA_ROWS_NORM && !gain)) return KOALA_E_NULL;
    if (form < KOALA_ROWS_PLAIN || form > KOALA_ROWS_SWIGLU || (x_dtype != KOALA_FP32 && x_dtype != KOALA_BF16) ||
        (form == KOALA_ROWS_NORM && gain_dtype != KOALA_FP32 && gain_dtype != KOALA_BF16))
        return KOALA_E_UNSUPPORTED;
    if (rows < 1 || cols < 1 || cols > (1 << 30) || x_stride < (form == KOALA_ROWS_SWIGLU ? 2ll * cols : cols) ||
        q_stride < (cols + 15) / 16 * 16 || (form == KOALA_ROWS_NORM && !(eps >= 0.f)))
        return KOALA_E_SHAPE;
    if (!aligned16(x) || !aligned16(q) || ((uintptr_t)scale & 3) || (x_stride * (x_dtype == KOALA_FP32 ? 4 : 2)) % 16 || q_stride % 16 ||
        (form == KOALA_ROWS_NORM && !aligned16(gain)))
        return KOALA_E_ALIGN;
    QuantArgs a{x, gain, (size_t)x_stride, (size_t)q_stride, cols, eps, q, scale, gain_dtype == KOALA_FP32};
    hipStream_t st = (hipStream_t)hip_stream;
    const bool f = x_dtype == KOALA_FP32;
    switch (form) {
    case KOALA_ROWS_PLAIN: f ? quantize<KOALA_ROWS_PLAIN, true>(st, a, rows) : quantize<KOALA_ROWS_PLAIN, false>(st, a, rows); break;
    case KOALA_ROWS_NORM: f ? quantize<KOALA_ROWS_NORM, true>(st, a, rows) : quantize<KOALA_ROWS_NORM, false>(st, a, rows); break;
    default: f ? quantize<KOALA_ROWS_SWIGLU, true>(st, a, rows) : quantize<KOALA_ROWS_SWIGLU, false>(st, a, rows); break;
    }
    return launched();
}

koala_status koala_linear_workspace_bytes(int rows, int out_features, int in_features, size_t *out) {
    if (!out) return KOALA_E_NULL;
    if (rows < 1 || out_features < 1 || in_features < 16 || in_features % 16 || in_features > 131056) return KOALA_E_SHAPE;
    *out = 0;
    return KOALA_OK;
}

koala_status koala_linear_quantized(void *hip_stream, int rows, int out_features, int in_features, const int8_t *q, int64_t q_stride,
                                    const float *q_scale, const int8_t *w, int64_t w_stride, const float *w_scale, int y_dtype,
                                    const void *add, void *y, int64_t y_stride, void *workspace, size_t workspace_bytes) {
    if (!q || !q_scale || !w || !w_scale || !y) return KOALA_E_NULL;
    if (y_dtype != KOALA_FP32 && y_dtype != KOALA_BF16) return KOALA_E_UNSUPPORTED;
    size_t need = 0;
    const koala_status rc = koala_linear_workspace_bytes(rows, out_features, in_features, &need);
    if (rc != KOALA_OK) return rc;
    if (q_stride < in_features || w_stride < in_features || y_stride < out_features) return KOALA_E_SHAPE;
    if (!aligned16(q) || !aligned16(w) || q_stride % 16 || w_stride % 16 || !aligned16(workspace) || ((uintptr_t)q_scale & 3) || ((uintptr_t)w_scale & 3) ||
        ((uintptr_t)y & (y_dtype == KOALA_FP32 ? 3 : 1)) || ((uintptr_t)add & (y_dtype == KOALA_FP32 ? 3 : 1)))
        return KOALA_E_ALIGN;
    if (need > 0 && (!workspace || workspace_bytes < need)) return KOALA_E_WORKSPACE;
    LinearArgs a{q, w, (size_t)q_stride, (size_t)w_stride, (size_t)y_stride, q_scale, w_scale, add, y, rows, out_features, in_features, 1, (int *)workspace};
    hipStream_t st = (hipStream_t)hip_stream;
    const dim3 g((out_features + 31) / 32, (rows + 63) / 64);
    if (g.y > 65535) return KOALA_E_SHAPE;
    if (y_dtype == KOALA_FP32) k_linear_rows<2, 4, 4, true><<<g, 256, 0, st>>>(a);
    else k_linear_rows<2, 4, 4, false><<<g, 256, 0, st>>>(a);
    return launched();
}

}  // extern "C"
