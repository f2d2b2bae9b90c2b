// The dense operators' passes over rows: dropout, quantisation, the join of a product's parts
// and the bias gradients' sums.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "dense.h"
#include "dense_math.h"

namespace geot {
namespace {

constexpr int kRowsBlock = 256;

unsigned grid_1d(int64_t items, int64_t per_block, int64_t most) {
    return (unsigned)std::min(std::max<int64_t>((items + per_block - 1) / per_block, 1), most);
}

// out = res + drop(x), eight columns (two blocks of words) a thread. Bound by memory: one read, one write
// of each element and the words in between.
template <int E, bool RES>
__global__ void __launch_bounds__(kRowsBlock) dropout_kernel(const void *x, int64_t ldx, const void *res, int64_t ldr,
                                                             int64_t rows, int64_t F, int64_t groups, const Drop d,
                                                             void *out, int64_t ldo) {
    const int64_t total = rows * groups, step = (int64_t)gridDim.x * kRowsBlock;
    for (int64_t i = (int64_t)blockIdx.x * kRowsBlock + threadIdx.x; i < total; i += step) {
        const int64_t r = i / groups, f = (i - r * groups) * 8, count = F - f;
        float v[8];
        load_wide<E, 8>(x, r * ldx + f, count, v);
        if (d.on) {
            drop4(v, (uint32_t)(f >> 2), (uint32_t)r, d);
            drop4(v + 4, (uint32_t)(f >> 2) + 1, (uint32_t)r, d);
        }
        if constexpr (RES) {
            float b[8];
            load_wide<E, 8>(res, r * ldr + f, count, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += b[j];
        }
        store_wide<E, 8>(out, r * ldo + f, count, v);
    }
}

// One wave a row: the largest magnitude, then x * (127 / largest) rounded to nearest even. A row that
// holds NaN or an infinity has no scale: it gets scale NaN and zeros, so that every product of it is NaN.
// The largest magnitude counts as at least 2^-100, so the factor stays finite.
template <int E>
__global__ void __launch_bounds__(kRowsBlock) quantize_kernel(const void *x, int64_t ldx, int64_t rows, int64_t F,
                                                              int8_t *q, int64_t ldq, float *scale) {
    const int lane = threadIdx.x & 63;
    const int64_t step = (int64_t)gridDim.x * (kRowsBlock / 64);
    for (int64_t r = (int64_t)blockIdx.x * (kRowsBlock / 64) + (threadIdx.x >> 6); r < rows; r += step) {
        float top = 0.0f;
        for (int64_t f = lane * 8; f < F; f += 512) {
            float v[8];
            load_wide<E, 8>(x, r * ldx + f, F - f, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = __builtin_elementwise_maximum(top, fabsf(v[j]));
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, o));
        const bool finite = top < INFINITY;
        const float a = fmaxf(top, 0x1p-100f), k = 127.0f / a;
        if (lane == 0) scale[r] = finite ? a / 127.0f : NAN;
        for (int64_t f = lane * 8; f < F; f += 512) {
            float v[8];
            const int64_t count = F - f;
            load_wide<E, 8>(x, r * ldx + f, count, v);
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int n = finite ? (int)rintf(v[j] * k) : 0;
                w[j / 4] |= (uint32_t)(n & 255) << (j % 4 * 8);
            }
            int8_t *p = q + r * ldq + f;
            typedef uint32_t two __attribute__((ext_vector_type(2), aligned(1)));
            if (count >= 8) {
                *reinterpret_cast<two *>(p) = two{w[0], w[1]};
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < count) p[j] = (int8_t)(w[j / 4] >> (j % 4 * 8));
            }
        }
    }
}

// The parts of a product added in order, then its epilogue: four columns a thread.
template <int E, int EPI, bool DUAL>
__global__ void __launch_bounds__(kRowsBlock) join_kernel(const DenseArgs a) {
    typedef typename std::conditional<E == ELEM_I8, int, float>::type Sum;
    const int64_t groups = (a.N + 3) / 4, total = a.M * groups, step = (int64_t)gridDim.x * kRowsBlock;
    const int64_t C = DUAL ? 2 * a.N : a.N, slab = a.M * C;
    for (int64_t i = (int64_t)blockIdx.x * kRowsBlock + threadIdx.x; i < total; i += step) {
        const int64_t m = i / groups, n = (i - m * groups) * 4, count = a.N - n;
        Sum g[4] = {0, 0, 0, 0}, u[4] = {0, 0, 0, 0};
        const Sum *p = (const Sum *)a.part + m * C + n;
        for (int s = 0; s < a.splits; ++s, p += slab) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < count) {
                    g[j] += p[j];
                    if constexpr (DUAL) u[j] += p[a.N + j];
                }
        }
        Columns<4> c;
        load_columns<E, EPI, 4>(a, n, c);
        if constexpr (EPI == DENSE_GATED)
            with_act(a.act, [&](auto act) { finish<E, EPI, decltype(act)::value, 4, DUAL>(a, 0, m, n, c, g, u); });
        else
            finish<E, EPI, ACT_NONE, 4, DUAL>(a, 0, m, n, c, g, u);
    }
}

// mid[y][c] = the sum of rows y, y + kColsumMid, ... of colsum
__global__ void __launch_bounds__(kRowsBlock) colsum_mid_kernel(const float *colsum, int64_t rows, int64_t C, float *mid) {
    const int64_t c = (int64_t)blockIdx.x * kRowsBlock + threadIdx.x;
    if (c >= C) return;
    float s = 0.0f;
    for (int64_t r = blockIdx.y; r < rows; r += kColsumMid) s += colsum[r * C + c];
    mid[blockIdx.y * C + c] = s;
}

template <int E>
__global__ void __launch_bounds__(kRowsBlock) colsum_kernel(const float *mid, int64_t N, void *out0, void *out1) {
    const int64_t c = (int64_t)blockIdx.x * kRowsBlock + threadIdx.x;
    if (c >= 2 * N) return;
    float s = 0.0f;
    for (int r = 0; r < kColsumMid; ++r) s += mid[r * 2 * N + c];
    void *out = c < N ? out0 : out1;
    if (out) store_wide<E, 1>(out, c < N ? c : c - N, 1, &s);
}

template <int E>
hipError_t dropout_of(const void *x, int64_t ldx, const void *res, int64_t ldr, int64_t rows, int64_t F, const Drop &d,
                      void *out, int64_t ldo, hipStream_t st) {
    const int64_t groups = (F + 7) / 8;
    const dim3 grid(grid_1d(rows * groups, kRowsBlock, 8192));
    if (res)
        hipLaunchKernelGGL((dropout_kernel<E, true>), grid, dim3(kRowsBlock), 0, st, x, ldx, res, ldr, rows, F, groups, d,
                           out, ldo);
    else
        hipLaunchKernelGGL((dropout_kernel<E, false>), grid, dim3(kRowsBlock), 0, st, x, ldx, res, ldr, rows, F, groups, d,
                           out, ldo);
    return hipGetLastError();
}

template <int E>
hipError_t quantize_of(const void *x, int64_t ldx, int64_t rows, int64_t F, int8_t *q, int64_t ldq, float *scale,
                       hipStream_t st) {
    hipLaunchKernelGGL(quantize_kernel<E>, dim3(grid_1d(rows, kRowsBlock / 64, 16384)), dim3(kRowsBlock), 0, st, x, ldx,
                       rows, F, q, ldq, scale);
    return hipGetLastError();
}

template <int E, int EPI, bool DUAL>
hipError_t join_of(const DenseArgs &a, hipStream_t st) {
    hipLaunchKernelGGL((join_kernel<E, EPI, DUAL>), dim3(grid_1d(a.M * ((a.N + 3) / 4), kRowsBlock, 16384)),
                       dim3(kRowsBlock), 0, st, a);
    return hipGetLastError();
}

template <int E>
hipError_t join_float(int epi, const DenseArgs &a, hipStream_t st) {
    if (epi == DENSE_GATED) return join_of<E, DENSE_GATED, true>(a, st);
    if (epi == DENSE_PLAIN) return join_of<E, DENSE_PLAIN, false>(a, st);
    return hipErrorInvalidValue;
}

template <int E>
hipError_t colsum_of(const float *mid, int64_t N, unsigned gx, void *out0, void *out1, hipStream_t st) {
    hipLaunchKernelGGL(colsum_kernel<E>, dim3(gx), dim3(kRowsBlock), 0, st, mid, N, out0, out1);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int elem, const void *x, int64_t ldx, const void *res, int64_t ldr, int64_t rows, int64_t F,
                          const Drop &d, void *out, int64_t ldo, hipStream_t st) {
    if (elem == ELEM_F32) return dropout_of<ELEM_F32>(x, ldx, res, ldr, rows, F, d, out, ldo, st);
    if (elem == ELEM_BF16) return dropout_of<ELEM_BF16>(x, ldx, res, ldr, rows, F, d, out, ldo, st);
    if (elem == ELEM_F16) return dropout_of<ELEM_F16>(x, ldx, res, ldr, rows, F, d, out, ldo, st);
    return hipErrorInvalidValue;
}

hipError_t launch_quantize_rows(int elem, const void *x, int64_t ldx, int64_t rows, int64_t F, int8_t *q, int64_t ldq,
                                float *scale, hipStream_t st) {
    if (elem == ELEM_F32) return quantize_of<ELEM_F32>(x, ldx, rows, F, q, ldq, scale, st);
    if (elem == ELEM_BF16) return quantize_of<ELEM_BF16>(x, ldx, rows, F, q, ldq, scale, st);
    if (elem == ELEM_F16) return quantize_of<ELEM_F16>(x, ldx, rows, F, q, ldq, scale, st);
    return hipErrorInvalidValue;
}

hipError_t launch_dense_join(int elem, int epi, const DenseArgs &a, hipStream_t st) {
    if (elem == ELEM_I8 && epi == DENSE_I8) return join_of<ELEM_I8, DENSE_I8, false>(a, st);
    if (elem == ELEM_F32) return join_float<ELEM_F32>(epi, a, st);
    if (elem == ELEM_BF16) return join_float<ELEM_BF16>(epi, a, st);
    if (elem == ELEM_F16) return join_float<ELEM_F16>(epi, a, st);
    return hipErrorInvalidValue;
}

hipError_t launch_colsum(int elem, const float *colsum, int64_t rows, int64_t N, float *mid, void *out0, void *out1,
                         hipStream_t st) {
    const unsigned gx = (unsigned)((2 * N + kRowsBlock - 1) / kRowsBlock);
    hipLaunchKernelGGL(colsum_mid_kernel, dim3(gx, (unsigned)kColsumMid), dim3(kRowsBlock), 0, st, colsum, rows, 2 * N,
                       mid);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (elem == ELEM_F32) return colsum_of<ELEM_F32>(mid, N, gx, out0, out1, st);
    if (elem == ELEM_BF16) return colsum_of<ELEM_BF16>(mid, N, gx, out0, out1, st);
    return colsum_of<ELEM_F16>(mid, N, gx, out0, out1, st);
}

}  // namespace geot
