// The matrix products of the dense operators on gfx950's matrix instructions.
//
// C[m, n] = sum_k A[m, k] B[n, k]: rows m are graph nodes (tokens), columns n output channels. A block
// takes a BM x BN tile and walks K in steps of 128 bytes of a row (64 16-bit, 32 fp32 or 128 8-bit
// elements), so one layout serves every type: a tile of R rows is R x 128 bytes in LDS, each row eight
// 16-byte chunks, and a lane's operand of a 16 x 16 matrix instruction is one chunk of its row (k in the
// order of the chunks, the same for both operands, so the order inside K does not matter).
//
// The weights are the instruction's row operand: its result then holds, in one lane, consecutive output
// columns of one row m. Weight rows are dealt to the fragments so that a lane's fragments together hold
// 4 * PF consecutive columns (n = 4 * PF * (lane / 16) + 4 f + i), one wide store a row.
//
// Chunks are exchanged inside their row by an XOR with a key of the row that differs between any eight
// lanes that read one bank group in one cycle.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "common.h"
#include "dense.h"
#include "dense_math.h"

namespace geot {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
// 16 bytes at any address of the element's alignment (global memory takes any alignment in one load)
typedef uint32_t chunk_any __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t chunk_t __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;

template <int E>
struct AccOf {
    typedef f32x4 type;
    typedef float scalar;
};
template <>
struct AccOf<ELEM_I8> {
    typedef i32x4 type;
    typedef int scalar;
};

// acc += W (16 x chunk of k) X^T: one matrix instruction (four for fp32, which has 16 x 16 x 4)
template <int E>
__device__ __forceinline__ typename AccOf<E>::type mma(chunk_t w, chunk_t x, typename AccOf<E>::type acc) {
    if constexpr (E == ELEM_BF16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc,
                                                       0, 0, 0);
    } else if constexpr (E == ELEM_F16) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), acc, 0,
                                                      0, 0);
    } else if constexpr (E == ELEM_I8) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, x), acc, 0,
                                                     0, 0);
    } else {
        const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], acc, 0, 0, 0);
        return acc;
    }
}

// 16 bytes at p, of which the row holds `left` (from p; any number); bytes beyond are 0 and not read
template <int E>
__device__ __forceinline__ chunk_t load_chunk(const char *p, int64_t left) {
    if (left >= 16) return *reinterpret_cast<const chunk_any *>(p);
    constexpr int ES = E == ELEM_F32 ? 4 : E == ELEM_I8 ? 1 : 2;
    chunk_t v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16 / ES; ++i) {
        if (i * ES < left) {
            uint32_t x;
            if constexpr (ES == 4) x = reinterpret_cast<const uint32_t *>(p)[i];
            else if constexpr (ES == 2) x = reinterpret_cast<const uint16_t *>(p)[i];
            else x = reinterpret_cast<const uint8_t *>(p)[i];
            v[i * ES / 4] |= x << (i * ES % 4 * 8);
        }
    }
    return v;
}

template <int E, int BM, int BN, int WM, int WN, int EPI, bool DUAL>
__global__ void __launch_bounds__(WM * WN * 64) dense_kernel(const DenseArgs a) {
    constexpr int T = WM * WN * 64;
    constexpr int ES = E == ELEM_F32 ? 4 : E == ELEM_I8 ? 1 : 2;
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int PF = DUAL ? FN / 2 : FN;          // fragments of one column operand
    constexpr int NV = 4 * PF;                      // consecutive columns of one lane
    constexpr int CA = BM * 8 / T, CB = BN * 8 / T; // chunks a thread stages
    constexpr int HB = DUAL ? BN / 2 : BN;          // columns of one operand in the tile
    typedef typename AccOf<E>::type Acc;
    __shared__ __align__(16) char lds[2][(BM + BN) * kStepBytes];

    // Blocks go round the chiplets in turn: give each chiplet a run of neighbouring tiles, so that what
    // they share stays in its L2.
    const int64_t nb = gridDim.x, b = blockIdx.x, x8 = b & 7, q8 = nb >> 3, r8 = nb & 7;
    const int64_t id = x8 * q8 + (x8 < r8 ? x8 : r8) + (b >> 3);
    const int64_t tiles = a.tiles_m * a.tiles_n;
    const int64_t split = id / tiles, t = id - split * tiles;
    // tiles in groups of 8 rows of tiles
    const int64_t per = 8 * a.tiles_n, grp = t / per, gm = a.tiles_m - grp * 8 < 8 ? a.tiles_m - grp * 8 : 8;
    const int64_t tm = grp * 8 + (t - grp * per) % gm, tn = (t - grp * per) / gm;
    const int64_t m0 = tm * BM, n0 = tn * HB;

    const int64_t kbytes = a.K * ES;
    const int64_t all = (kbytes + kStepBytes - 1) / kStepBytes;
    const int64_t s0 = split * a.steps_per, s1 = s0 + a.steps_per < all ? s0 + a.steps_per : all;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave % WM, wn = wave / WM;

    // staging: thread's chunk c of row (tid + c T) / 8. Rows beyond the end read the last row; what
    // they give is never stored.
    const char *pa[CA], *pb[CB];
    int la[CA], lb[CB];
    const int chunk = tid & 7;
#pragma unroll
    for (int c = 0; c < CA; ++c) {
        const int row = (tid + c * T) >> 3;
        const int64_t m = m0 + row < a.M ? m0 + row : a.M - 1;
        pa[c] = (const char *)a.a + m * a.lda * ES + chunk * 16;
        la[c] = row * kStepBytes + ((chunk ^ (row & 7)) << 4);
    }
#pragma unroll
    for (int c = 0; c < CB; ++c) {
        const int row = (tid + c * T) >> 3, col = DUAL ? row % HB : row;
        const int64_t n = n0 + col < a.N ? n0 + col : a.N - 1;
        const void *base = DUAL && row >= HB ? a.b1 : a.b0;
        pb[c] = (const char *)base + n * a.ldb * ES + chunk * 16;
        const int key = (row & 3) | (((row / NV) & 1) << 2);
        lb[c] = (BM + row) * kStepBytes + ((chunk ^ key) << 4);
    }

    Acc acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Acc{0, 0, 0, 0};

    chunk_t ra[CA], rb[CB];
    auto fetch = [&](int64_t s) {
        const int64_t at = s * kStepBytes, left = kbytes - at - chunk * 16;
        if (at + kStepBytes <= kbytes) {
#pragma unroll
            for (int c = 0; c < CA; ++c) ra[c] = *reinterpret_cast<const chunk_any *>(pa[c] + at);
#pragma unroll
            for (int c = 0; c < CB; ++c) rb[c] = *reinterpret_cast<const chunk_any *>(pb[c] + at);
        } else {
#pragma unroll
            for (int c = 0; c < CA; ++c) ra[c] = load_chunk<E>(pa[c] + at, left);
#pragma unroll
            for (int c = 0; c < CB; ++c) rb[c] = load_chunk<E>(pb[c] + at, left);
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int c = 0; c < CA; ++c) *reinterpret_cast<chunk_t *>(&lds[buf][la[c]]) = ra[c];
#pragma unroll
        for (int c = 0; c < CB; ++c) *reinterpret_cast<chunk_t *>(&lds[buf][lb[c]]) = rb[c];
    };

    // fragment addresses: row of the tile and its key; the chunk is (4 kk + lane / 16) ^ key
    const int r16 = lane & 15, c4 = lane >> 4;
    const int arow = wm * (BM / WM) + r16, akey = arow & 7;
    int brow[FN], bkey[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
        const int f = j % PF;
        const int row = (j / PF) * HB + wn * (16 * PF) + NV * (r16 >> 2) + 4 * f + (r16 & 3);
        brow[j] = (BM + row) * kStepBytes;
        bkey[j] = (row & 3) | (((row / NV) & 1) << 2);
    }

    if (s0 < s1) {
        fetch(s0);
        put(0);
    }
    __syncthreads();
    for (int64_t s = s0; s < s1; ++s) {
        const int buf = (int)(s - s0) & 1;
        if (s + 1 < s1) fetch(s + 1);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            chunk_t fa[FM], fb[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j)
                fb[j] = *reinterpret_cast<const chunk_t *>(&lds[buf][brow[j] + (((4 * kk + c4) ^ bkey[j]) << 4)]);
#pragma unroll
            for (int i = 0; i < FM; ++i)
                fa[i] = *reinterpret_cast<const chunk_t *>(
                    &lds[buf][(arow + 16 * i) * kStepBytes + (((4 * kk + c4) ^ akey) << 4)]);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mma<E>(fb[j], fa[i], acc[i][j]);
        }
        if (s + 1 < s1) put(buf ^ 1);
        __syncthreads();
    }

    // epilogue: this lane has columns n .. n + NV of rows m + 16 i
    const int64_t n = n0 + wn * (16 * PF) + NV * c4;
    const int64_t mrow = m0 + wm * (BM / WM) + r16;
    float csg[NV], csu[NV];
    if constexpr (EPI == DENSE_GATED_BWD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) csg[v] = csu[v] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t m = mrow + 16 * i;
        if (m < a.M && n < a.N) {
            typename AccOf<E>::scalar g[NV], u[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                g[v] = acc[i][v / 4][v % 4];
                if constexpr (DUAL) u[v] = acc[i][PF + v / 4][v % 4];
            }
            finish<E, EPI, NV, DUAL>(a, split, m, n, g, u);
            if constexpr (EPI == DENSE_GATED_BWD) {
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    csg[v] += g[v];
                    csu[v] += u[v];
                }
            }
        }
    }
    if constexpr (EPI == DENSE_GATED_BWD) {
        if (a.colsum) {
            float *dst = a.colsum + (tm * WM + wm) * 2 * a.N;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) {
                    csg[v] += __shfl_xor(csg[v], o);
                    csu[v] += __shfl_xor(csu[v], o);
                }
                if (r16 == 0 && n + v < a.N) {
                    dst[n + v] = csg[v];
                    dst[a.N + n + v] = csu[v];
                }
            }
        }
    }
}

template <int E, int EPI, bool DUAL>
hipError_t launch_tile(int big, const DenseArgs &a, int64_t blocks, hipStream_t st) {
    if (big)
        hipLaunchKernelGGL((dense_kernel<E, 256, 256, 2, 4, EPI, DUAL>), dim3((unsigned)blocks), dim3(512), 0, st, a);
    else
        hipLaunchKernelGGL((dense_kernel<E, 128, 128, 2, 2, EPI, DUAL>), dim3((unsigned)blocks), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int E>
hipError_t launch_float(int epi, bool dual, int big, const DenseArgs &a, int64_t blocks, hipStream_t st) {
    switch (epi) {
        case DENSE_GATED: return launch_tile<E, DENSE_GATED, true>(big, a, blocks, st);
        case DENSE_GATED_BWD: return launch_tile<E, DENSE_GATED_BWD, true>(big, a, blocks, st);
        case DENSE_PLAIN: return launch_tile<E, DENSE_PLAIN, false>(big, a, blocks, st);
        case DENSE_PART:
            return dual ? launch_tile<E, DENSE_PART, true>(big, a, blocks, st)
                        : launch_tile<E, DENSE_PART, false>(big, a, blocks, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace
}  // namespace geot
