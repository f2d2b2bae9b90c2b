// What the sums of a product's row become: the activations of the gated block with their derivatives, its
// dropout, the 8-bit product's scales, and the stores. Everything is computed in fp32; each output is
// rounded once, to nearest even, when it is stored in a 16-bit type.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dense.h"

namespace geot {
namespace {

// element type of storage
template <int E>
struct StoreOf {
    typedef float type;
};
template <>
struct StoreOf<ELEM_BF16> {
    typedef __bf16 type;
};
template <>
struct StoreOf<ELEM_F16> {
    typedef _Float16 type;
};

// V elements at any address that the element's own alignment allows
template <int E, int V>
struct Pack {
    typedef typename StoreOf<E>::type type __attribute__((ext_vector_type(V), aligned(sizeof(typename StoreOf<E>::type))));
};

// v[0..V) = p[0..V), the first `count` of them (the others 0)
template <int E, int V>
__device__ __forceinline__ void load_wide(const void *base, int64_t at, int64_t count, float *v) {
    const auto *p = (const typename StoreOf<E>::type *)base + at;
    constexpr int W = E == ELEM_F32 ? 4 : 8, S = V < W ? V : W;
    if (count >= V) {
#pragma unroll
        for (int i = 0; i < V; i += S) {
            const auto x = *reinterpret_cast<const typename Pack<E, S>::type *>(p + i);
#pragma unroll
            for (int j = 0; j < S; ++j) v[i + j] = (float)x[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = i < count ? (float)p[i] : 0.0f;
    }
}

template <int E, int V>
__device__ __forceinline__ void store_wide(void *base, int64_t at, int64_t count, const float *v) {
    auto *p = (typename StoreOf<E>::type *)base + at;
    constexpr int W = E == ELEM_F32 ? 4 : 8, S = V < W ? V : W;
    if (count >= V) {
#pragma unroll
        for (int i = 0; i < V; i += S) {
            typename Pack<E, S>::type x;
#pragma unroll
            for (int j = 0; j < S; ++j) x[j] = (typename StoreOf<E>::type)v[i + j];
            *reinterpret_cast<typename Pack<E, S>::type *>(p + i) = x;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < count) p[i] = (typename StoreOf<E>::type)v[i];
    }
}

// 16-bit results take the short exponential and reciprocal (a few units of the 24th bit), fp32 ones the
// library's.
template <int E>
__device__ __forceinline__ float sigmoid(float g) {
    if constexpr (E == ELEM_F32) return 1.0f / (1.0f + expf(-g));
    else return __builtin_amdgcn_rcpf(1.0f + __expf(-g));
}

// the activation, and its derivative in *d
template <int E>
__device__ __forceinline__ float activate(int act, float g, float *d) {
    switch (act) {
        case ACT_SILU: {
            const float s = sigmoid<E>(g);
            *d = s * (1.0f + g * (1.0f - s));
            return g * s;
        }
        case ACT_GELU: {
            const float c = 0.5f * (1.0f + erff(g * 0.70710678f));
            const float e = E == ELEM_F32 ? expf(-0.5f * g * g) : __expf(-0.5f * g * g);
            *d = c + g * e * 0.39894228f;
            return g * c;
        }
        case ACT_RELU:
            *d = g > 0.0f ? 1.0f : 0.0f;
            return g > 0.0f ? g : (g != g ? g : 0.0f);
        case ACT_SIGMOID: {
            const float s = sigmoid<E>(g);
            *d = s * (1.0f - s);
            return s;
        }
        default: *d = 1.0f; return g;
    }
}

// Row m, columns n .. n + NV (as many as there are) of the product. g, u: the sums on entry;
// DENSE_GATED_BWD leaves dG, dU there (0 beyond the last column).
template <int E, int EPI, int NV, bool DUAL, class Sum>
__device__ __forceinline__ void finish(const DenseArgs &a, int64_t split, int64_t m, int64_t n, Sum *g, Sum *u) {
    const int64_t count = a.N - n;
    if constexpr (EPI == DENSE_PART) {
        const int64_t C = DUAL ? 2 * a.N : a.N;
        Sum *p = (Sum *)a.part + (split * a.M + m) * C + n;
#pragma unroll
        for (int h = 0; h < (DUAL ? 2 : 1); ++h) {
            const Sum *s = h ? u : g;
            typedef Sum Vec __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
            for (int v = 0; v < NV; v += 4) {
                if (v + 4 <= count) {
                    *reinterpret_cast<Vec *>(p + h * a.N + v) = Vec{s[v], s[v + 1], s[v + 2], s[v + 3]};
                } else {
#pragma unroll
                    for (int i = v; i < v + 4; ++i)
                        if (i < count) p[h * a.N + i] = s[i];
                }
            }
        }
    } else if constexpr (EPI == DENSE_PLAIN) {
        const bool second = a.out1 && m >= a.rows0;
        store_wide<E, NV>(second ? a.out1 : a.out, (second ? m - a.rows0 : m) * a.ldo + n, count, (const float *)g);
    } else if constexpr (EPI == DENSE_I8) {
        float y[NV], sw[NV], bias[NV];
        const float sx = a.sx[m];
        load_wide<ELEM_F32, NV>(a.sw, n, count, sw);
        if (a.bias0) load_wide<ELEM_F32, NV>(a.bias0, n, count, bias);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            y[v] = (float)g[v] * sx * sw[v];
            if (a.bias0) y[v] += bias[v];
        }
        if (a.out_elem == ELEM_BF16) store_wide<ELEM_BF16, NV>(a.out, m * a.ldo + n, count, y);
        else if (a.out_elem == ELEM_F16) store_wide<ELEM_F16, NV>(a.out, m * a.ldo + n, count, y);
        else store_wide<ELEM_F32, NV>(a.out, m * a.ldo + n, count, y);
    } else {
        if (a.bias0) {
            float b[NV];
            load_wide<E, NV>(a.bias0, n, count, b);
#pragma unroll
            for (int v = 0; v < NV; ++v) g[v] += b[v];
        }
        if (a.bias1) {
            float b[NV];
            load_wide<E, NV>(a.bias1, n, count, b);
#pragma unroll
            for (int v = 0; v < NV; ++v) u[v] += b[v];
        }
        if constexpr (EPI == DENSE_GATED) {
            float y[NV], d;
#pragma unroll
            for (int v = 0; v < NV; ++v) y[v] = activate<E>(a.act, g[v], &d) * u[v];
            if (a.drop.on) {
#pragma unroll
                for (int v = 0; v < NV; v += 4) drop4(y + v, (uint32_t)((n + v) >> 2), (uint32_t)m, a.drop);
            }
            store_wide<E, NV>(a.out, m * a.ldo + n, count, y);
        } else {
            float y[NV];
            load_wide<E, NV>(a.grad, m * a.ldg + n, count, y);
            if (a.drop.on) {
#pragma unroll
                for (int v = 0; v < NV; v += 4) drop4(y + v, (uint32_t)((n + v) >> 2), (uint32_t)m, a.drop);
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float d;
                const float h = activate<E>(a.act, g[v], &d);
                g[v] = v < count ? y[v] * u[v] * d : 0.0f;
                u[v] = v < count ? y[v] * h : 0.0f;
            }
            store_wide<E, NV>(a.out, m * a.ldo + n, count, g);
            store_wide<E, NV>(a.out1, m * a.ldo + n, count, u);
        }
    }
}

}  // namespace
}  // namespace geot
