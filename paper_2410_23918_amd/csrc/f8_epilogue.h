// What follows a product: y = act(a + bias) + residual, or, where the rows of the weight are gates above values,
//     y = g / (1 + exp(-g)) u + residual,   (g, u) = the halves of a + bias,
// on the fp32 sums a, rounded once to the type of y.
#pragma once
#include <hip/hip_runtime.h>

#include "f8.h"

namespace bitstack {

// N consecutive elements as floats, at any element's address; those at or past `n` zero
template <int T, int N>
__device__ __forceinline__ void load_few(const void* from, size_t at, int n, float (&v)[N]) {
    typedef typename Elem<T>::type E;
    typedef E some __attribute__((ext_vector_type(N)));
    typedef some loose __attribute__((aligned(sizeof(E))));
    const E* const p = static_cast<const E*>(from) + at;
    if (n >= N) {
        const some u = *reinterpret_cast<const loose*>(p);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = float(u[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = e < n ? float(p[e]) : 0.0f;
    }
}
template <int N>
__device__ __forceinline__ void load_as(int dtype, const void* from, size_t at, int n, float (&v)[N]) {
    if (dtype == BITSTACK_T_F32) load_few<BITSTACK_T_F32, N>(from, at, n, v);
    else if (dtype == BITSTACK_T_F16) load_few<BITSTACK_T_F16, N>(from, at, n, v);
    else load_few<BITSTACK_T_BF16, N>(from, at, n, v);
}

// and back; those at or past `n` are not stored
template <int T, int N>
__device__ __forceinline__ void store_few(void* to, size_t at, int n, const float (&v)[N]) {
    typedef typename Elem<T>::type E;
    typedef E some __attribute__((ext_vector_type(N)));
    typedef some loose __attribute__((aligned(sizeof(E))));
    E* const p = static_cast<E*>(to) + at;
    if (n >= N) {
        some u;
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] = E(v[e]);
        *reinterpret_cast<loose*>(p) = u;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < n) p[e] = E(v[e]);
    }
}
template <int N>
__device__ __forceinline__ void store_as(int dtype, void* to, size_t at, int n, const float (&v)[N]) {
    if (dtype == BITSTACK_T_F32) store_few<BITSTACK_T_F32, N>(to, at, n, v);
    else if (dtype == BITSTACK_T_F16) store_few<BITSTACK_T_F16, N>(to, at, n, v);
    else store_few<BITSTACK_T_BF16, N>(to, at, n, v);
}

template <int N>
__device__ __forceinline__ void add_bias(const F8Params& p, int n, int at, float (&a)[N]) {   // columns n .. of y, rows at .. of the weight
    if (!p.bias) return;
    float b[N];
    load_as<N>(p.bias_dtype, p.bias, size_t(at), p.cols - n, b);
#pragma unroll
    for (int e = 0; e < N; ++e) a[e] += b[e];
}
template <int N>
__device__ __forceinline__ void add_residual(const F8Params& p, int row, int n, float (&a)[N]) {
    if (!p.residual) return;
    float r[N];
    load_as<N>(p.y_dtype, p.residual, size_t(row) * p.ld_r + n, p.cols - n, r);
#pragma unroll
    for (int e = 0; e < N; ++e) a[e] += r[e];
}

// What an activation costs in the largest tiles, where nothing hides it: 2048 tokens, 28672 x 8192, bf16, in a graph: the bare product 398 us, with a bias 409, and
// relu 411, gelu_tanh 419, silu 429, gelu 434 (by erfcf 477); with a residual, 117 MB, 447, 449, 454, 463 and 470.
// v Phi(v).  Phi(-s) = exp(-s^2 / 2) t P(t), t = 1 / (1 + 0.305 s), for s >= 0, so that no digits are lost where it is small: P of degree 7 by least relative error over
// 0 <= s <= 14: the polynomial's 1.26e-7, coefficients and 0.305 as fp32 numbers (fitted; all in fp32 14 half steps of a value, and the exponent's rounding, 2^-23 s^2 of it, where it is small).
__device__ __forceinline__ float gelu(float v) {
    const float s = fabsf(v), t = __builtin_amdgcn_rcpf(fmaf(s, 0.305f, 1.0f));
    float q = fmaf(t, 0.0366993621f, -0.15298903f);
    q = fmaf(t, q, 0.185718149f);
    q = fmaf(t, q, -0.0379779823f);
    q = fmaf(t, q, 0.121022284f);
    q = fmaf(t, q, 0.10342069f);
    q = fmaf(t, q, 0.122466847f);
    q = fmaf(t, q, 0.121639729f) * t * __builtin_amdgcn_exp2f(s * s * -0.72134752044448170368f);   // 1 / (2 ln 2)
    return v < -40.0f ? 0.0f : v * (v > 0.0f ? 1.0f - q : q);
}
// v / (1 + exp(-2 sqrt(2 / pi) (v + 0.044715 v^3))): seven instructions, the exponent's rounding, 2^-22 of it, counts where the value is small
__device__ __forceinline__ float gelu_tanh(float v) {
    constexpr float kA = -2.3022081986f, kB = -0.1029432397f;   // -2 sqrt(2 / pi) / ln 2, and times 0.044715
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * fmaf(v * v, kB, kA)));
}

template <int N>
__device__ __forceinline__ void activate(int act, float (&a)[N]) {
    auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < N; ++e) a[e] = f(a[e]);
    };
    if (act == BITSTACK_ACT_RELU) each([](float v) { return v < 0.0f ? 0.0f : v; });
    else if (act == BITSTACK_ACT_GELU) each([](float v) { return gelu(v); });
    else if (act == BITSTACK_ACT_GELU_TANH) each([](float v) { return gelu_tanh(v); });
    else if (act == BITSTACK_ACT_SILU) each([](float v) { return f8_gate(v, 1.0f); });
}

// a: sums of columns n .. n + N - 1 of a row of y (n < cols), in place
template <int N>
__device__ __forceinline__ void epilogue(const F8Params& p, int row, int n, float (&a)[N]) {
    add_bias<N>(p, n, n, a);
    activate<N>(p.act, a);
    add_residual<N>(p, row, n, a);
}
template <int N>
__device__ __forceinline__ void epilogue_gated(const F8Params& p, int row, int n, float (&a)[N], float (&u)[N]) {
    add_bias<N>(p, n, n, a);
    add_bias<N>(p, n, p.cols + n, u);
#pragma unroll
    for (int e = 0; e < N; ++e) a[e] = f8_gate(a[e], u[e]);
    add_residual<N>(p, row, n, a);
}
__device__ __forceinline__ v4f epilogue4(const F8Params& p, int row, int n, const v4f& v) {
    float a[4] = {v[0], v[1], v[2], v[3]};
    epilogue<4>(p, row, n, a);
    return v4f{a[0], a[1], a[2], a[3]};
}
__device__ __forceinline__ v4f epilogue4_gated(const F8Params& p, int row, int n, const v4f& g, const v4f& v) {
    float a[4] = {g[0], g[1], g[2], g[3]}, u[4] = {v[0], v[1], v[2], v[3]};
    epilogue_gated<4>(p, row, n, a, u);
    return v4f{a[0], a[1], a[2], a[3]};
}

}  // namespace bitstack
