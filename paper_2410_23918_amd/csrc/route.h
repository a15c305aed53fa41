// A token's choice of experts, by one wavefront: shared by the routing (experts.hip) and the layer of experts for a few tokens (expert_layer.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace bitstack {

// Orders like the logit; 0: not to be taken (NaN, -infinity)
__device__ __forceinline__ unsigned route_key(float l) {
    if (!(l > -INFINITY)) return 0;
    l = fminf(l, 3.402823466e38f) + 0.0f;   // -0 -> 0
    const unsigned b = __float_as_uint(l);
    return b ^ (unsigned(int(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float route_value(unsigned key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// Over a wavefront, by row operations: each adds what lies 1, 2, 4, 8 lanes before, then the rows' last lanes; 0 where nothing lies
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_before(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
template <class OP>
__device__ __forceinline__ int wave_all(int v, OP op) {
    v = op(v, from_before<0x111, 0xf>(v));   // row_shr:1
    v = op(v, from_before<0x112, 0xf>(v));
    v = op(v, from_before<0x114, 0xf>(v));
    v = op(v, from_before<0x118, 0xf>(v));
    v = op(v, from_before<0x142, 0xa>(v));   // row_bcast:15
    v = op(v, from_before<0x143, 0xc>(v));   // row_bcast:31
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
    return unsigned(wave_all(int(v), [](int a, int b) { return int(max(unsigned(a), unsigned(b))); }));
}
__device__ __forceinline__ float wave_sum(float v) {
    return __int_as_float(wave_all(__float_as_int(v), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}

// The j-th lane ends with the j-th choice (-1: none) and its key; first: the largest key.
template <int NL>
__device__ __forceinline__ void choose_experts(int top_k, const unsigned (&key)[NL], int lane, int& expert, unsigned& mine, unsigned& first) {
    unsigned left[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) left[i] = key[i];
    mine = first = 0;
    expert = -1;
    for (int j = 0; j < top_k; ++j) {
        unsigned best = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) best = max(best, left[i]);
        best = wave_max(best);
        if (best == 0) break;
        if (j == 0) first = best;
        int e = -1;   // of equal ones the lowest
#pragma unroll
        for (int i = NL - 1; i >= 0; --i) {
            const unsigned long long here = __ballot(left[i] == best);
            if (here) e = i * 64 + __builtin_ctzll(here);
        }
        if (lane == j) {
            mine = best;
            expert = e;
        }
#pragma unroll
        for (int i = 0; i < NL; ++i)
            if (i * 64 + lane == e) left[i] = 0;
    }
}
// and the j-th choice's weight
template <int NL>
__device__ __forceinline__ float choice_weight(bool renormalise, const unsigned (&key)[NL], unsigned mine, unsigned first) {
    const float most = route_value(first);
    const float share = mine ? expf(route_value(mine) - most) : 0.0f;
    float total;
    if (renormalise) {
        total = wave_sum(share);
    } else {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NL; ++i) sum += key[i] ? expf(route_value(key[i]) - most) : 0.0f;
        total = wave_sum(sum);
    }
    return mine ? share / total : 0.0f;
}
template <int NL>
__device__ __forceinline__ void choose(int top_k, bool renormalise, const unsigned (&key)[NL], int lane, int& expert, float& weight) {
    unsigned mine, first;
    choose_experts<NL>(top_k, key, lane, expert, mine, first);
    weight = choice_weight<NL>(renormalise, key, mine, first);
}
// Sums of the lanes up to each one
__device__ __forceinline__ int wave_scan(int v) {
    v += from_before<0x111, 0xf>(v);
    v += from_before<0x112, 0xf>(v);
    v += from_before<0x114, 0xf>(v);
    v += from_before<0x118, 0xf>(v);
    v += from_before<0x142, 0xa>(v);
    v += from_before<0x143, 0xc>(v);
    return v;
}

}  // namespace bitstack
