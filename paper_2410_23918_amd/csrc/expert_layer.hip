// A layer of experts for a few tokens, from the router's logits to the weighted sums, in two kernels:
//
//     p[t], e[t] = the top_k choices of token t (as bitstack_route makes them)
//     (g, u) = W1[e] x[t],   h[t, j] = g / (1 + exp(-g)) u,   y[t] = sum_j p[t, j] W2[e] h[t, j]  (+ residual[t])
//
// k_layer_up routes (every workgroup for itself: a launch and a pass over memory less) and writes h; k_layer_down multiplies with W2 and sums.
//   The weights are e4m3 with a scale for each 128 x 128; the activations are not brought to 8 bits.  A few tokens are bound by the stream of the weights,
// 3 width x hidden bytes for every expert that has a token, and the matrix cores have time for operands of 16 bits: an e4m3 number is an fp16 and a
// bf16 number, x of 16 bits is taken as it is, x of 32 bits as the sum of three bf16 numbers (8 bits each, exact), h as the sum of two (16 bits, 2^-17 of a
// value) for outputs of 16 bits and of three for fp32.  Sums are fp32: a block of 128 columns starts from zero and is added times its scale.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "expert_layer.h"
#include "f8_epilogue.h"
#include "kparams.h"
#include "route.h"

namespace bitstack {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v4f multiply8(const v8h& w, const v8h& x, const v4f& c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(w, x, c, 0, 0, 0); }
__device__ __forceinline__ v4f multiply8(const v8bf& w, const v8bf& x, const v4f& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }

// Between a product and what reads its result lie eight wait states, which the hardware does not keep.  The compiler does within a block of instructions; where it had moved the
// reader past a branch there was one.  What has read the product is settled before any branch.
__device__ __forceinline__ void settle(v4f& v) { asm volatile("" : "+v"(v)); }

// eight e4m3 numbers as fp16 or bf16, exactly
__device__ __forceinline__ void widen(int lo, int hi, v8h& to) {
    const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true),
              c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    to = v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void widen(int lo, int hi, v8bf& to) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    to = v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The upper half of an fp32 number is a bf16 number; what is left over is exact (and 0 for an infinity, which the upper half holds)
__device__ __forceinline__ float upper(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ __forceinline__ float left_over(float v, float up) { return __builtin_isinf(v) ? 0.0f : v - up; }
__device__ __forceinline__ unsigned short upper16(float v) { return (unsigned short)(__float_as_uint(v) >> 16); }

// A lane's share of a block of columns: 16 from 16 kg on and 16 from 64 + 16 kg on, as four pieces of eight
__device__ __forceinline__ int piece_column(int c, int kg) { return (c >> 1) * 64 + kg * 16 + (c & 1) * 8; }

// The last pieces of a row that does not end with a block were loaded `k` elements early, so that nothing past the row is read: moves them down by k, zeros behind.
__device__ __forceinline__ void move_down(unsigned (&d)[4], int k) {   // eight elements of 16 bits
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned next = i < 3 ? d[i + 1] : 0u;
        d[i] = k & 1 ? d[i] >> 16 | next << 16 : d[i];
    }
#pragma unroll
    for (int s = 1; s <= 4; s <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = k >> 1 & s ? (i + s < 4 ? d[i + s] : 0u) : d[i];
}
__device__ __forceinline__ void move_down(float (&d)[8], int k) {
#pragma unroll
    for (int s = 1; s <= 8; s <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = k & s ? (i + s < 8 ? d[i + s] : 0.0f) : d[i];
}

// Activations as they come: 32 columns of a token
template <int T>
struct RawX {
    static constexpr int kParts = 1;
    typedef typename std::conditional<T == BITSTACK_T_F16, v8h, v8bf>::type V;
    V v[4];
    __device__ __forceinline__ void load(const typename Elem<T>::type* row, int b, int kg, int in) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            v[c] = __builtin_bit_cast(V, *reinterpret_cast<const typename Piece<T>::loose*>(row + min(b * 128 + piece_column(c, kg), in - 8)));
    }
    __device__ __forceinline__ void end(int b, int kg, int in) {
        asm volatile("" : "+v"(kg));   // nothing of this is made ahead and kept in registers
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const v4u u = __builtin_bit_cast(v4u, v[c]);
            unsigned d[4] = {u[0], u[1], u[2], u[3]};
            move_down(d, min(max(b * 128 + piece_column(c, kg) - (in - 8), 0), 8));
            v[c] = __builtin_bit_cast(V, v4u{d[0], d[1], d[2], d[3]});
        }
    }
    __device__ __forceinline__ V part(int, int c) const { return v[c]; }
};
template <>
struct RawX<BITSTACK_T_F32> {
    static constexpr int kParts = 3;   // the smallest first
    typedef v8bf V;
    v4f v[4][2];
    __device__ __forceinline__ void load(const float* row, int b, int kg, int in) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float* const from = row + min(b * 128 + piece_column(c, kg), in - 8);
            v[c][0] = *reinterpret_cast<const Piece<BITSTACK_T_F32>::loose*>(from);
            v[c][1] = *reinterpret_cast<const Piece<BITSTACK_T_F32>::loose*>(from + 4);
        }
    }
    __device__ __forceinline__ void end(int b, int kg, int in) {
        asm volatile("" : "+v"(kg));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = v[c][i >> 2][i & 3];
            move_down(d, min(max(b * 128 + piece_column(c, kg) - (in - 8), 0), 8));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i >> 2][i & 3] = d[i];
        }
    }
    __device__ __forceinline__ v8bf part(int q, int c) const {
        v4u o;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            unsigned bits[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float a = v[c][d >> 1][(d & 1) * 2 + e];
                if (q < 2) a = left_over(a, upper(a));
                if (q < 1) a = left_over(a, upper(a));
                bits[e] = __float_as_uint(a);
            }
            o[d] = bits[0] >> 16 | (bits[1] & 0xffff0000u);
        }
        return __builtin_bit_cast(v8bf, o);
    }
};

// The same kept for many products: fp32 numbers in their parts, so that they are taken apart once
template <int T>
struct KeptX {
    RawX<T> x;
    __device__ __forceinline__ void keep(const RawX<T>& from) { x = from; }
    __device__ __forceinline__ typename RawX<T>::V part(int q, int c) const { return x.part(q, c); }
};
template <>
struct KeptX<BITSTACK_T_F32> {
    v8bf p[3][4];
    __device__ __forceinline__ void keep(const RawX<BITSTACK_T_F32>& from) {
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c) p[q][c] = from.part(q, c);
    }
    __device__ __forceinline__ v8bf part(int q, int c) const { return p[q][c]; }
};

// a scale of the weight as it lies in memory
template <bool S_F32>
__device__ __forceinline__ float scale_value(int raw) {
    if constexpr (S_F32) return __int_as_float(raw);
    else return raw == 255 ? __uint_as_float(0x7fc00000u) : __builtin_amdgcn_ldexpf(1.0f, raw - 127);
}
template <bool S_F32>
__device__ __forceinline__ int load_scale(__amdgpu_buffer_rsrc_t s, unsigned at) {
    if constexpr (S_F32) return __builtin_amdgcn_raw_buffer_load_b32(s, int(at * 4u), 0, 0);
    else return __builtin_amdgcn_raw_buffer_load_b8(s, int(at), 0, 0);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* p, unsigned bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(bytes), 0x00020000);
}

// zeroes the bytes of a 16-byte piece from its column `n` on
__device__ __forceinline__ v4i cut_columns(v4i v, int n) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int k = n - 4 * d;
        v[d] &= k >= 4 ? -1 : k <= 0 ? 0 : (1 << (8 * k)) - 1;
    }
    return v;
}

// FR fragments of 16 rows of the weight, a block of columns of them
template <int FR>
struct RawW {
    v4i v[FR][2];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t w, const unsigned (&row)[FR], int b, int kg, int in) {
#pragma unroll
        for (int j = 0; j < FR; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h)   // always inside the row
                v[j][h] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(w, int(row[j] + unsigned(min(b * 128 + h * 64 + kg * 16, (in - 1) & ~15))), 0, 0));
    }
    __device__ __forceinline__ void end(int b, int kg, int in) {   // the rows may go on with anything
        asm volatile("" : "+v"(kg));   // nothing of this is made ahead and kept in registers
#pragma unroll
        for (int j = 0; j < FR; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) v[j][h] = cut_columns(v[j][h], in - (b * 128 + h * 64 + kg * 16));
    }
    template <class V>
    __device__ __forceinline__ void widened(int j, V (&to)[4]) const {
#pragma unroll
        for (int c = 0; c < 4; ++c) widen(v[j][c >> 1][(c & 1) * 2], v[j][c >> 1][(c & 1) * 2 + 1], to[c]);
    }
};

// ---- routing, by every workgroup: who goes where, in LDS
struct LayerLds {
    unsigned long long* mask;   // [experts] the tokens of an expert
    LayerExpert* list;          // [most] the experts that have any
    int* base;                  // [experts] an expert's first row
    int* count;                 // experts with tokens
    float* weight;              // [rows] by row: rows sorted by expert, then token
    unsigned char* token;       // [rows]
    float* chosen_weight;       // [rows] by (token, j)
    short* chosen;              // [rows]
};
__host__ __device__ inline unsigned layer_lds_bytes(int experts, int rows, int most) {
    return unsigned(16 + 16 * most + 12 * experts + 11 * rows + 15) & ~15u;   // a multiple of 16
}
__device__ __forceinline__ LayerLds layer_lds(unsigned char* at, int experts, int rows, int most) {
    LayerLds l;
    l.count = reinterpret_cast<int*>(at);
    at += 16;
    l.list = reinterpret_cast<LayerExpert*>(at);
    at += 16 * most;
    l.mask = reinterpret_cast<unsigned long long*>(at);
    at += 8 * experts;
    l.base = reinterpret_cast<int*>(at);
    at += 4 * experts;
    l.weight = reinterpret_cast<float*>(at);
    at += 4 * rows;
    l.chosen_weight = reinterpret_cast<float*>(at);
    at += 4 * rows;
    l.chosen = reinterpret_cast<short*>(at);
    at += 2 * rows;
    l.token = at;
    return l;
}

__device__ __forceinline__ unsigned load_key(const LayerParams& p, int token, int expert) {
    const size_t at = size_t(token) * p.ld_logits + min(expert, p.experts - 1);
    float v;
    if (p.logits_dtype == BITSTACK_T_F32) v = static_cast<const float*>(p.logits)[at];
    else if (p.logits_dtype == BITSTACK_T_F16) v = float(static_cast<const _Float16*>(p.logits)[at]);
    else v = float(static_cast<const __bf16*>(p.logits)[at]);
    return expert < p.experts ? route_key(v) : 0;
}
template <int NL>
__device__ __forceinline__ void layer_choose(const LayerParams& p, const LayerLds& l, int wave, int lane) {
    for (int t = wave; t < p.tokens; t += 8) {
        unsigned key[NL];
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            key[i] = load_key(p, t, i * 64 + lane);
        }
        int expert;
        unsigned mine, first;
        choose_experts<NL>(p.top_k, key, lane, expert, mine, first);
        float weight = 0.0f;
        if (blockIdx.x == 0) weight = choice_weight<NL>(p.renormalise != 0, key, mine, first);   // it writes them down
        if (lane < p.top_k) {
            l.chosen[t * p.top_k + lane] = short(expert);
            l.chosen_weight[t * p.top_k + lane] = weight;
            if (expert >= 0) atomicOr(reinterpret_cast<unsigned*>(&l.mask[expert]) + (t >> 5), 1u << (t & 31));   // bits: the order does not matter
        }
    }
}

// The same for up to 16 NK experts and 16 choices: sixteen lanes a token, four tokens a wavefront, NK keys a lane.  57 tokens, six of 64 experts: a wavefront a token
// takes ten microseconds, which every workgroup waits for.
template <int CTRL>
__device__ __forceinline__ unsigned rotated(unsigned v) { return unsigned(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ unsigned row_most(unsigned v) {   // over sixteen lanes
    v = max(v, rotated<0x128>(v));   // row_ror:8
    v = max(v, rotated<0x124>(v));
    v = max(v, rotated<0x122>(v));
    return max(v, rotated<0x121>(v));
}
__device__ __forceinline__ float row_sum(float v) {   // the same bits in every lane: both sides of a sum are the same
    v += __uint_as_float(rotated<0x128>(__float_as_uint(v)));
    v += __uint_as_float(rotated<0x124>(__float_as_uint(v)));
    v += __uint_as_float(rotated<0x122>(__float_as_uint(v)));
    return v + __uint_as_float(rotated<0x121>(__float_as_uint(v)));
}
template <int NK>
__device__ __forceinline__ void layer_choose_by_rows(const LayerParams& p, const LayerLds& l, int wave, int lane) {
    const int at = lane & 15;
    for (int t0 = 4 * wave; t0 < p.tokens; t0 += 32) {
        const int t = t0 + (lane >> 4);
        unsigned key[NK], left[NK];
#pragma unroll
        for (int i = 0; i < NK; ++i) key[i] = load_key(p, min(t, p.tokens - 1), i * 16 + at);
#pragma unroll
        for (int i = 0; i < NK; ++i) left[i] = key[i];
        unsigned mine = 0, first = 0;
        int expert = -1;
        for (int j = 0; j < p.top_k; ++j) {
            unsigned best = left[0];
#pragma unroll
            for (int i = 1; i < NK; ++i) best = max(best, left[i]);
            best = row_most(best);
            if (j == 0) first = best;
            unsigned e = 0;   // of equal ones the lowest, as the largest of 2^16 less it; 0: none is left
#pragma unroll
            for (int i = NK - 1; i >= 0; --i) e = left[i] == best ? 65536u - unsigned(i * 16 + at) : e;
            e = row_most(e);
            if (at == j) {
                mine = best;
                expert = best ? 65536 - int(e) : -1;
            }
#pragma unroll
            for (int i = 0; i < NK; ++i) left[i] = 65536u - unsigned(i * 16 + at) == e ? 0 : left[i];
        }
        float weight = 0.0f;
        if (blockIdx.x == 0) {   // it writes them down
            const float most = route_value(first), share = mine ? expf(route_value(mine) - most) : 0.0f;
            float all = share;
            if (!p.renormalise) {
                all = 0.0f;
#pragma unroll
                for (int i = 0; i < NK; ++i) all += key[i] ? expf(route_value(key[i]) - most) : 0.0f;
            }
            all = row_sum(all);
            weight = mine ? share / all : 0.0f;
        }
        if (at < p.top_k && t < p.tokens) {
            l.chosen[t * p.top_k + at] = short(expert);
            l.chosen_weight[t * p.top_k + at] = weight;
            if (expert >= 0) atomicOr(reinterpret_cast<unsigned*>(&l.mask[expert]) + (t >> 5), 1u << (t & 31));   // bits: the order does not matter
        }
    }
}

__device__ __forceinline__ void layer_route(const LayerParams& p, const LayerLds& l) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int e = tid; e < p.experts; e += 512) l.mask[e] = 0;
    __syncthreads();
    if (p.top_k <= 16 && p.experts <= 16) layer_choose_by_rows<1>(p, l, wave, lane);
    else if (p.top_k <= 16 && p.experts <= 64) layer_choose_by_rows<4>(p, l, wave, lane);
    else if (p.top_k <= 16 && p.experts <= 128) layer_choose_by_rows<8>(p, l, wave, lane);
    else if (p.top_k <= 16 && p.experts <= 256) layer_choose_by_rows<16>(p, l, wave, lane);
    else if (p.experts <= 256) layer_choose<4>(p, l, wave, lane);
    else layer_choose<16>(p, l, wave, lane);
    __syncthreads();
    if (wave == 0) {   // experts with tokens and their first rows, 64 at a time; both sums in one word (fewer than 2^12 rows)
        const int cap = 16 * p.fragments;
        int before = 0;
        for (int e0 = 0; e0 < p.experts; e0 += 64) {
            const int e = e0 + lane;
            unsigned long long m = e < p.experts ? l.mask[e] : 0;
            const int tokens = __popcll(m), mine = (tokens + cap - 1) / cap << 16 | tokens, sum = wave_scan(mine);
            int at = before + sum - mine;
            if (e < p.experts) l.base[e] = at & 0xffff;
            while (__popcll(m) > cap) {   // more tokens than fit a unit: the expert comes again
                unsigned long long some = 0;
                for (int i = 0; i < cap; ++i) {
                    some |= m & -m;
                    m &= m - 1;
                }
                l.list[at >> 16] = LayerExpert{e, at & 0xffff, some};
                at += 1 << 16 | cap;
            }
            if (m) l.list[at >> 16] = LayerExpert{e, at & 0xffff, m};
            before += __builtin_amdgcn_readlane(sum, 63);
        }
        if (lane == 0) *l.count = before >> 16;
    }
    __syncthreads();
    for (int i = tid; i < p.tokens * p.top_k; i += 512) {
        const int e = l.chosen[i], t = i / p.top_k;
        if (e < 0) continue;
        const int row = l.base[e] + __popcll(l.mask[e] & ((1ull << t) - 1));
        l.weight[row] = l.chosen_weight[i];
        l.token[row] = (unsigned char)t;
    }
    __syncthreads();
}

// an expert's entry, in scalar registers
struct Active {
    int expert, base, rows;
};
__device__ __forceinline__ Active active_of(const LayerExpert* list, int a) {
    const LayerExpert e = list[a];
    return {__builtin_amdgcn_readfirstlane(e.expert), __builtin_amdgcn_readfirstlane(e.base), __builtin_amdgcn_readfirstlane(__popcll(e.tokens))};
}

// ---- h.  A unit: 8 FR of an expert's gates and the values next to them (FR = 1: both in one fragment of 16 rows) for all its tokens, NF fragments of 16 at
// most; its eight wavefronts take every eighth block of columns each and meet in LDS.  A workgroup has a run of units and requests the weight DEPTH blocks ahead, over
// the ends of units.
//   KEEP > 0: a wavefront has at most KEEP blocks of columns and keeps its tokens' share of them in registers for as long as the units are the same expert's; a
// compute unit's registers hold 16 tokens of 6144 or 32 of 4096.  KEEP = 0: they are read anew for every unit, FR = 4 so that there are more rows to each load (64
// tokens through two of eight experts, 28672 x 4096: FR = 2 328 us, FR = 4 247, kept 187; 183 without the tokens' loads, timing only).
//   ODD: width is no multiple of 4, so that a lane's four rows may have two scales.
//   Bound by the stream of the weights where there is enough of it.  28672 x 4096 an expert: one token, two experts, 46 us (5.1 TB/s; 45.5 without the products,
// timing only), 64 tokens, all eight, 185 (5.1); 57 tokens, six of 64 of 2048 x 4096, 101 (5.3).  Before the stream comes the routing, 2 us for one token: one token,
// six of 64, 15.3 us (3.3).  16 tokens, two of eight of 2112 x 2001, fp32, 15.7 (2.2): some 522 units, three to a workgroup at most where the mean is two, and rows of an odd
// length; fp32 activations are three products for one, 1.3 us there, and their parts, where they are not kept, are made anew for every 32 rows.
template <int T, int FR, int NF, int DEPTH, int KEEP, bool S_F32, bool ODD>
__global__ __launch_bounds__(512, 2) void k_layer_up(LayerParams p) {
    typedef typename Elem<T>::type E;
    typedef typename RawX<T>::V V;
    static_assert(!ODD || FR == 1, "one fragment");
    static_assert(KEEP % DEPTH == 0, "a block's stage is the same in every unit");
    constexpr int kBufs = FR * NF > 4 ? 1 : 2, kRed = 8 * FR * NF * 256;   // floats
    constexpr int kAhead = KEEP ? 0 : T == BITSTACK_T_F32 ? 1 : NF < 2 ? NF : 2;   // fragments of tokens that are requested ahead (registers); others when they are multiplied
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    float* const red = reinterpret_cast<float*>(smem);
    const int tid = threadIdx.x, lane = tid & 63, ln = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rows = p.tokens * p.top_k;
    const LayerLds l = layer_lds(smem + kBufs * kRed * 4, p.experts, rows, p.most);
    layer_route(p, l);
    const int actives = __builtin_amdgcn_readfirstlane(*l.count);
    if (blockIdx.x == 0) {   // for the other kernel
        if (tid == 0) *p.count = actives;
        for (int a = tid; a < actives; a += 512) p.list[a] = l.list[a];
        for (int i = tid; i < rows; i += 512) {
            p.row_weight[i] = l.weight[i];
            p.row_token[i] = l.token[i];
        }
        for (int i = tid; i < p.tiles_down; i += 512) p.arrived[i] = 0;
    }
    const int kb = (p.hidden + 127) / 128, steps = KEEP ? KEEP : (kb + 7) / 8, tiles = (p.width + 8 * FR - 1) / (8 * FR);
    const long long units = (long long)actives * tiles;
    const int u0 = int(units * blockIdx.x / gridDim.x), u1 = int(units * (blockIdx.x + 1) / gridDim.x);
    if (u0 >= u1) return;
    const bool ragged = p.hidden % 128 != 0;
    const unsigned w_extent = unsigned(size_t(2 * p.width - 1) * p.ld_w1 + (p.hidden + 15) / 16 * 16);
    const int s_rows = (2 * p.width + 127) / 128;

    // where the loads are
    struct Place {
        Active a;
        int ai, tile, step;
    };
    Place at = {active_of(l.list, u0 / tiles), u0 / tiles, u0 % tiles, 0};
    int left = u1 - u0;
    unsigned w_row[FR], s_row[FR], s_row2 = 0;
    const unsigned char* w_base;
    const unsigned char* s_base;
    const E* x_row[kAhead + 1];   // of the loads
    const E* x_late[NF];          // of the products
    auto token_row = [&](const Active& a, int f) {   // of the f-th fragment's token ln
        const int r = a.base + min(16 * f + ln, a.rows - 1);
        return static_cast<const E*>(p.x) + size_t(l.token[r]) * p.ld_x;
    };
    auto enter = [&]() __attribute__((always_inline)) {
        const int n0 = at.tile * 8 * FR;
        w_base = p.w1 + size_t(at.a.expert) * (2 * p.width) * p.ld_w1;
        s_base = p.s1 + size_t(at.a.expert) * s_rows * kb * (S_F32 ? 4 : 1);
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            // the weight's row that this lane loads, and the first of the four whose sums it gets
            const int n = FR == 1 ? n0 + (ln & 7) : n0 + 16 * (j >> 1) + ln, m = FR == 1 ? n0 + 4 * (kg & 1) : n0 + 16 * (j >> 1) + 4 * kg;
            const bool value = FR == 1 ? ln >= 8 : j & 1, value_sum = FR == 1 ? kg >= 2 : j & 1;
            w_row[j] = unsigned((value ? p.width : 0) + min(n, p.width - 1)) * unsigned(p.ld_w1);
            const int first = (value_sum ? p.width : 0) + min(m, p.width - 1);
            s_row[j] = unsigned(first >> 7) * unsigned(kb);
            if constexpr (ODD) s_row2 = unsigned(min(first + 3, 2 * p.width - 1) >> 7) * unsigned(kb);
        }
    };
    struct Stage {
        RawW<FR> w;
        RawX<T> x[kAhead + 1];
        int s[FR], s2;
    };
    Stage st[DEPTH];
    auto load = [&](Stage& s) __attribute__((always_inline)) {
        const int b = min(wave + 8 * at.step, kb - 1);
        const bool live = left > 0 && wave + 8 * at.step < kb;   // past the last block nothing is read and zeros arrive
        s.w.load(buffer_of(w_base, live ? w_extent : 0), w_row, b, kg, p.hidden);
#pragma unroll
        for (int f = 0; f < kAhead; ++f) s.x[f].load(x_row[f], b, kg, p.hidden);
        const __amdgpu_buffer_rsrc_t sr = buffer_of(s_base, live ? unsigned(s_rows) * unsigned(kb) * (S_F32 ? 4u : 1u) : 0);
#pragma unroll
        for (int j = 0; j < FR; ++j) s.s[j] = load_scale<S_F32>(sr, s_row[j] + unsigned(b));
        if constexpr (ODD) s.s2 = load_scale<S_F32>(sr, s_row2 + unsigned(b));
        if (++at.step == steps) {
            at.step = 0;
            if (--left > 0) {
                if (++at.tile == tiles) {
                    at.tile = 0;
                    at.a = active_of(l.list, ++at.ai);
#pragma unroll
                    for (int f = 0; f < kAhead; ++f) x_row[f] = token_row(at.a, f);
                }
                enter();
            }
        }
    };
#pragma unroll
    for (int f = 0; f < kAhead; ++f) x_row[f] = token_row(at.a, f);
    Place now = at;   // where the products are
    int nf;           // their fragments of tokens
    auto enter_late = [&]() __attribute__((always_inline)) {
        nf = (now.a.rows + 15) / 16;
        if constexpr (KEEP == 0) {
#pragma unroll
            for (int f = kAhead; f < NF; ++f) x_late[f] = token_row(now.a, f);
        }
    };
    enter_late();
    enter();
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(st[d]);
    v4f acc[FR][NF];
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < FR; ++j)
#pragma unroll
            for (int f = 0; f < NF; ++f) acc[j][f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    };
    clear();
    KeptX<T> kept[KEEP + 1][NF];
    auto keep = [&]() __attribute__((always_inline)) {   // the tokens of the unit that comes
        const E* row[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) row[f] = token_row(now.a, f);
        int kg_here = kg;
        asm volatile("" : "+v"(kg_here));   // nothing of this is made ahead and kept in registers
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            const int b = min(wave + 8 * k, kb - 1);
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                RawX<T> x;
                x.load(row[f], b, kg_here, p.hidden);
                if (ragged && b == kb - 1) x.end(b, kg_here, p.hidden);
                kept[k][f].keep(x);
                if constexpr (T == BITSTACK_T_F32) __builtin_amdgcn_sched_barrier(0);   // registers
            }
        }
    };
    auto products = [&](Stage& s, const KeptX<T> (&own)[NF]) __attribute__((always_inline)) {
        const int b = wave + 8 * now.step;
        if (b >= kb) return;
        const bool end = ragged && b == kb - 1;
        if (end) {
            s.w.end(b, kg, p.hidden);
#pragma unroll
            for (int f = 0; f < kAhead; ++f) s.x[f].end(b, kg, p.hidden);
        }
        float scale[FR][4];
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            const float first = scale_value<S_F32>(s.s[j]);
#pragma unroll
            for (int v = 0; v < 4; ++v) scale[j][v] = first;
            if constexpr (ODD) {
                const int row = (kg >= 2 ? p.width : 0) + min(now.tile * 8 + 4 * (kg & 1), p.width - 1);
#pragma unroll
                for (int v = 1; v < 4; ++v)
                    if ((row + v) >> 7 != row >> 7) scale[j][v] = scale_value<S_F32>(s.s2);
            }
        }
        // The products of one fragment of rows and one of tokens
        auto multiply = [&](const V (&w)[4], int j, const auto& x, int f) __attribute__((always_inline)) {
            v4f part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int q = 0; q < RawX<T>::kParts; ++q)
#pragma unroll
                for (int c = 0; c < 4; ++c) part = multiply8(w[c], x.part(q, c), part);
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[j][f][v] = fmaf(part[v], scale[j][v], acc[j][f][v]);
            if constexpr (NF > 1) settle(acc[j][f]);
        };
        if constexpr (KEEP > 0) {   // a fragment of rows at a time: registers
#pragma unroll
            for (int j = 0; j < FR; ++j) {
                V w[4];
                s.w.widened(j, w);
#pragma unroll
                for (int f = 0; f < NF; ++f)
                    if (f < nf) multiply(w, j, own[f], f);
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
        V w[FR][4];
#pragma unroll
        for (int j = 0; j < FR; ++j) s.w.widened(j, w[j]);
        auto multiply_rows = [&](const RawX<T>& x, int f) __attribute__((always_inline)) {
            if constexpr (RawX<T>::kParts > 1) {   // taken apart once for all rows
                KeptX<T> parts;
                parts.keep(x);
#pragma unroll
                for (int j = 0; j < FR; ++j) multiply(w[j], j, parts, f);
            } else {
#pragma unroll
                for (int j = 0; j < FR; ++j) multiply(w[j], j, x, f);
            }
        };
#pragma unroll
        for (int f = 0; f < kAhead; ++f)
            if (f < nf) multiply_rows(s.x[f], f);
#pragma unroll
        for (int f = kAhead; f < NF; ++f) {
            if (f < nf) {
                RawX<T> x;
                x.load(x_late[f], b, kg, p.hidden);
                if (end) x.end(b, kg, p.hidden);
                multiply_rows(x, f);
            }
        }
    };
    int buf = 0;
    auto finish = [&]() __attribute__((always_inline)) {   // a unit's sums
        float* const r = red + buf * kRed;
#pragma unroll
        for (int j = 0; j < FR; ++j)
#pragma unroll
            for (int f = 0; f < NF; ++f)
                if (f < nf) *reinterpret_cast<v4f*>(r + ((wave * FR + j) * NF + f) * 256 + lane * 4) = acc[j][f];
        lds_barrier();
        constexpr int kEach = FR == 1 ? 128 : FR / 2 * 256;   // outputs of a fragment of tokens
        const int padded = (p.width + 7) & ~7, n0 = now.tile * 8 * FR;
        for (int o = tid; o < kEach * nf; o += 512) {
            const int f = o / kEach, k = o % kEach, jj = FR == 1 ? 0 : k / 256, kk = FR == 1 ? k : k % 256;
            const int rank = 16 * f + (kk >> 2 & 15), n = n0 + 16 * jj + 4 * (kk >> 6) + (kk & 3);
            const float* const g = r + (2 * jj * NF + f) * 256 + kk;
            const float* const u = FR == 1 ? g + 128 : g + NF * 256;
            float gate = g[0], value = u[0];
#pragma unroll
            for (int w = 1; w < 8; ++w) {
                gate += g[w * FR * NF * 256];
                value += u[w * FR * NF * 256];
            }
            if (rank >= now.a.rows || n >= padded) continue;
            const float h = n < p.width ? f8_gate(gate, value) : 0.0f;
            // where k_layer_down's lanes load it: see there
            const int column = n & 127, piece = (column >> 6) * 2 + (column >> 3 & 1), lane_of = (column >> 4 & 3) * 16 + rank - 16 * f, parts = p.h_parts;
            const int kb_down = (p.width + 127) / 128, per_part = p.pack ? 128 : 2048;
            unsigned short* const to = p.h + (p.pack ? (size_t(n >> 7) * rows + now.a.base + rank) * (parts * 128) + column
                                                     : ((size_t(now.ai) * NF + f) * kb_down + (n >> 7)) * (parts * 2048) + piece * 512 + lane_of * 8 + (column & 7));
            const float rest = left_over(h, upper(h));
            to[(parts - 1) * per_part] = upper16(h);   // the largest last
            if (parts == 2) {
                to[0] = __builtin_bit_cast(unsigned short, __bf16(rest));
            } else {
                to[per_part] = upper16(rest);
                to[0] = upper16(left_over(rest, upper(rest)));
            }
        }
        if (kBufs == 2) buf ^= 1;
        else lds_barrier();
        clear();
    };
    auto next_expert = [&]() __attribute__((always_inline)) {
        now.tile = 0;
        now.a = active_of(l.list, ++now.ai);
        enter_late();
    };
    if constexpr (KEEP > 0) {
        for (int u = u0; u < u1;) {
            keep();
            for (const int end = min(u1, u + tiles - now.tile); u < end; ++u, ++now.tile) {
#pragma unroll
                for (int k = 0; k < KEEP; ++k) {
                    __builtin_amdgcn_sched_barrier(0);   // a block's products at a time: registers
                    products(st[k % DEPTH], kept[k]);
                    __builtin_amdgcn_sched_barrier(0);
                    load(st[k % DEPTH]);
                    ++now.step;
                }
                finish();
                now.step = 0;
            }
            if (u < u1) next_expert();
        }
    } else {
        const int total = (u1 - u0) * steps;
        for (int i = 0; i < total; i += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (i + d < total) {   // (the loads are in no branch: the compiler would wait for all of them where its ways meet)
                    products(st[d], kept[0]);
                    if (++now.step == steps) {
                        finish();
                        now.step = 0;
                        if (++now.tile == tiles && i + d + 1 < total) next_expert();
                    }
                }
                load(st[d]);
            }
        }
    }
}

// ---- y.  A workgroup has 16 FR rows of W2 and a part of the (expert, block of columns) pairs; its eight wavefronts take every eighth of these each.  At an
// expert's end a wavefront adds its sums, times the tokens' weights, to its own tokens' sums in LDS; these meet there, and the parts in memory, where
// the last workgroup to arrive adds them up: in order, so that the result does not depend on what arrives when.
//   PACK: so few tokens that the parts of h are columns of one fragment, 16 / PARTS of them each, and are added up at an expert's end.
//   What it takes without its main loop is 3.0 us for one token and 5.8 for 64: the lists, eight wavefronts' sums, the parts in memory.  4096 x 14336 an expert: one token, two
// experts, 31 us (3.8 TB/s); 64 tokens, all eight, 122 (3.9), where h, 16 KB to each 8 KB of the weight, comes from L2 for every tile.  57 tokens, six of 64 of 4096 x
// 1024, 54 (5.0); one token, six of them, 11.9 (2.1).
template <int FR, int NF, int PARTS, bool PACK, int DEPTH, bool S_F32>
__global__ __launch_bounds__(512, 2) void k_layer_down(LayerParams p) {
    static_assert(!PACK || NF == 1, "one fragment");
    constexpr int kLoads = PACK ? 1 : PARTS, kPack = PACK ? 16 / PARTS : 16;   // tokens of a fragment
    // One fragment of h is requested with the weight.  Of several the first kNext are requested after the products before (they come from L2), the others when they are
    // multiplied: registers
    constexpr int kNext = NF == 1 ? 0 : PARTS > 2 ? 1 : 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, ln = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rows = p.tokens * p.top_k;
    constexpr int kN = 16 * FR, kLd = kN + 4;   // floats from token to token
    float* const sums = reinterpret_cast<float*>(smem) + wave * p.tokens * kLd;
    unsigned char* at = smem + 8 * p.tokens * kLd * 4;
    LayerExpert* const list = reinterpret_cast<LayerExpert*>(at);
    at += 16 * p.most;
    float* const row_weight = reinterpret_cast<float*>(at);
    at += 4 * rows;
    int& last_here = *reinterpret_cast<int*>(at);
    unsigned char* const row_token = at + 16;
    const int actives = __builtin_amdgcn_readfirstlane(*p.count);
    for (int a = tid; a < p.most; a += 512) list[a] = p.list[a];   // those past the last one may be anything
    for (int i = tid; i < rows; i += 512) {
        row_weight[i] = p.row_weight[i];
        row_token[i] = p.row_token[i];
    }
    for (int i = lane; i < p.tokens * (kLd / 4); i += 64) reinterpret_cast<v4f*>(sums)[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();
    const int tile = blockIdx.x / p.splits, split = blockIdx.x % p.splits, n0 = tile * kN;
    const int kb = (p.width + 127) / 128;
    const int i0 = int((long long)actives * kb * split / p.splits), i1 = int((long long)actives * kb * (split + 1) / p.splits);
    const int mine = i1 - i0 > wave ? (i1 - i0 - wave + 7) / 8 : 0;   // pairs of this wavefront
    if (mine > 0) {
        const bool ragged = p.width % 128 != 0;
        const int padded = (p.width + 7) & ~7, s_rows = (p.hidden + 127) / 128;
        const int w_rows = min(kN, p.hidden - n0);
        const unsigned w_extent = unsigned((w_rows - 1) * p.ld_w2 + (p.width + 15) / 16 * 16);
        unsigned w_row[FR];
#pragma unroll
        for (int j = 0; j < FR; ++j) w_row[j] = unsigned(min(16 * j + ln, w_rows - 1)) * unsigned(p.ld_w2);
        const __amdgpu_buffer_rsrc_t hr = buffer_of(p.h, p.h_bytes);
        struct Place {
            Active a;
            int ai, b;
        };
        auto place = [&](int i) { return Place{active_of(list, i / kb), i / kb, i % kb}; };
        Place from = place(i0 + wave);
        int left = mine;
        // h lies as the lanes load it, 1024 bytes in a row to an instruction (a lane's 16 bytes of a row of its own would be a lookup of its own in L1, of which
        // there is one a clock): [entry of the list][fragment of tokens][block][part, the smallest first][piece][lane][8].  Few tokens, which would leave most of that
        // empty: [block][row][part][128].
        auto h_lane = [&](const Active& a, int f) {   // a lane's place, in elements; no token: nothing is read
            const int r = PACK ? ln % kPack : 16 * f + ln;
            const bool there = r < a.rows && (!PACK || ln < PARTS * kPack);
            return !there ? 0x40000000u : PACK ? unsigned((a.base + r) * PARTS + ln / kPack) * 128u + unsigned(kg) * 16u : unsigned(lane) * 8u;
        };
        constexpr unsigned kFragment = unsigned(PARTS) * 2048;
        auto h_at = [&](int ai, int f) { return PACK ? 0u : unsigned((ai * NF + f) * kb) * kFragment; };
        const unsigned h_block = PACK ? unsigned(rows) * (PARTS * 128) : kFragment;
        const unsigned char* w_base;
        const unsigned char* s_base;
        unsigned h_from;
        auto enter = [&]() __attribute__((always_inline)) {
            w_base = p.w2 + (size_t(from.a.expert) * p.hidden + n0) * p.ld_w2;
            s_base = p.s2 + (size_t(from.a.expert) * s_rows + n0 / 128) * kb * (S_F32 ? 4 : 1);
            h_from = h_lane(from.a, 0);
        };
        enter();
        struct H {
            v8bf v[kLoads][4];   // the smallest first
        };
        auto load_h = [&](H& h, unsigned lane_at, unsigned fragment, int b, bool live) __attribute__((always_inline)) {
            const unsigned from = fragment + unsigned(b) * h_block;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const unsigned none = live && b * 128 + piece_column(c, kg) < padded ? 0u : 0x80000000u;   // zeros arrive
#pragma unroll
                for (int q = 0; q < kLoads; ++q)
                    h.v[q][c] = __builtin_bit_cast(v8bf, __builtin_amdgcn_raw_buffer_load_b128(hr, int((lane_at * 2u) | none), int((from + unsigned(PACK ? piece_column(c, 0) : (q * 4 + c) * 512)) * 2u), 0));
            }
        };
        struct Stage {
            RawW<FR> w;
            H h;   // NF = 1
            int s;
        };
        Stage st[DEPTH];
        auto load = [&](Stage& s) __attribute__((always_inline)) {
            const bool live = left > 0;
            s.w.load(buffer_of(w_base, live ? w_extent : 0), w_row, from.b, kg, p.width);
            if constexpr (NF == 1) load_h(s.h, h_from, h_at(from.ai, 0), from.b, live);
            s.s = load_scale<S_F32>(buffer_of(s_base, live ? unsigned(kb) * (S_F32 ? 4u : 1u) : 0), unsigned(from.b));
            if (--left > 0) {
                from.b += 8;
                if (from.b >= kb) {
                    do {
                        from.b -= kb;
                        ++from.ai;
                    } while (from.b >= kb);
                    from.a = active_of(list, from.ai);
                    enter();
                }
            }
        };
        Place now = from;
        int nf = (now.a.rows + 15) / 16;
        v4f acc[FR][NF];
        auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < FR; ++j)
#pragma unroll
                for (int f = 0; f < NF; ++f) acc[j][f] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        };
        clear();
        H next[kNext + 1];
        auto load_next = [&](bool live) __attribute__((always_inline)) {
#pragma unroll
            for (int f = 0; f < kNext; ++f) load_h(next[f], h_lane(now.a, f), h_at(now.ai, f), now.b, live);
        };
        auto products = [&](Stage& s) __attribute__((always_inline)) {
            if (ragged && now.b == kb - 1) s.w.end(now.b, kg, p.width);
            const float scale = scale_value<S_F32>(s.s);
            auto add = [&](const v4f& part, int j, int f) __attribute__((always_inline)) {
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[j][f][v] = fmaf(part[v], scale, acc[j][f][v]);
                if constexpr (NF > 1) settle(acc[j][f]);
            };
            constexpr v4f kNone = {0.0f, 0.0f, 0.0f, 0.0f};
            if constexpr (NF == 1) {
                v8bf w[FR][4];
                v4f part[FR];
#pragma unroll
                for (int j = 0; j < FR; ++j) {
                    s.w.widened(j, w[j]);
                    part[j] = kNone;
                }
#pragma unroll
                for (int q = 0; q < kLoads; ++q)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int j = 0; j < FR; ++j) part[j] = multiply8(w[j][c], s.h.v[q][c], part[j]);
#pragma unroll
                for (int j = 0; j < FR; ++j) add(part[j], j, 0);
            } else if constexpr (kNext == NF) {
                static_assert(NF == 2, "two fragments");
                const bool two = nf == 2;
#pragma unroll
                for (int j = 0; j < FR; ++j) {   // a fragment of rows at a time: registers
                    v8bf w[4];
                    s.w.widened(j, w);
                    v4f part[2] = {kNone, kNone};
                    if (two) {
#pragma unroll
                        for (int q = 0; q < kLoads; ++q)
#pragma unroll
                            for (int c = 0; c < 4; ++c)
#pragma unroll
                                for (int f = 0; f < 2; ++f) part[f] = multiply8(w[c], next[f].v[q][c], part[f]);
                        add(part[0], j, 0);
                        add(part[1], j, 1);
                    } else {
#pragma unroll
                        for (int q = 0; q < kLoads; ++q)
#pragma unroll
                            for (int c = 0; c < 4; ++c) part[0] = multiply8(w[c], next[0].v[q][c], part[0]);
                        add(part[0], j, 0);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    if (f >= nf) break;
                    auto multiply = [&](const H& h) __attribute__((always_inline)) {
#pragma unroll
                        for (int j = 0; j < FR; ++j) {
                            v8bf w[4];
                            s.w.widened(j, w);
                            v4f part = kNone;
#pragma unroll
                            for (int q = 0; q < kLoads; ++q)
#pragma unroll
                                for (int c = 0; c < 4; ++c) part = multiply8(w[c], h.v[q][c], part);
                            add(part, j, f);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    };
                    if (f < kNext) {
                        multiply(next[f]);
                    } else {
                        H h;
                        load_h(h, h_lane(now.a, f), h_at(now.ai, f), now.b, true);
                        multiply(h);
                    }
                }
            }
        };
        auto finish = [&]() __attribute__((always_inline)) {   // an expert's sums
            if constexpr (PACK) {
#pragma unroll
                for (int j = 0; j < FR; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float v = acc[j][0][k];   // the smallest part's lane has the sum of all
#pragma unroll
                        for (int q = 1; q < PARTS; ++q) v += __shfl(acc[j][0][k], lane + q * kPack & 63);
                        acc[j][0][k] = v;
                    }
            }
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                if (16 * f + ln < now.a.rows) {
                    const int r = now.a.base + 16 * f + ln;
                    const float weight = row_weight[r];
                    float* const to = sums + row_token[r] * kLd + 4 * kg;
#pragma unroll
                    for (int j = 0; j < FR; ++j) {
                        v4f v = *reinterpret_cast<v4f*>(to + 16 * j);
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = fmaf(weight, acc[j][f][k], v[k]);
                        *reinterpret_cast<v4f*>(to + 16 * j) = v;
                    }
                }
            }
            clear();
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            load(st[d]);
            if (d == 0) load_next(true);
        }
        for (int i = 0; i < mine; i += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (i + d < mine) {   // (the loads are in no branch: the compiler would wait for all of them where its ways meet)
                    products(st[d]);
                    now.b += 8;
                    const bool more = i + d + 1 < mine;
                    if (now.b >= kb || !more) finish();
                    if (now.b >= kb && more) {
                        do {
                            now.b -= kb;
                            ++now.ai;
                        } while (now.b >= kb);
                        now.a = active_of(list, now.ai);
                        nf = (now.a.rows + 15) / 16;
                    }
                }
                if constexpr (NF > 1) load_next(i + d + 1 < mine);   // before the weight: loads are waited for in their order
                load(st[d]);
            }
        }
    }
    __syncthreads();
    const v4f* const all = reinterpret_cast<const v4f*>(smem);
    auto own = [&](int t, int n) {   // the eight wavefronts' sums of four columns
        v4f v = all[t * (kLd / 4) + n];
#pragma unroll
        for (int w = 1; w < 8; ++w) v += all[(w * p.tokens + t) * (kLd / 4) + n];
        return v;
    };
    const int outputs = p.tokens * (kN / 4);   // four each
    const __amdgpu_buffer_rsrc_t parts = buffer_of(p.part + size_t(tile) * p.splits * outputs * 4, unsigned(p.splits) * unsigned(outputs) * 16u);
    constexpr int kAgentScope = 16;
    if (p.splits > 1) {
        // Write-through stores, complete before the counter says so, and loads that pass the caches which other XCDs' stores do not reach: no cache is written
        // back or emptied as a whole.
        for (int o = tid; o < outputs; o += 512)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, own(o / (kN / 4), o % (kN / 4))), parts, int(unsigned(split * outputs + o) * 16u), 0, kAgentScope);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) last_here = __hip_atomic_fetch_add(&p.arrived[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == unsigned(p.splits - 1);
        __syncthreads();
        if (!last_here) return;
    }
    for (int o = tid; o < outputs; o += 512) {
        const int t = o / (kN / 4), n = n0 + o % (kN / 4) * 4;
        if (n >= p.hidden) continue;
        v4f v;
        if (p.splits > 1) {
            v = v4f{0.0f, 0.0f, 0.0f, 0.0f};
            for (int s = 0; s < p.splits; s += 4) {   // past the last one zeros arrive
                v4f few[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) few[k] = __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(parts, int(unsigned((s + k) * outputs + o) * 16u), 0, kAgentScope));
#pragma unroll
                for (int k = 0; k < 4; ++k) v += few[k];
            }
        } else {
            v = own(t, o % (kN / 4));
        }
        float a[4] = {v[0], v[1], v[2], v[3]};
        const int n_left = p.hidden - n;
        if (p.residual) {
            float r[4];
            load_as<4>(p.dtype, p.residual, size_t(t) * p.ld_r + n, n_left, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] += r[e];
        }
        store_as<4>(p.dtype, p.y, size_t(t) * p.ld_y + n, n_left, a);
    }
}

constexpr int kLayerGroups = 256;   // workgroups of k_layer_up: one on each compute unit

template <class K>
static hipError_t go(K kernel, std::atomic<int>& allowed, unsigned grid, unsigned lds, const LayerParams& p, hipStream_t st) {
    if (int(lds) > allowed && lds > 65536) {   // (doing it twice is harmless)
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, 163840);
        if (e != hipSuccess) return e;
        allowed = 163840;
    }
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(512), lds, st, p);
    return hipGetLastError();
}

template <int T, int FR, int NF, int DEPTH, int KEEP, bool S_F32, bool ODD = false>
static hipError_t up_as(const LayerParams& p, hipStream_t st) {
    static std::atomic<int> allowed{0};
    constexpr unsigned kRed = (FR * NF > 4 ? 1 : 2) * 8 * FR * NF * 1024;
    return go(&k_layer_up<T, FR, NF, DEPTH, KEEP, S_F32, ODD>, allowed, kLayerGroups, kRed + layer_lds_bytes(p.experts, p.tokens * p.top_k, p.most), p, st);
}
template <int T, bool S_F32>
static hipError_t up(const LayerParams& p, hipStream_t st) {
    constexpr bool kF32 = T == BITSTACK_T_F32;
    const int steps = ((p.hidden + 127) / 128 + 7) / 8;   // blocks of columns of a wavefront
    if (p.width % 4 != 0) return p.fragments == 1 ? up_as<T, 1, 1, kF32 ? 2 : 4, 0, S_F32, true>(p, st) : up_as<T, 1, 2, 2, 0, S_F32, true>(p, st);
    if constexpr (kF32) {
        if (p.fragments == 1) return steps <= 2 ? up_as<T, 2, 1, 2, 2, S_F32>(p, st) : up_as<T, 4, 1, 2, 0, S_F32>(p, st);
        return up_as<T, 4, 2, 1, 0, S_F32>(p, st);
    } else {
        if (p.fragments == 1 && steps > 2 && steps <= 4 && p.up_few) return up_as<T, 1, 1, 4, 4, S_F32>(p, st);
        if (p.fragments == 1) return steps <= 2 ? up_as<T, 4, 1, 2, 2, S_F32>(p, st) : steps <= 4 ? up_as<T, 2, 1, 4, 4, S_F32>(p, st) : steps <= 6 ? up_as<T, 2, 1, 2, 6, S_F32>(p, st) : up_as<T, 4, 1, 3, 0, S_F32>(p, st);
        return steps <= 2 ? up_as<T, 4, 2, 2, 2, S_F32>(p, st) : steps <= 4 ? up_as<T, 2, 2, 2, 4, S_F32>(p, st) : up_as<T, 4, 2, 2, 0, S_F32>(p, st);
    }
}
static unsigned down_lds_bytes(int rows, int tokens, int top_k, int most) { return unsigned(8 * tokens * (rows + 4) * 4 + 16 * most + 5 * tokens * top_k + 16); }
template <int FR, int NF, int PARTS, bool PACK, int DEPTH, bool S_F32>
static hipError_t down_as(const LayerParams& p, hipStream_t st) {
    static std::atomic<int> allowed{0};
    return go(&k_layer_down<FR, NF, PARTS, PACK, DEPTH, S_F32>, allowed, unsigned(p.tiles_down * p.splits), down_lds_bytes(16 * FR, p.tokens, p.top_k, p.most), p, st);
}
template <int PARTS, bool S_F32>
static hipError_t down(const LayerParams& p, hipStream_t st) {
    constexpr int kMore = PARTS == 2 ? 2 : 1;
    if (p.down_rows == 32) return p.fragments == 1 ? down_as<2, 1, PARTS, false, 2, S_F32>(p, st) : down_as<2, 2, PARTS, false, 2, S_F32>(p, st);
    if (p.pack) return down_as<4, 1, PARTS, true, 3, S_F32>(p, st);
    if (p.fragments == 1) return down_as<4, 1, PARTS, false, kMore, S_F32>(p, st);
    return down_as<4, 2, PARTS, false, kMore, S_F32>(p, st);
}

LayerPlan layer_plan(int tokens, int hidden, int width, int experts, int top_k, bool f32) {
    LayerPlan plan;
    const int rows = tokens * top_k;
    const double each = double(rows) / experts;   // tokens of an expert, in the mean
    // Entries of 16 tokens, each of which takes the expert's weights anew, or of 32, which take twice the registers.  Eight experts of 4096 x 2048, two chosen, bf16: 32 tokens, 8 to an
    // expert in the mean, 53.1 us and 56.4, 48 tokens 57.3 and 59.3, 64 tokens 68.5 and 61.0; fp32, 64 tokens 76.7 and 100.  In nine layers the other choice was faster by 8 % at
    // most (profiles/expert_layer_choices.txt).
    plan.fragments = tokens <= 16 || each <= (f32 ? 16 : 8) ? 1 : 2;
    const int cap = 16 * plan.fragments;
    plan.most = std::min(experts, rows) + (tokens > cap ? rows / cap : 0);
    const double actives = experts * (1.0 - std::pow(1.0 - double(top_k) / experts, tokens));
    // Rounds of units, the last one in part empty: units of half as many rows where they fill theirs better.  One token, six experts of 2048 x 4096, 1.5 rounds or 3:
    // the layer 30.5 us and 28.7; eight tokens, eight of 28672 x 4096, 28 or 56: 197.6 and 202.4.  With hidden sizes of 2304 to 4096 (no other form looks at it) the other choice was
    // faster by 6 % at most (profiles/expert_layer_choices.txt).
    const auto filled = [&](int n) {
        const double rounds = actives * ((width + n - 1) / n) / kLayerGroups;
        return rounds / std::ceil(rounds);
    };
    plan.up_few = filled(8) > 1.1 * filled(16);
    plan.down_rows = 64;
    if (down_lds_bytes(plan.down_rows, tokens, top_k, plan.most) > 163840) plan.down_rows = 32;   // 64 tokens with many choices of many experts
    plan.pack = tokens <= 16 / (f32 ? 3 : 2) && plan.down_rows == 64;
    plan.tiles_down = (hidden + plan.down_rows - 1) / plan.down_rows;
    // Parts of the columns: a workgroup of each compute unit takes a part of 2.5 us and the bytes at 25 a nanosecond (more than an equal share of what the memory gives).  In 14 layers
    // the fastest number was faster by 5 % at most (the same table).
    plan.splits = 1;
    double best = 1e30;
    const double tile_us = actives * plan.down_rows * width / 25e3;
    for (int s = 1; s <= 16; ++s) {
        const double rounds = std::ceil(double(plan.tiles_down) * s / 256), us = rounds * (2.5 + tile_us / s) + (s > 1 ? 1.0 + 0.1 * s : 0.0);
        if (us < best) {
            best = us;
            plan.splits = s;
        }
    }
    return plan;
}

hipError_t launch_expert_layer(const LayerParams& p, hipStream_t st) {
    hipError_t e;
    if (p.dtype == BITSTACK_T_F16) e = p.s1_f32 ? up<BITSTACK_T_F16, true>(p, st) : up<BITSTACK_T_F16, false>(p, st);
    else if (p.dtype == BITSTACK_T_BF16) e = p.s1_f32 ? up<BITSTACK_T_BF16, true>(p, st) : up<BITSTACK_T_BF16, false>(p, st);
    else e = p.s1_f32 ? up<BITSTACK_T_F32, true>(p, st) : up<BITSTACK_T_F32, false>(p, st);
    if (e != hipSuccess) return e;
    if (p.h_parts == 2) return p.s2_f32 ? down<2, true>(p, st) : down<2, false>(p, st);
    return p.s2_f32 ? down<3, true>(p, st) : down<3, false>(p, st);
}

}  // namespace bitstack
