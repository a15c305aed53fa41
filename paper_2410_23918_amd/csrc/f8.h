// Shared by the 8-bit kernels (f8_rows.hip, f8_product.h), the routing (experts.hip), the layer of experts (expert_layer.hip) and their host code (f8_host.cpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/bitstack_f8.h"
#include "rebuild.h"

namespace bitstack {

constexpr int kF8Block = 128;      // columns (and weight rows) that share a scale
constexpr float kF8Max = 448.0f;   // largest e4m3 value
constexpr int kMaxExperts = 1024, kMaxTopK = 32;

// one piece of a product: rows [row0, row0 + rows) of y with expert's weight; expert < 0: rows of zeros; rows 0: nothing
struct F8Tile {
    int expert, row0, rows, all;   // all: tiles that have rows, in every one
};

struct F8Params {
    const unsigned char* x;    // [x_rows][kp], e4m3, zero past `in`; or (x_dtype) as it came, rows x_ld bytes apart
    const unsigned char* xs;   // [ks / 4][x_rows][4] biased exponents
    const unsigned char* w;    // [experts][out] rows of e4m3, ldw bytes apart
    const void* ws;            // [experts][ceil(out / 128)][kb]
    void* y;
    const int* index;          // [rows] or null
    const F8Tile* tiles;       // null: one group
    size_t ldw, ldy;
    int out, in, kb, kp, ks;   // kb: blocks of columns, kp = 128 kb, ks = kb rounded up to 4
    int x_rows, rows;          // rows of x, of y
    int x_dtype;               // BITSTACK_T_F8, or the type of what is to be brought to 8 bits on the way
    unsigned x_bytes, x_ld;    // extent of x
    float* part;               // partial sums of the column slices
    int slices, slice_blocks;  // of the columns; blocks in one
    int n_tiles;               // tiles of rows (an upper bound where they are grouped)
    int y_dtype, ws_f32;       // ws_f32: fp32 scales
    // what follows the product, where anything does (epi)
    int epi, act;              // F8Epi, BITSTACK_ACT_*
    int cols;                  // of y: out, or half of it
    int bias_dtype, parts_only;   // parts_only: no tile is finished by itself
    const void* bias;          // [out] or null
    const void* residual;      // [rows][cols] of y_dtype, or null
    size_t ld_r;
};
enum F8Epi { kEpiNone, kEpiPlain, kEpiGated };

// float of an element, and back
template <int T>
struct Elem;
template <>
struct Elem<BITSTACK_T_F16> {
    typedef _Float16 type;
    static constexpr int kPer16 = 8;
};
template <>
struct Elem<BITSTACK_T_BF16> {
    typedef __bf16 type;
    static constexpr int kPer16 = 8;
};
template <>
struct Elem<BITSTACK_T_F32> {
    typedef float type;
    static constexpr int kPer16 = 4;
};

// 16 bytes of elements that lie at any element's address: the hardware loads and stores them at once.  (Element by element rows of an odd width took
// twice as long: 2048 x 8191 in fp16 to 8 bits 24.6 us.)
template <int T>
struct Piece {
    typedef typename Elem<T>::type type __attribute__((ext_vector_type(Elem<T>::kPer16)));
    typedef type loose __attribute__((aligned(sizeof(typename Elem<T>::type))));
};

// N consecutive elements as floats, those at or past `n` zero
template <int T, int N>
__device__ __forceinline__ void load_elems(const typename Elem<T>::type* p, int n, float (&v)[N]) {
    constexpr int K = Elem<T>::kPer16;
    static_assert(N % K == 0, "whole 16-byte pieces");
    if (n >= N) {
#pragma unroll
        for (int i = 0; i < N / K; ++i) {
            const typename Piece<T>::type u = reinterpret_cast<const typename Piece<T>::loose*>(p)[i];
#pragma unroll
            for (int e = 0; e < K; ++e) v[i * K + e] = float(u[e]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < n ? float(p[i]) : 0.0f;
    }
}

// The least e with amax <= 448 * 2^e, at least -126, biased by 127 (448 = 1.75 * 2^8; amax = 1.f * 2^q): exact, and so is the division by
// 2^e.  amax finite.
__device__ __forceinline__ int f8_exponent(float amax) {
    const unsigned bits = __float_as_uint(amax);
    const int e = int(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < 1 ? 1 : e;
}
__device__ __forceinline__ float f8_inverse(int biased) { return __uint_as_float(unsigned(254 - biased) << 23); }   // 2^-e; biased <= 247

// Four floats, at most 448 in magnitude, to e4m3 (round to nearest even)
__device__ __forceinline__ unsigned f8_x4(float a, float b, float c, float d) {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return unsigned(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}
// |v| as an integer that orders like it, NaN and infinity above all others
__device__ __forceinline__ unsigned f8_magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// g / (1 + exp(-g)) u by the hardware's exp2 and reciprocal (1 ulp each), relative error 8 * 2^-24 (of which they are 4).  -g / ln 2 is rounded, and at 50 that
// is 50 half steps of the result: what it misses, in units of ln 2, comes after as a factor 1 + d.  Below -64 both terms of the denominator are taken 2^-64 times,
// so that the product is there as long as fp32, denormals included, holds it (down to gates of -132).
__device__ __forceinline__ float f8_gate(float g, float u) {
    constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147182464599609375f, kLn2Rest = -1.904654299957767878e-9f;   // ln 2 = their sum
    const float p = __builtin_amdgcn_fmed3f(g * -kLog2e, -150.0f, 250.0f);   // beyond, exp2 is 0 or infinite and g may be anything
    const float d = fmaf(-kLn2Rest, p, fmaf(-kLn2, p, -g));
    const bool far = g < -64.0f;
    const float k = far ? 0x1p-64f : 1.0f;
    return g * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(p - (far ? 64.0f : 0.0f)), 1.0f + d, k)) * u * k;
}

// The work list of a product grouped by expert: made by the launch that brings the activations to 8 bits, or (rows 0 there) by itself
struct F8WorkList {
    const int* offsets = nullptr;   // null: none
    int experts = 0, rows = 0, tile_rows = 0, n_tiles = 0;
    F8Tile* tiles = nullptr;
};
hipError_t launch_f8_quantise(const void* x, int dtype, size_t ld, int rows, int in, bool gated, unsigned char* q, unsigned char* s,
                              const F8WorkList& list, hipStream_t st);
hipError_t launch_f8_quantise_weight(const void* w, int dtype, size_t ld, int out, int in, unsigned char* q, size_t ld_q,
                                     unsigned char* s, hipStream_t st);
// Kernel and column slices of a product, from sizes alone
struct F8Plan {
    int kernel, slices, tile_rows, n_tiles;   // tile_rows: rows of y in a tile; n_tiles: tiles of y's rows, at most
    int tiles;                                // of the weight's rows and y's
    size_t part_bytes;                        // partial sums
};
// room: bytes for the work list and the partial sums; with less than they need there are fewer slices
F8Plan f8_plan(int rows, int out, int in, int experts, bool grouped, bool exact, bool ws_f32, size_t room = ~size_t(0));
// The same for a product of one group all of whose sums are left as partial ones
F8Plan f8_plan_parts(int rows, int out, int in, bool exact, bool ws_f32, size_t room = ~size_t(0));
// a launch has fewer than 2^32 threads, 512 to a workgroup
inline bool f8_launchable(const F8Plan& plan) { return size_t(plan.tiles) * plan.slices <= (size_t(1) << 23) - 8; }
hipError_t launch_f8_product(const F8Params& p, const F8Plan& plan, hipStream_t st);
hipError_t launch_f8_epilogue(const F8Params& p, const F8Plan& plan, hipStream_t st);   // its kernels with an epilogue
hipError_t launch_f8_gated(const F8Params& p, const F8Plan& plan, hipStream_t st);
bool f8_force_kernel(int kernel);   // measurement hook, 0: the choice by size; false: no such kernel

size_t route_workspace_bytes(int tokens, int experts);
struct RouteParams {
    const void* logits;
    size_t ld;
    int tokens, experts, top_k, renormalise;
    int* chosen;
    float* weights;
    int* slots;
    int* index;
    int* offsets;
    int* counts;   // [chunks][experts]
    int chunks;
};
hipError_t launch_route(RouteParams p, int dtype, void* workspace, hipStream_t st);
struct CombineParams {
    const void* h;
    void* y;
    const int* slots;
    const float* weights;
    size_t ld_h, ld_y;
    int h_rows, width, tokens, top_k;
};
hipError_t launch_combine(const CombineParams& p, int dtype, hipStream_t st);

int hip_error(hipError_t e);   // host.cpp: remembers e for bitstack_last_hip_error, BITSTACK_E_HIP

}  // namespace bitstack
