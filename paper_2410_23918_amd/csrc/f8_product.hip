// Products in 8-bit floating point with a scale for each 128 columns of a token and for each 128 x 128 of the weight,
//
//     y[t][o] = sum_b sx[t][b] sw[o / 128][b] sum_{j in block b} x8[t][j] w8[o][j],
//
// and the same with the rows of y grouped by expert.  v_mfma_scale_f32_16x16x128_f8f6f4 multiplies one block of 16 rows and 16 tokens and
// takes powers of two as scales of its operands: those of the activations, and those of weights that hold them so, cost nothing.
// A weight's fp32 scale is the same for the whole block: the product goes into zeros and is added with it.
//   That instruction (and the unscaled one for 8 bits) adds eight neighbouring columns at a time, with every product cut to a multiple of
// 2^-13 of the largest one's power of two; what it adds these sums to is fp32.  (Measured: 2^16 + 2^2 loses its second term within eight columns, 2^16 + 2^3 does
// not; across them 24 bits are kept.)  Outputs of 16 bits are coarser: 5e-5 of y's norm with a few columns 30 times louder than the rest, 4.9e-4 is
// half a step of fp16.  Outputs in fp32 are asked for where that is too much: their operands are turned into fp16, which holds every e4m3
// number, and v_mfma_f32_16x16x32_f16 keeps fp32 throughout, at half the rate.
//   The matrix instruction's columns: a lane holds 32 bytes of row lane % 16; which of the block's columns they are is free as long as both
// operands agree, since they share the scale.  D: lane l holds rows 4 (l / 16) .. + 3 of the weight and token l % 16.
#include <hip/hip_runtime.h>

#include "f8.h"
#include "kparams.h"

namespace bitstack {

typedef int v8i __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v4f mfma_f8(const v8i& w, const v8i& x, const v4f& c, int w_scale, int x_scale) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, 0, w_scale, 0, x_scale);
}
constexpr int kOne = 127;   // the scale 1

__device__ __forceinline__ v8i join(const v4i& a, const v4i& b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// zeroes the bytes of a 16-byte piece from its column `n` on (n may be anything)
__device__ __forceinline__ v4i keep_columns(v4i v, int n) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int k = n - 4 * d;
        v[d] &= k >= 4 ? -1 : k <= 0 ? 0 : (1 << (8 * k)) - 1;
    }
    return v;
}

// four outputs of a token, rows n .. n + 3
__device__ __forceinline__ void store4(const F8Params& p, int row, int n, const v4f& v) {
    if (n >= p.out) return;
    const size_t at = size_t(row) * p.ldy + n;
    const bool whole = p.y_vec && n + 4 <= p.out;
    if (p.y_dtype == BITSTACK_T_F32) {
        float* const y = static_cast<float*>(p.y) + at;
        if (whole) *reinterpret_cast<v4f*>(y) = v;
        else
            for (int i = 0; i < 4 && n + i < p.out; ++i) y[i] = v[i];
    } else if (p.y_dtype == BITSTACK_T_F16) {
        typedef _Float16 v4h __attribute__((ext_vector_type(4)));
        const v4h h = {_Float16(v[0]), _Float16(v[1]), _Float16(v[2]), _Float16(v[3])};
        _Float16* const y = static_cast<_Float16*>(p.y) + at;
        if (whole) *reinterpret_cast<v4h*>(y) = h;
        else
            for (int i = 0; i < 4 && n + i < p.out; ++i) y[i] = h[i];
    } else {
        typedef __bf16 v4b __attribute__((ext_vector_type(4)));
        const v4b h = {__bf16(v[0]), __bf16(v[1]), __bf16(v[2]), __bf16(v[3])};
        __bf16* const y = static_cast<__bf16*>(p.y) + at;
        if (whole) *reinterpret_cast<v4b*>(y) = h;
        else
            for (int i = 0; i < 4 && n + i < p.out; ++i) y[i] = h[i];
    }
}

// How a tile is multiplied: the scales of the weight are powers of two, or fp32 numbers; or the outputs are fp32 (either scales)
enum F8Mode { kModeE8M0, kModeF32, kModeExact };

__device__ __forceinline__ float scale_of(int byte) {   // 2^(byte - 127), 255: NaN
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : unsigned(byte) << 23);
}

// 32 e4m3 numbers as fp16, exactly
struct Halves {
    v8h h[4];
};
__device__ __forceinline__ Halves to_halves(const v8i& v) {
    Halves o;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
        const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[d], 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v[d], 1.0f, true);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            o.h[d / 2][4 * (d & 1) + e] = lo[e];
            o.h[d / 2][4 * (d & 1) + 2 + e] = hi[e];
        }
    }
    return o;
}
__device__ __forceinline__ v4f mfma_halves(const Halves& w, const Halves& x) {
    v4f c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.h[k], x.h[k], c, 0, 0, 0);
    return c;
}

// acc += a block's products of FR x FT fragments, with its scales (xs: of the lane's token in each fragment; sw: the weight's, in bits).  D's
// columns are the tokens: a lane's four results have one scale.
template <int FR, int FT, int MODE>
__device__ __forceinline__ void multiply(v4f (&acc)[FR][FT], const v8i (&w)[FR], const v8i (&x)[FT], const int (&xs)[FT], int sw, bool sw_f32) {
    if constexpr (MODE == kModeExact) {
        const float f = sw_f32 ? __int_as_float(sw) : scale_of(sw);
        Halves wh[FR];
#pragma unroll
        for (int j = 0; j < FR; ++j) wh[j] = to_halves(w[j]);
#pragma unroll
        for (int i = 0; i < FT; ++i) {
            const Halves xh = to_halves(x[i]);
            const float g = scale_of(xs[i]);
#pragma unroll
            for (int j = 0; j < FR; ++j) {
                const v4f part = mfma_halves(wh[j], xh);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[j][i][v] = fmaf(part[v] * g, f, acc[j][i][v]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < FT; ++i)
#pragma unroll
            for (int j = 0; j < FR; ++j) {
                if constexpr (MODE == kModeF32) {
                    const v4f part = mfma_f8(w[j], x[i], v4f{0.0f, 0.0f, 0.0f, 0.0f}, kOne, xs[i]);
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[j][i][v] = fmaf(part[v], __int_as_float(sw), acc[j][i][v]);
                } else {
                    acc[j][i] = mfma_f8(w[j], x[i], acc[j][i], sw, xs[i]);
                }
            }
    }
}

// A tile of 16 FR rows of the weight x 16 FT tokens.  The eight wavefronts of a workgroup take every eighth block of columns each, straight
// from memory into registers (nothing of a tile is read by two of them), DEPTH blocks ahead; their sums meet in LDS.
template <int FR, int FT, int DEPTH, int MODE>
__global__ __launch_bounds__(512, 2) void k_f8_slices(F8Params p) {
    __shared__ v4f red[8 * FR * FT * 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ln = lane & 15, kg = lane >> 4;
    // ids are dealt round-robin to the 8 XCDs: all token tiles of a row tile meet in one L2
    const int nrt = (p.out + 16 * FR - 1) / (16 * FR);
    const int xcd = blockIdx.x & 7, place = blockIdx.x >> 3;
    const int rt = xcd + 8 * (place / p.n_tiles), tt = place % p.n_tiles;
    if (rt >= nrt) return;
    F8Tile t = {0, tt * 16 * FT, min(16 * FT, p.rows - tt * 16 * FT), 0};
    if (p.tiles) t = p.tiles[tt];
    const int expert = __builtin_amdgcn_readfirstlane(t.expert), row0 = __builtin_amdgcn_readfirstlane(t.row0),
              rows = __builtin_amdgcn_readfirstlane(t.rows);
    if (rows <= 0) return;
    const int n0 = rt * 16 * FR;
    v4f acc[FR][FT];
#pragma unroll
    for (int j = 0; j < FR; ++j)
#pragma unroll
        for (int i = 0; i < FT; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    if (expert >= 0) {
        const unsigned char* const wbase = p.w + (size_t(expert) * p.out + n0) * p.ldw;
        const int w_rows = min(16 * FR, p.out - n0);
        const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(wbase), 0,
                                                                            int((w_rows - 1) * p.ldw + (p.in + 15) / 16 * 16), 0x00020000);
        const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(p.x), 0, int(unsigned(p.x_rows) * unsigned(p.kp)), 0x00020000);
        const bool s_f32 = MODE == kModeF32 || (MODE == kModeExact && p.ws_f32);
        const int s_size = s_f32 ? 4 : 1;
        const size_t s_row = (size_t(expert) * ((p.out + 127) / 128) + n0 / 128) * p.kb;
        const __amdgpu_buffer_rsrc_t sr = __builtin_amdgcn_make_buffer_rsrc(
const_cast<unsigned char*>(static_cast<const unsigned char*>(p.ws)) + s_row * s_size, 0, p.kb * s_size, 0x00020000);
        const __amdgpu_buffer_rsrc_t xsr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(p.xs), 0, int(unsigned(p.x_rows) * unsigned(p.ks)), 0x00020000);
        unsigned w_off[FR], x_off[FT], xs_off[FT];
#pragma unroll
        for (int j = 0; j < FR; ++j) w_off[j] = unsigned(min(16 * j + ln, w_rows - 1)) * unsigned(p.ldw) + kg * 16;
#pragma unroll
        for (int i = 0; i < FT; ++i) {
            int r = row0 + min(16 * i + ln, rows - 1);
            if (p.index) r = p.index[r];
            const bool there = unsigned(r) < unsigned(p.x_rows);
            x_off[i] = there ? unsigned(r) * unsigned(p.kp) + kg * 16 : 0x80000000u;
            xs_off[i] = there ? unsigned(r) * unsigned(p.ks) : 0x80000000u;
        }
        struct Stage {
            v4i w[FR][2], x[FT][2];
            int xs[FT];
            int sw;
        };
        Stage st[DEPTH];
        // past the last block nothing is read and zeros arrive
        auto load = [&](Stage& s, int b) __attribute__((always_inline)) {
            const bool in = b < p.kb;
            const unsigned oob = in ? 0u : 0x80000000u, col = in ? unsigned(b) * 128u : 0u;
#pragma unroll
            for (int j = 0; j < FR; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) s.w[j][h] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(wr, int((w_off[j] + col + h * 64) | oob), 0, 0));
#pragma unroll
            for (int i = 0; i < FT; ++i) {
#pragma unroll
                for (int h = 0; h < 2; ++h) s.x[i][h] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(xr, int((x_off[i] + col + h * 64) | oob), 0, 0));
                s.xs[i] = __builtin_amdgcn_raw_buffer_load_b8(xsr, int((xs_off[i] + b) | oob), 0, 0);
            }
            if (s_f32) s.sw = __builtin_amdgcn_raw_buffer_load_b32(sr, int((unsigned(b) * 4u) | oob), 0, 0);
            else s.sw = __builtin_amdgcn_raw_buffer_load_b8(sr, int(unsigned(b) | oob), 0, 0);
        };
        const bool ragged = p.in % 128 != 0;
        auto products = [&](Stage& s, int b) __attribute__((always_inline)) {
            if (ragged && b == p.kb - 1) {   // the last block ends early: the weight's rows may go on with anything
#pragma unroll
                for (int j = 0; j < FR; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) s.w[j][h] = keep_columns(s.w[j][h], p.in - (b * 128 + h * 64 + kg * 16));
            }
            v8i w[FR], x[FT];
#pragma unroll
            for (int j = 0; j < FR; ++j) w[j] = join(s.w[j][0], s.w[j][1]);
#pragma unroll
            for (int i = 0; i < FT; ++i) x[i] = join(s.x[i][0], s.x[i][1]);
            multiply<FR, FT, MODE>(acc, w, x, s.xs, s.sw, s_f32);
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) load(st[d], wave + 8 * d);
        for (int b = wave; b < p.kb; b += 8 * DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (b + 8 * d < p.kb) products(st[d], b + 8 * d);
                load(st[d], b + 8 * (DEPTH + d));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < FR; ++j)
#pragma unroll
        for (int i = 0; i < FT; ++i) red[((wave * FR + j) * FT + i) * 64 + lane] = acc[j][i];
    __syncthreads();
    for (int k = tid; k < FR * FT * 64; k += 512) {
        v4f sum = red[k];
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += red[w * FR * FT * 64 + k];
        const int l = k & 63, i = (k >> 6) % FT, j = (k >> 6) / FT;
        const int tok = 16 * i + (l & 15);
        if (tok < rows) store4(p, row0 + tok, n0 + 16 * j + 4 * (l >> 4), sum);
    }
}

template <int FR, int FT, int DEPTH>
static void slices(const F8Params& p, hipStream_t st) {
    const int nrt = (p.out + 16 * FR - 1) / (16 * FR);
    const dim3 grid(unsigned(8 * ((nrt + 7) / 8)) * unsigned(p.n_tiles));
    if (p.y_dtype == BITSTACK_T_F32) hipLaunchKernelGGL((k_f8_slices<FR, FT, DEPTH, kModeExact>), grid, dim3(512), 0, st, p);
    else if (p.ws_f32) hipLaunchKernelGGL((k_f8_slices<FR, FT, DEPTH, kModeF32>), grid, dim3(512), 0, st, p);
    else hipLaunchKernelGGL((k_f8_slices<FR, FT, DEPTH, kModeE8M0>), grid, dim3(512), 0, st, p);
}

size_t f8_worklist_entries(int rows, int experts) { return size_t(rows) / 16 + 2 + size_t(rows < experts ? rows : experts); }

hipError_t launch_f8_product(const F8Params& args, int experts, F8Tile* list, const int* offsets, hipStream_t st) {
    F8Params p = args;
    const int tile_rows = p.rows <= 16 ? 16 : 64;
    p.n_tiles = (p.rows + tile_rows - 1) / tile_rows;
    if (offsets) {
        // every group's rows, rounded up to tiles, and those of the rows past the last group
        p.n_tiles = p.rows / tile_rows + 1 + (p.rows < experts ? p.rows : experts);
        p.tiles = list;
        const hipError_t e = launch_f8_worklist(offsets, experts, p.rows, tile_rows, list, p.n_tiles, st);
        if (e != hipSuccess) return e;
    }
    if (tile_rows == 16) slices<1, 1, 4>(p, st);
    else slices<4, 4, 1>(p, st);
    return hipGetLastError();
}

}  // namespace bitstack
