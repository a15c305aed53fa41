// Products in 8-bit floating point with a scale for each 128 columns of a token and for each 128 x 128 of the weight,
//
//     y[t][o] = sum_b sx[t][b] sw[o / 128][b] sum_{j in block b} x8[t][j] w8[o][j],
//
// and the same with the rows of y grouped by expert.  v_mfma_scale_f32_16x16x128_f8f6f4 multiplies one block of 16 rows and 16 tokens and
// takes powers of two as scales of its operands: those of the activations, and those of weights that hold them so, cost nothing.
// A weight's fp32 scale is the same for the whole block: its power of two goes to the instruction too, the product goes into zeros and is added
// times the rest.
//   That instruction (and the unscaled one for 8 bits) adds eight neighbouring columns at a time, with every product cut to a multiple of
// 2^-13 of the largest one's power of two; what it adds these sums to is fp32.  (Measured: 2^16 + 2^2 loses its second term within eight columns, 2^16 + 2^3 does
// not; across them 24 bits are kept.)  Outputs of 16 bits are coarser: 5e-5 of y's norm with a few columns 30 times louder than the rest, 4.9e-4 is
// half a step of fp16.  Outputs in fp32 are asked for where that is too much: their operands are turned into fp16, which holds every e4m3
// number, and v_mfma_f32_16x16x32_f16 keeps fp32 throughout, at half the rate.
//   The matrix instruction's columns: a lane holds 32 bytes of row lane % 16; which of the block's columns they are is free as long as both
// operands agree, since they share the scale.  D: lane l holds rows 4 (l / 16) .. + 3 of the weight and token l % 16.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>

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
template <int T>
__device__ __forceinline__ void store4_as(const F8Params& p, int row, int n, const v4f& v) {
    typedef typename Elem<T>::type E;
    typedef E four __attribute__((ext_vector_type(4)));
    typedef four loose __attribute__((aligned(sizeof(E))));
    const four o = {E(v[0]), E(v[1]), E(v[2]), E(v[3])};
    E* const y = static_cast<E*>(p.y) + size_t(row) * p.ldy + n;
    if (n + 4 <= p.out) {
        *reinterpret_cast<loose*>(y) = o;
    } else {
        for (int i = 0; i < 4 && n + i < p.out; ++i) y[i] = o[i];
    }
}
__device__ __forceinline__ void store4(const F8Params& p, int row, int n, const v4f& v) {
    if (p.y_dtype == BITSTACK_T_F32) store4_as<BITSTACK_T_F32>(p, row, n, v);
    else if (p.y_dtype == BITSTACK_T_F16) store4_as<BITSTACK_T_F16>(p, row, n, v);
    else store4_as<BITSTACK_T_BF16>(p, row, n, v);
}

template <class E>
__device__ __forceinline__ v2u pack4(const v4f& v) {
    typedef E v4e __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(v2u, v4e{E(v[0]), E(v[1]), E(v[2]), E(v[3])});
}

// How a tile is multiplied: the scales of the weight are powers of two, or fp32 numbers; or the outputs are fp32 (either scales)
enum F8Mode { kModeE8M0, kModeF32, kModeExact };

// A block's scale of the weight (sw, in bits, the same in all lanes) as factor * 2^(byte - 127), in scalar registers.  An fp32 scale's power of two is taken
// off it and goes where that of the activations is, so that nothing passes fp32's range, or drops below it, on the way to a y that does not; the
// factor is in [1, 2) (0, less than 1 for a denormal scale, or no number).
struct WeightScale {
    int byte;
    float factor;
};
__device__ __forceinline__ WeightScale weight_scale(int sw, bool sw_f32) {
    sw = __builtin_amdgcn_readfirstlane(sw);
    if (!sw_f32) return {sw, sw == 255 ? __uint_as_float(0x7fc00000u) : 1.0f};
    int byte = sw >> 23 & 255, factor = (sw & 0x807fffff) | 0x3f800000;
    if (__builtin_expect(unsigned(byte - 1) >= 254u, 0)) {   // zero, denormal or no number
        byte = byte ? 254 : 1;
        factor = __builtin_amdgcn_readfirstlane(__float_as_int(__builtin_amdgcn_ldexpf(__int_as_float(sw), kOne - byte)));
    }
    return {byte, __int_as_float(factor)};
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

// acc += a block's products of FR fragments of the weight and one of the activations, with their scales (xs: of the lane's token; sw: the
// weight's).  D's columns are the tokens: a lane's four results have one scale.
template <int FR, int MODE, class Weights>
__device__ __forceinline__ void multiply(v4f* const (&acc)[FR], const Weights (&w)[FR], const v8i& x, int xs, const WeightScale& sw) {
    if constexpr (MODE == kModeExact) {
        // Both powers of two in two halves: a block's sum lies between 2^-18 and 2^25, and neither half takes it out of range where y is not.  One
        // rounding, that of the sum.
        const int e = sw.byte + xs - 2 * kOne, half = e >> 1;   // half >= -127, where 0 will do
        const float f = __builtin_amdgcn_ldexpf(sw.factor, e - half), g = __int_as_float((half + 127) << 23);
        const Halves xh = to_halves(x);
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            const v4f part = mfma_halves(w[j], xh);
#pragma unroll
            for (int v = 0; v < 4; ++v) (*acc[j])[v] = fmaf(part[v] * g, f, (*acc[j])[v]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            if constexpr (MODE == kModeF32) {
                const v4f part = mfma_f8(w[j], x, v4f{0.0f, 0.0f, 0.0f, 0.0f}, sw.byte, xs);
#pragma unroll
                for (int v = 0; v < 4; ++v) (*acc[j])[v] = fmaf(part[v], sw.factor, (*acc[j])[v]);
            } else {
                *acc[j] = mfma_f8(w[j], x, *acc[j], sw.byte, xs);
            }
        }
    }
}
// the same for FT fragments of the activations; after(i) follows those of fragment i
template <int FR, int FT, int MODE, class After>
__device__ __forceinline__ void multiply_all(v4f (&acc)[FR][FT], const v8i (&w)[FR], const v8i (&x)[FT], const int (&xs)[FT], const WeightScale& sw, After after) {
    typedef typename std::conditional<MODE == kModeExact, Halves, v8i>::type Weights;
    Weights f[FR];
#pragma unroll
    for (int j = 0; j < FR; ++j) {
        if constexpr (MODE == kModeExact) f[j] = to_halves(w[j]);
        else f[j] = w[j];
    }
#pragma unroll
    for (int i = 0; i < FT; ++i) {
        v4f* to[FR];
#pragma unroll
        for (int j = 0; j < FR; ++j) to[j] = &acc[j][i];
        multiply<FR, MODE>(to, f, x[i], xs[i], sw);
        after(i);
    }
}

// The activations of a lane as they come, 32 columns of a token in a block, of type T (16 bits), to e4m3: what k_f8_quantise makes of them
constexpr int kRowsF8 = BITSTACK_T_F8;
template <int T>
__device__ __forceinline__ void columns_to_f8(const v4i (&raw)[4], v8i& x, int& scale) {
    typedef typename Elem<T>::type piece __attribute__((ext_vector_type(8)));
    float v[32];
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v[i] = float(__builtin_bit_cast(piece, raw[i / 8])[i % 8]);
        m = max(m, f8_magnitude(v[i]));
    }
    m = max(m, unsigned(__shfl_xor(int(m), 16)));   // the other lanes of the token
    m = max(m, unsigned(__shfl_xor(int(m), 32)));
    const bool bad = m >= 0x7f800000u;
    scale = bad ? kOne : f8_exponent(__uint_as_float(m));
    const float inv = f8_inverse(scale);
#pragma unroll
    for (int d = 0; d < 8; ++d) x[d] = bad ? 0x7f7f7f7f : int(f8_x4(v[4 * d] * inv, v[4 * d + 1] * inv, v[4 * d + 2] * inv, v[4 * d + 3] * inv));
}

// The tile of a workgroup.  Ids are dealt round-robin to the 8 XCDs: each takes an eighth of the tiles there are, as many as the next to within one, neighbours
// in an order in which a few tiles of tokens go through all rows of the weight, so that what 32 compute units read at a time meets in one L2.  (Every fourth
// tile of rows x every second of tokens instead left half the XCDs with twice as many where there are three tiles of tokens: 14336 x 4096, 300 tokens, 256 x 128 in
// five slices: 60.6 us, 41.5.)
__device__ __forceinline__ bool tile_of(const F8Params& p, int nrt, unsigned together, int& rt, int& tt, int& slice) {
    const unsigned nt = p.tiles ? unsigned(min(__builtin_amdgcn_readfirstlane(p.tiles[0].all), p.n_tiles)) : unsigned(p.n_tiles);
    const unsigned each = unsigned(nrt) * nt, all = each * unsigned(p.slices), per = (all + 7) / 8, place = blockIdx.x >> 3;
    unsigned v = (blockIdx.x & 7) * per + place;
    if (place >= per || v >= all) return false;
    slice = int(v / each);
    v %= each;
    const unsigned group = v / (unsigned(nrt) * together), size = min(together, nt - group * together);
    v -= group * (unsigned(nrt) * together);
    rt = int(v / size);
    tt = int(group * together + v % size);
    return true;
}

// A tile of 16 FR rows of the weight x 16 FT tokens.  The eight wavefronts of a workgroup take every eighth block of columns each, straight
// from memory into registers (nothing of a tile is read by two of them), DEPTH blocks ahead; their sums meet in LDS.
//   Bound by the stream of the weight, of which four wavefronts a SIMD keep 16 to 32 KB in flight on a compute unit: one token through two of eight 14336 x 4096
// experts 26.6 us, 4.4 TB/s, 57 tokens through six of 64 experts of 1024 x 4096 48.6 us, 4.6 TB/s (16 rows as tokens stay in registers; tiles of 64 x 16, so that a
// block of the activations is read for 64 rows).  Small weights are bound by
// the launch and three latencies (first load, LDS, store): 57 tokens through 1056 x 2001 in fp32, 16 x 16 tiles, 6.2 us.  With 32 and 64 tokens each
// wavefront's operands come from L2 again for every 64 rows.
//   T: type of the activations.  With one fragment of tokens they may come as they are, in no groups, and are brought to 8 bits on the way (a block of a token
// lies in four lanes), by every workgroup anew: one launch instead of two.  One token through 1024 x 4096: 7.0 us, 5.5 and 2.4 + a launch for the rows
// quantised before; 14336 x 4096 16.7, 16.2 and 2.4; 4096 x 14336, where 256 workgroups convert 112 blocks each, 20.4, 14.4 and 2.5.
template <int FR, int FT, int DEPTH, int MODE, int T>
__global__ __launch_bounds__(512, 2) void k_f8_slices(F8Params p) {
    constexpr bool kRaw = T != kRowsF8;
    static_assert(!kRaw || FT == 1, "one fragment of raw tokens");
    if constexpr (kRaw) p.tiles = nullptr, p.index = nullptr;   // in no groups, rows as they come
    __shared__ v4f red[8 * FR * FT * 64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ln = lane & 15, kg = lane >> 4;
    int rt, tt, slice;
    if (!tile_of(p, (p.out + 16 * FR - 1) / (16 * FR), unsigned(p.n_tiles), rt, tt, slice)) return;
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
        const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(p.x), 0, int(unsigned(p.x_bytes)), 0x00020000);
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
            x_off[i] = !there ? 0x80000000u : kRaw ? unsigned(r) * unsigned(p.x_ld) : unsigned(r) * unsigned(p.kp) + kg * 16;
            xs_off[i] = there ? unsigned(r) * 4u : 0x80000000u;
        }
        struct Stage {
            v4i w[FR][2], x[FT][2];
            v4i raw[kRaw ? 4 : 1];
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
                if constexpr (kRaw) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int c = b * 128 + h * 64 + kg * 16;
                        const unsigned at = (x_off[i] + unsigned(c) * 2u) | oob | (c < p.in ? 0u : 0x80000000u);
#pragma unroll
                        for (int k = 0; k < 2; ++k) s.raw[h * 2 + k] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(xr, int(at + k * 16), 0, 0));
                    }
                    continue;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) s.x[i][h] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(xr, int((x_off[i] + col + h * 64) | oob), 0, 0));
                s.xs[i] = __builtin_amdgcn_raw_buffer_load_b8(xsr, int((xs_off[i] + (b & 3)) | oob), int(in ? unsigned(b >> 2) * unsigned(p.x_rows) * 4u : 0u), 0);
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
            for (int i = 0; i < FT; ++i) {
                if constexpr (kRaw) columns_to_f8<T>(s.raw, x[i], s.xs[i]);
                else x[i] = join(s.x[i][0], s.x[i][1]);
            }
            multiply_all<FR, FT, MODE>(acc, w, x, s.xs, weight_scale(s.sw, s_f32), [](int) __attribute__((always_inline)) {
                if constexpr (MODE == kModeExact && FT == 4) __builtin_amdgcn_sched_barrier(0);   // one fragment's conversions at a time: registers
            });
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

// Larger tiles: eight wavefronts, WR x WT, each with 16 FR rows of the weight x 16 FT tokens; both operands go through LDS, a block of columns (a
// step) at a time, in a ring that the loads fill directly.
//   The two wavefronts of a SIMD take turns: while one reads its fragments of a step from LDS the other one multiplies, and a barrier ends each
// phase.  Wavefronts 0-3 read step b in phase 2 b and multiply it in 2 b + 1, wavefronts 4-7 one phase later.  So the buffer of step b is free
// after phase 2 b + 1, and the step RING further on is requested into it at the beginning of the next one.
//   LDS: a row's 128 bytes, its 16-byte piece c at position c ^ f(row), f such that the sixteen rows that a fragment's read touches at a time
// meet every bank once.  Row i of the weight's fragment j is row (i / 4) 4 FR + 4 j + i % 4 of the wavefront's tile, so that a lane ends with 4 FR neighbouring
// outputs of a token.
//   Bound by LDS and latency: a phase reads 32 to 64 KB of fragments (128 bytes a clock) and multiplies for 128 to 256 clocks; 128 x 64 takes 0.54 us a step alone and
// 0.9 for two workgroups of a compute unit, 128 x 128 0.78, 256 x 128 1.08; products alone would take 0.12, 0.25 and 0.50.  300 tokens
// through 4096 x 14336 (256 x 128, five column slices, fp32 scales): 36.9 us, 0.95 PFLOP/s, and 6.6 to join them.
//   The activations' scales come with the step, four bytes a token (four steps' scales, of which one is used); the weight's, the same for 128
// rows, are kept one to a lane for 64 steps.
template <int FR, int FT, int WR, int WT, int MODE>
struct F8TileShape {
    static constexpr int kWaves = 8, kRows = 16 * FR * WR, kToks = 16 * FT * WT;
    static constexpr int kStep = (kRows + kToks) * 128 + 4 * 256;   // bytes, a multiple of 128 (the scales of 4 x 64 tokens)
    // Small tiles: two workgroups on a compute unit, with half the LDS each, so that one multiplies while the other one waits.  128 x 64, 1024 tokens
    // through 4096 x 4096: 41 us and 31; 128 x 128 there, where two leave a ring of two: 28 and 36, so those stay alone.
    static constexpr bool kTwo = kRows * kToks <= 128 * 64;
    static constexpr int kRing = ((kTwo ? 81920 : 163840) - 256) / kStep;
    static constexpr int kSize = MODE == kModeExact ? 4 : 2, kOutLd = kRows * kSize + 16;   // the output tile in LDS
    static constexpr int kRingLds = kRing * kStep + 256, kLds = kRingLds > kToks * kOutLd ? kRingLds : kToks * kOutLd;
    static_assert(WR * WT == 8 && WR <= 4 && kRing >= 2 && kLds <= 163840 && 16 * FR <= 128 && kRows % (8 * kWaves) == 0 && kToks % 64 == 0 && kToks <= 256, "whole loads, one weight scale a wavefront, scales for the first four wavefronts");
};

// A tile's sums leave the kernel (all LDS is free).  FR x FT fragments a wavefront, WR x WT wavefronts.
template <class S, int FR, int FT, int WR>
__device__ __forceinline__ void finish_tile(const F8Params& p, unsigned char* smem, const v4f (&acc)[FR][FT], size_t tile, int n0, int row0, int rows) {
    const int tid = threadIdx.x, lane = tid & 63, ln = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave % WR, wt = wave / WR;
    if (p.slices > 1) {   // partial sums, as the lanes hold them: k_f8_join adds them up
        v4f* const to = reinterpret_cast<v4f*>(p.part) + (tile * 8 + wave) * (FR * FT * 64) + lane;
#pragma unroll
        for (int j = 0; j < FR; ++j)
#pragma unroll
            for (int i = 0; i < FT; ++i) to[(j * FT + i) * 64] = acc[j][i];
        return;
    }
    // the tile's outputs meet in LDS, token by token, and leave in 16-byte pieces
    constexpr int kSize = S::kSize, kLd = S::kOutLd;
    unsigned char* const mine = smem + (wt * 16 * FT + ln) * kLd + (wr * 16 * FR + kg * 4 * FR) * kSize;
    auto put = [&](auto turn) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < FT; ++i)
#pragma unroll
            for (int j = 0; j < FR; ++j) turn(acc[j][i], mine + i * 16 * kLd + j * 4 * kSize);
    };
    if constexpr (S::kSize == 4) put([](const v4f& v, unsigned char* to) { *reinterpret_cast<v4f*>(to) = v; });
    else if (p.y_dtype == BITSTACK_T_F16) put([](const v4f& v, unsigned char* to) { *reinterpret_cast<v2u*>(to) = pack4<_Float16>(v); });
    else put([](const v4f& v, unsigned char* to) { *reinterpret_cast<v2u*>(to) = pack4<__bf16>(v); });
    __syncthreads();
    constexpr int kPieces = S::kRows * kSize / 16, kEach = 16 / kSize;
    for (int k = tid; k < S::kToks * kPieces; k += 64 * S::kWaves) {
        const int tok = k / kPieces, piece = k % kPieces, n = n0 + piece * kEach;
        if (tok >= rows) break;
        if (n >= p.out) continue;
        const unsigned char* const from = smem + tok * kLd + piece * 16;
        unsigned char* const y = static_cast<unsigned char*>(p.y) + (size_t(row0 + tok) * p.ldy + n) * kSize;
        if (n + kEach <= p.out) {
            typedef v4i loose __attribute__((aligned(2)));   // y lies at any element
            *reinterpret_cast<loose*>(y) = *reinterpret_cast<const v4i*>(from);
        } else {
            for (int e = 0; e < kEach && n + e < p.out; ++e) {
                if constexpr (kSize == 4) reinterpret_cast<float*>(y)[e] = reinterpret_cast<const float*>(from)[e];
                else reinterpret_cast<unsigned short*>(y)[e] = reinterpret_cast<const unsigned short*>(from)[e];
            }
        }
    }
}

template <int FR, int FT, int WR, int WT, int MODE>
__global__ __launch_bounds__(512, (F8TileShape<FR, FT, WR, WT, MODE>::kTwo ? 4 : 2)) void k_f8_tile(F8Params p) {
    typedef F8TileShape<FR, FT, WR, WT, MODE> S;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave % WR, wt = wave / WR;
    const bool late = wave >= 4;
    const int ln = lane & 15, kg = lane >> 4;
    const int nrt = (p.out + S::kRows - 1) / S::kRows;
    int rt, tt, slice;
    if (!tile_of(p, nrt, p.tiles ? 8 : 4, rt, tt, slice)) return;
    const int first = slice * p.slice_blocks, last = min(first + p.slice_blocks, p.kb);   // blocks of columns
    F8Tile t = {0, tt * S::kToks, min(S::kToks, p.rows - tt * S::kToks), 0};
    if (p.tiles) t = p.tiles[tt];
    const int expert = __builtin_amdgcn_readfirstlane(t.expert), row0 = __builtin_amdgcn_readfirstlane(t.row0),
              rows = __builtin_amdgcn_readfirstlane(t.rows);
    if (rows <= 0) return;
    const int n0 = rt * S::kRows;

    v4f acc[FR][FT];
#pragma unroll
    for (int j = 0; j < FR; ++j)
#pragma unroll
        for (int i = 0; i < FT; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    if (expert >= 0) {
        const unsigned char* const wbase = p.w + (size_t(expert) * p.out + n0) * p.ldw;
        const int w_rows = min(S::kRows, p.out - n0);
        const v4i wrs = buffer_over(wbase, unsigned((w_rows - 1) * p.ldw + (p.in + 15) / 16 * 16));
        const v4i xrs = buffer_over(p.x, unsigned(p.x_rows) * unsigned(p.kp));
        const v4i xsrs = buffer_over(p.xs, unsigned(p.x_rows) * unsigned(p.ks));
        constexpr int kWLoads = S::kRows / 8 / S::kWaves, kXLoads = S::kToks / 8 / S::kWaves;
        constexpr int kLoads = kWLoads + kXLoads;   // of a step; one more for those that load scales
        auto w_turn = [](int r) { return (r >> 1 & 1) | (r / (4 * FR) & 3) << 1; };
        unsigned x_off[kXLoads];
        // load i of the weight brings rows 8 (wave kWLoads + i) .. + 7 of the tile; past the last row the descriptor ends, and zeros arrive
        const unsigned w_lane = unsigned(lane >> 3) * unsigned(p.ldw);
        const unsigned w_load = unsigned(8 * wave * kWLoads) * unsigned(p.ldw), w_next = 8u * unsigned(p.ldw);
        auto x_row = [&](int r) {   // of token r of the tile
            int at = row0 + min(r, rows - 1);
            if (p.index) at = p.index[at];
            return at;
        };
#pragma unroll
        for (int i = 0; i < kXLoads; ++i) {
            const int r = 8 * (wave * kXLoads + i) + (lane >> 3), at = x_row(r);
            x_off[i] = unsigned(at) < unsigned(p.x_rows) ? unsigned(at) * unsigned(p.kp) + unsigned((lane & 7) ^ (r >> 1 & 7)) * 16u : 0x80000000u;
        }
        // The scales of tokens 64 wave .. + 63, a word for four blocks: the first four wavefronts load them
        const bool s_mine = 64 * wave < S::kToks;
        const int s_at = s_mine ? x_row(64 * wave + lane) : -1;
        const unsigned s_off = unsigned(s_at) < unsigned(p.x_rows) ? unsigned(s_at) * 4u : 0x80000000u;
        const unsigned lds0 = lds_address(smem);
        const int ragged = p.in % 128;
        int q = first;   // next step to request; past the last one zeros arrive
        unsigned q_dst = lds0;
        // part `part` of `parts` of a step's loads; scales_too: in the first four wavefronts
        auto request = [&](bool scales_too, int part, int parts) __attribute__((always_inline)) {
            const unsigned none = q < last ? 0u : 0x80000000u, col = q < last ? unsigned(q) * 128u : 0u;
#pragma unroll
            for (int i = 0; i < kWLoads; ++i) {
                if (i % parts != part) continue;
                const int piece = (lane & 7) ^ w_turn(8 * (wave * kWLoads + i) + (lane >> 3));
                unsigned off = (w_lane + unsigned(piece) * 16u) | none;
                if (ragged && q == p.kb - 1 && piece * 16 >= ragged) off = 0x80000000u;   // zeros past the last column's piece
                load_to_lds(wrs, q_dst + unsigned(wave * kWLoads + i) * 1024u, off, col + w_load + unsigned(i) * w_next);
            }
#pragma unroll
            for (int i = 0; i < kXLoads; ++i) {
                if ((kWLoads + i) % parts != part) continue;
                load_to_lds(xrs, q_dst + S::kRows * 128u + unsigned(wave * kXLoads + i) * 1024u, x_off[i] | none, col);
            }
            if (scales_too && part == 0)
                load4_to_lds(xsrs, q_dst + (S::kRows + S::kToks) * 128u + unsigned(wave) * 256u, s_off | none, q < last ? unsigned(q >> 2) * unsigned(p.x_rows) * 4u : 0u);
            if (part == parts - 1) {
                ++q;
                q_dst = q_dst == lds0 + (S::kRing - 1) * S::kStep ? lds0 : q_dst + S::kStep;
            }
        };
        // fragments: a lane's row has the turn (ln / 2) % 8 in both operands
        const int wrow = wr * 16 * FR + (ln >> 2) * 4 * FR + (ln & 3), xrow = wt * 16 * FT + ln;
        const unsigned p0 = unsigned(kg ^ (ln >> 1 & 7)) * 16u;
        const unsigned w_frag = lds0 + unsigned(wrow) * 128u + p0, x_frag = lds0 + unsigned(S::kRows + xrow) * 128u + p0;
        const unsigned s_frag = lds0 + (S::kRows + S::kToks) * 128u + xrow * 4u;
        unsigned r_src = 0;   // of the step to be read next, from lds0
        auto read_piece = [&](unsigned at) __attribute__((always_inline)) { return join(read_lds<v4i>(at), read_lds<v4i>(at ^ 64u)); };   // pieces kg, kg + 4
        auto read_w = [&](int j) __attribute__((always_inline)) { return read_piece(w_frag + r_src + j * 512); };
        auto read_x = [&](int i) __attribute__((always_inline)) { return read_piece(x_frag + r_src + i * 2048); };
        auto read_s = [&](int i, int b) __attribute__((always_inline)) { return int(read_lds<unsigned char>(s_frag + r_src + i * 64 + (b & 3))); };
        // the weight's scales of 64 steps, one to a lane
        const bool s_f32 = MODE == kModeF32 || (MODE == kModeExact && p.ws_f32);
        const size_t s_row = (size_t(expert) * ((p.out + 127) / 128) + min(n0 + wr * 16 * FR, p.out - 1) / 128) * p.kb;
        int scales = 0;
        auto load_scales = [&](int b0) {
            const int b = min(b0 + lane, p.kb - 1);
            const int v = s_f32 ? static_cast<const int*>(p.ws)[s_row + b] : static_cast<const unsigned char*>(p.ws)[s_row + b];
            asm volatile("v_mov_b32 %0, %1" : "=v"(scales) : "v"(v));   // waited for here, not at every step's use
        };
        v8i w[FR], x[FT];
        int xs[FT];
        WeightScale sw{};
        auto read = [&](int b) __attribute__((always_inline)) {
            if (ragged % 16 && b == p.kb - 1 && !late) {
                // The last block ends inside a 16-byte piece, and the weight's rows may go on with anything: the wavefronts that read first clear the
                // rows that they read, which are all (the other ones come after a barrier)
                for (int r = wr * 16 * FR + lane; r < (wr + 1) * 16 * FR; r += 64) {
                    const unsigned at = lds0 + r_src + unsigned(r) * 128u + unsigned(ragged / 16 ^ w_turn(r)) * 16u;
                    for (int e = ragged % 16; e < 16; ++e) write_lds<unsigned char>(at + e, 0);
                }
                wavefront_lds_order();
            }
#pragma unroll
            for (int i = 0; i < FT; ++i) xs[i] = read_s(i, b);
#pragma unroll
            for (int j = 0; j < FR; ++j) w[j] = read_w(j);
#pragma unroll
            for (int i = 0; i < FT; ++i) x[i] = read_x(i);
            if ((b - first & 63) == 0) load_scales(b);
            sw = weight_scale(__builtin_amdgcn_readlane(scales, b - first & 63), s_f32);   // here, where the other side multiplies
            r_src = r_src == (S::kRing - 1) * S::kStep ? 0 : r_src + S::kStep;
        };
        auto products = [&](auto after) __attribute__((always_inline)) {
            __builtin_amdgcn_s_setprio(1);
            multiply_all<FR, FT, MODE>(acc, w, x, xs, sw, after);
            __builtin_amdgcn_s_setprio(0);
        };
        // A loop for each side: with branches inside, the compiler moves the products past the barriers.  kAhead: loads that may still be on their way when a
        // step has to be there, those of later ones.
        if (!late) {
            constexpr int kAhead = (S::kRing - 2) * (kLoads + 1);
#pragma unroll
            for (int i = 0; i < S::kRing; ++i) request(true, 0, 1);
            loads_barrier<kAhead + kLoads + 1>();   // step 0
            for (int b = first; b < last; ++b) {
                read(b);
                if (b > first) request(true, 0, 1);   // step b + RING - 1
                lds_barrier();
                __builtin_amdgcn_sched_barrier(0);
                products([](int) {});
                __builtin_amdgcn_sched_barrier(0);
                loads_barrier<kAhead>();   // step b + 1
            }
            lds_barrier();
        } else {
            constexpr int kAhead = (S::kRing - 2) * kLoads;
#pragma unroll
            for (int i = 0; i < S::kRing; ++i) request(false, 0, 1);
            loads_barrier<kAhead + kLoads>();   // step 0
            loads_barrier<kAhead>();            // step 1
            for (int b = first; b < last; ++b) {
                read(b);
                loads_barrier<kAhead>();   // step b + 1
                __builtin_amdgcn_sched_barrier(0);
                request(false, 0, 1);
                __builtin_amdgcn_sched_barrier(0);
                products([](int) {});
                __builtin_amdgcn_sched_barrier(0);
                lds_barrier();
            }
        }
        loads_barrier<0>();   // nothing may land in LDS any more
    }
    finish_tile<S, FR, FT, WR>(p, smem, acc, size_t(slice) * nrt * p.n_tiles + size_t(rt) * p.n_tiles + tt, n0, row0, rows);
}

// The largest tile, 256 rows x 256 tokens, eight wavefronts of 128 x 64 that take turns as in k_f8_tile.  Two buffers for a step of both operands are all that LDS
// has, and what is requested in the phase after a buffer's last read has less than two phases to arrive; all in one phase it also
// comes faster than a compute unit takes it (16 clocks a load, 64 loads a step, a phase is 1024 clocks of products).  So the operands are
// requested in turn: the weight in even phases; the tokens in odd ones, a step earlier, those that the first wavefronts read into the
// buffer that these have just read, the others' into a ring of three.
//   Up to 128 tokens the last four wavefronts have none and only load.
//   28672 x 8192, 2048 tokens: 390 us, 2.47 PFLOP/s, 8192 x 8192, 8192 tokens 408, 2.69 (replayed in a graph); the matrix cores work in 56 % of the clocks (both
// operands requested in one phase: 37 %, 460 us), of which there are then 2.1 in a nanosecond and not 2.35: power is the bound.  Without the loads it takes 279 us, without the
// products 290.  fp32 scales of the weight: 511 us.  They add four multiply-adds to a matrix instruction, whose
// product goes into zeros.
constexpr unsigned kBigW = 32768, kBigX = 16384, kBigS = 1024;                                          // bytes of a buffer
constexpr unsigned kBigEarly = 2 * kBigW, kBigLate = kBigEarly + 2 * kBigX, kBigScales = kBigLate + 3 * kBigX;
struct F8BigShape {
    static constexpr int kWaves = 8, kRows = 256, kToks = 256, kSize = 2, kOutLd = kRows * kSize + 16;
    static constexpr int kLds = int(kBigScales + 3 * kBigS);
    static_assert(kLds <= 163840 && kToks * kOutLd <= kLds, "the output tile reuses the buffers");
};
template <int MODE>
__global__ __launch_bounds__(512, 2) void k_f8_tile256(F8Params p) {
    constexpr int FR = 8, FT = 4, WR = 2;
    typedef F8BigShape S;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), side_wave = wave & 3;
    const int wr = wave % WR;
    const bool late = wave >= 4;
    const int ln = lane & 15, kg = lane >> 4;
    const int nrt = (p.out + 255) / 256;
    int rt, tt, slice;
    if (!tile_of(p, nrt, p.tiles ? 8 : 4, rt, tt, slice)) return;
    const int first = slice * p.slice_blocks, last = min(first + p.slice_blocks, p.kb);   // blocks of columns
    F8Tile t = {0, tt * 256, min(256, p.rows - tt * 256), 0};
    if (p.tiles) t = p.tiles[tt];
    const int expert = __builtin_amdgcn_readfirstlane(t.expert), row0 = __builtin_amdgcn_readfirstlane(t.row0),
              rows = __builtin_amdgcn_readfirstlane(t.rows);
    if (rows <= 0) return;
    const int n0 = rt * 256;

    v4f acc[FR][FT];
#pragma unroll
    for (int j = 0; j < FR; ++j)
#pragma unroll
        for (int i = 0; i < FT; ++i) acc[j][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    if (expert >= 0) {
        const unsigned char* const wbase = p.w + (size_t(expert) * p.out + n0) * p.ldw;
        const int w_rows = min(256, p.out - n0);
        const v4i wrs = buffer_over(wbase, unsigned((w_rows - 1) * p.ldw + (p.in + 15) / 16 * 16));
        const v4i xrs = buffer_over(p.x, p.x_bytes);
        const v4i xsrs = buffer_over(p.xs, unsigned(p.x_rows) * unsigned(p.ks));
        const unsigned lds0 = lds_address(smem);
        const int ragged = p.in % 128;
        auto x_row = [&](int r) {   // of token r of the tile
            int at = row0 + min(r, rows - 1);
            if (p.index) at = p.index[at];
            return at;
        };
        // Load i of the weight brings rows 32 wave + 8 i .. + 7 of the tile, of the tokens as many; past the last row of the weight the descriptor ends, and
        // zeros arrive.  Turns of the 16-byte pieces as in k_f8_tile; the weight's, (row / 2 % 2) + row / 32 % 4 * 2, is the same for a wavefront's loads.
        const int w_piece = (lane & 7) ^ ((lane >> 4 & 1) | (wave & 3) << 1);
        const unsigned w_lane = unsigned(lane >> 3) * unsigned(p.ldw) + unsigned(w_piece) * 16u, w_load = unsigned(32 * wave) * unsigned(p.ldw);
        const unsigned w_tail = ragged && w_piece * 16 >= ragged ? 0x80000000u : w_lane;   // in the last block: zeros past the last column's piece
        unsigned x_off[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 32 * wave + 8 * i + (lane >> 3), at = x_row(r);
            x_off[i] = unsigned(at) < unsigned(p.x_rows) ? unsigned(at) * unsigned(p.kp) + unsigned((lane & 7) ^ (r >> 1 & 7)) * 16u : 0x80000000u;
        }
        // the scales of tokens 64 wave .. + 63, a word for four blocks: the first four wavefronts load them
        const int s_at = late ? -1 : x_row(64 * wave + lane);
        const unsigned s_off = unsigned(s_at) < unsigned(p.x_rows) ? unsigned(s_at) * 4u : 0x80000000u;
        int qw = first, qx = first;   // next steps to request; past the last one zeros arrive
        unsigned w_dst = lds0 + unsigned(wave) * 4096u, x_dst = lds0 + (late ? kBigLate : kBigEarly) + unsigned(side_wave) * 4096u, s_dst = lds0 + kBigScales + unsigned(side_wave) * 256u;
        const unsigned x_end = x_dst + (late ? 3 : 2) * kBigX, s_end = s_dst + 3 * kBigS;
        auto request_w = [&](int i) __attribute__((always_inline)) {
            const bool in = qw < last;
            const unsigned off = !in ? 0x80000000u : qw == p.kb - 1 ? w_tail : w_lane;
            load_to_lds(wrs, w_dst + unsigned(i) * 1024u, off, (in ? unsigned(qw) * 128u : 0u) + w_load + unsigned(i) * 8u * unsigned(p.ldw));
            if (i == 3) {
                ++qw;
                w_dst = w_dst < lds0 + kBigW ? w_dst + kBigW : w_dst - kBigW;
            }
        };
        auto request_x = [&](int i, bool early_wave) __attribute__((always_inline)) {
            const bool in = qx < last;
            const unsigned none = in ? 0u : 0x80000000u;
            load_to_lds(xrs, x_dst + unsigned(i) * 1024u, x_off[i] | none, in ? unsigned(qx) * 128u : 0u);
            if (i < 3) return;
            if (early_wave) load4_to_lds(xsrs, s_dst, s_off | none, in ? unsigned(qx >> 2) * unsigned(p.x_rows) * 4u : 0u);
            ++qx;
            x_dst = x_dst + kBigX == x_end ? x_end - (early_wave ? 2 : 3) * kBigX : x_dst + kBigX;
            s_dst = s_dst + kBigS == s_end ? s_end - 3 * kBigS : s_dst + kBigS;
        };
        // fragments: a lane's row has the turn (ln / 2) % 8 in both operands
        const int wrow = wr * 128 + (ln >> 2) * 32 + (ln & 3), xrow = (side_wave >> 1) * 64 + ln;   // of the side's tokens
        const unsigned p0 = unsigned(kg ^ (ln >> 1 & 7)) * 16u;
        unsigned w_src = lds0 + unsigned(wrow) * 128u + p0, x_src = lds0 + (late ? kBigLate : kBigEarly) + unsigned(xrow) * 128u + p0;
        unsigned s_src = lds0 + kBigScales + unsigned((late ? 128 : 0) + xrow) * 4u;
        const unsigned x_wrap = x_src + (late ? 2 : 1) * kBigX, s_wrap = s_src + 2 * kBigS;
        const unsigned w_clear = lds0 + unsigned(wr * 128) * 128u;
        auto read_piece = [&](unsigned at) __attribute__((always_inline)) { return join(read_lds<v4i>(at), read_lds<v4i>(at ^ 64u)); };   // pieces kg, kg + 4
        // the weight's scales of 64 steps, one to a lane
        const size_t s_row = (size_t(expert) * ((p.out + 127) / 128) + min(n0 + wr * 128, p.out - 1) / 128) * p.kb;
        int scales = 0;
        auto load_scales = [&](int b0) {
            const int b = min(b0 + lane, p.kb - 1);
            const int v = MODE == kModeF32 ? static_cast<const int*>(p.ws)[s_row + b] : static_cast<const unsigned char*>(p.ws)[s_row + b];
            asm volatile("v_mov_b32 %0, %1" : "=v"(scales) : "v"(v));   // waited for here, not at every step's use
        };
        v8i w[FR], x[FT];
        int xs[FT];
        WeightScale sw{};
        auto read = [&](int b, bool early_wave) __attribute__((always_inline)) {
            if (early_wave && ragged % 16 && b == p.kb - 1) {
                // the last block ends inside a 16-byte piece: cleared by those that read first, as in k_f8_tile
                for (int r = lane; r < 128; r += 64) {
                    const unsigned at = w_clear + ((b - first) & 1 ? kBigW : 0u) + unsigned(r) * 128u + unsigned(ragged / 16 ^ ((r >> 1 & 1) | (r >> 5 & 3) << 1)) * 16u;
                    for (int e = ragged % 16; e < 16; ++e) write_lds<unsigned char>(at + e, 0);
                }
                wavefront_lds_order();
            }
#pragma unroll
            for (int i = 0; i < FT; ++i) xs[i] = int(read_lds<unsigned char>(s_src + i * 64 + (b & 3)));
#pragma unroll
            for (int j = 0; j < FR; ++j) w[j] = read_piece(w_src + j * 512);
#pragma unroll
            for (int i = 0; i < FT; ++i) x[i] = read_piece(x_src + i * 2048);
            if ((b - first & 63) == 0) load_scales(b);
            sw = weight_scale(__builtin_amdgcn_readlane(scales, b - first & 63), MODE == kModeF32);
            w_src = (b - first) & 1 ? w_src - kBigW : w_src + kBigW;
            x_src = x_src == x_wrap ? x_wrap - (early_wave ? 1 : 2) * kBigX : x_src + kBigX;
            s_src = s_src == s_wrap ? s_wrap - 2 * kBigS : s_src + kBigS;
        };
        auto products = [&](auto after) __attribute__((always_inline)) {
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            multiply_all<FR, FT, MODE>(acc, w, x, xs, sw, [&](int i) __attribute__((always_inline)) {
                __builtin_amdgcn_sched_barrier(0);
                after(i);
                __builtin_amdgcn_sched_barrier(0);
            });
            __builtin_amdgcn_s_setprio(0);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto begin = [&](bool early_wave) __attribute__((always_inline)) {   // two steps
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 4; ++i) request_w(i);
#pragma unroll
                for (int i = 0; i < 4; ++i) request_x(i, early_wave);
            }
        };
        // (a loop for each side: with branches inside, the compiler moves the products past the barriers)
        if (!late) {
            constexpr int kX = 5;   // loads of a step's tokens and scales
            begin(true);
            loads_barrier<4 + kX>();   // the first step
            for (int b = first; b < last; ++b) {
                read(b, true);
                if (b > first) {   // the weight of step b + 1
#pragma unroll
                    for (int i = 0; i < 4; ++i) request_w(i);
                }
                lds_barrier();
                products([&](int i) __attribute__((always_inline)) { request_x(i, true); });   // the tokens of step b + 2
                loads_barrier<kX>();                                                           // step b + 1
            }
            lds_barrier();
        } else if (rows > 128) {
            constexpr int kX = 4;
            begin(false);
            loads_barrier<4 + kX>();
            lds_barrier();
            for (int b = first; b < last; ++b) {
                read(b, false);
#pragma unroll
                for (int i = 0; i < 4; ++i) request_x(i, false);   // the tokens of step b + 2
                loads_barrier<kX>();                               // step b + 1
                products([&](int i) __attribute__((always_inline)) { request_w(i); });   // the weight of step b + 2
                lds_barrier();
            }
        } else {   // no tokens here
#pragma unroll
            for (int i = 0; i < 8; ++i) request_w(i & 3);
            loads_barrier<4>();
            lds_barrier();
            for (int b = first; b < last; ++b) {
                loads_barrier<0>();   // step b + 1
#pragma unroll
                for (int i = 0; i < 4; ++i) request_w(i);   // step b + 2
                lds_barrier();
            }
        }
        loads_barrier<0>();   // nothing may land in LDS any more
    }
    finish_tile<S, FR, FT, WR>(p, smem, acc, size_t(slice) * nrt * p.n_tiles + size_t(rt) * p.n_tiles + tt, n0, row0, rows);
}

// y from the partial sums of p.slices column slices, added up in order: a wavefront takes what one of k_f8_tile's held of a tile, FR fragments
// of 4 rows a lane at a time, which are 4 FR neighbouring outputs of a token.  Bound by memory and the launch: five slices of 300 x 4096, 25 MB, 6.8 us.
template <int FR, int FT, int WR, int WT>
__global__ __launch_bounds__(256) void k_f8_join(F8Params p) {
    const int lane = threadIdx.x & 63, ln = lane & 15, kg = lane >> 4;
    const unsigned unit = blockIdx.x * 4 + (threadIdx.x >> 6);   // tile, wavefront of it, fragment of the activations
    const int nrt = (p.out + 16 * FR * WR - 1) / (16 * FR * WR);
    const unsigned tiles = unsigned(nrt) * unsigned(p.n_tiles);
    const int i = unit % FT, wave = unit / FT % 8;
    const unsigned tile = unit / (FT * 8);
    if (tile >= tiles) return;
    const int rt = int(tile / p.n_tiles), tt = int(tile % p.n_tiles);
    constexpr int kToks = 16 * FT * WT;
    F8Tile t = {0, tt * kToks, min(kToks, p.rows - tt * kToks), 0};
    if (p.tiles) t = p.tiles[tt];
    const int tok = wave / WR * 16 * FT + 16 * i + ln, n = rt * 16 * FR * WR + wave % WR * 16 * FR + kg * 4 * FR;
    if (tok >= t.rows) return;
    const v4f* from = reinterpret_cast<const v4f*>(p.part) + (size_t(tile) * 8 + wave) * (FR * FT * 64) + i * 64 + lane;
    v4f sum[FR];
#pragma unroll
    for (int j = 0; j < FR; ++j) sum[j] = from[j * FT * 64];
    for (int s = 1; s < p.slices; ++s) {
        from += size_t(tiles) * 8 * (FR * FT * 64);
#pragma unroll
        for (int j = 0; j < FR; ++j) sum[j] += from[j * FT * 64];
    }
#pragma unroll
    for (int j = 0; j < FR; ++j) store4(p, t.row0 + tok, n + 4 * j, sum[j]);
}

static hipError_t allow_lds(const void* kernel, std::atomic<bool>& done, int bytes) {   // (doing it twice is harmless)
    if (done) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done = true;
    return e;
}
static unsigned tile_grid(const F8Params& p, int tile_rows) {
    return 8 * ((unsigned((p.out + tile_rows - 1) / tile_rows) * unsigned(p.n_tiles) * unsigned(p.slices) + 7) / 8);
}
template <int FR, int FT, int WR, int WT>
static hipError_t join(const F8Params& p, hipStream_t st) {
    if (p.slices > 1) {
        const size_t units = size_t((p.out + 16 * FR * WR - 1) / (16 * FR * WR)) * p.n_tiles * 8 * FT;
        hipLaunchKernelGGL((k_f8_join<FR, FT, WR, WT>), dim3(unsigned((units + 3) / 4)), dim3(256), 0, st, p);
    }
    return hipGetLastError();
}
template <int FR, int FT, int WR, int WT, int MODE>
static hipError_t tiles(const F8Params& p, hipStream_t st) {
    typedef F8TileShape<FR, FT, WR, WT, MODE> S;
    static std::atomic<bool> done{false};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&k_f8_tile<FR, FT, WR, WT, MODE>), done, S::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_f8_tile<FR, FT, WR, WT, MODE>), dim3(tile_grid(p, S::kRows)), dim3(512), S::kLds, st, p);
    return join<FR, FT, WR, WT>(p, st);
}
template <int MODE>
static hipError_t tiles256(const F8Params& p, hipStream_t st) {
    static std::atomic<bool> done{false};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&k_f8_tile256<MODE>), done, F8BigShape::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_f8_tile256<MODE>), dim3(tile_grid(p, 256)), dim3(512), F8BigShape::kLds, st, p);
    return join<8, 4, 2, 4>(p, st);
}

template <int FR, int FT, int DEPTH, int MODE, int T>
static void slices_as(const F8Params& p, hipStream_t st) {
    hipLaunchKernelGGL((k_f8_slices<FR, FT, DEPTH, MODE, T>), dim3(tile_grid(p, 16 * FR)), dim3(512), 0, st, p);
}
template <int FR, int FT, int DEPTH, int T>
static hipError_t slices_of(const F8Params& p, hipStream_t st) {
    if (p.y_dtype == BITSTACK_T_F32) slices_as<FR, FT, DEPTH, kModeExact, T>(p, st);
    else if (p.ws_f32) slices_as<FR, FT, DEPTH, kModeF32, T>(p, st);
    else slices_as<FR, FT, DEPTH, kModeE8M0, T>(p, st);
    return hipGetLastError();
}
template <int FR, int FT, int DEPTH>
static hipError_t slices(const F8Params& p, hipStream_t st) {
    if constexpr (FT == 1) {
        if (p.x_dtype == BITSTACK_T_F16) return slices_of<FR, FT, DEPTH, BITSTACK_T_F16>(p, st);
        if (p.x_dtype == BITSTACK_T_BF16) return slices_of<FR, FT, DEPTH, BITSTACK_T_BF16>(p, st);
    }
    return slices_of<FR, FT, DEPTH, BITSTACK_T_F8>(p, st);
}

// Kernels by their tile (rows of the weight x of y): 16 x 16, 64 x 16, 64 x 32, 64 x 64 without LDS, 128 x 64, 128 x 128, 256 x 128, 256 x 256
enum F8Kernel { kSlices16 = 16, kSlices16Wide = 17, kSlices32 = 32, kSlices64 = 64, kTile64 = 65, kTile128 = 128, kTile128Wide = 129, kTile256 = 256 };
struct F8KernelShape {
    int kernel, rows, toks;
};
constexpr F8KernelShape kShapes[] = {{kSlices16, 16, 16}, {kSlices16Wide, 64, 16}, {kSlices32, 64, 32}, {kSlices64, 64, 64}, {kTile64, 128, 64}, {kTile128, 128, 128}, {kTile128Wide, 256, 128}, {kTile256, 256, 256}};

static std::atomic<int> g_forced{0};   // measurement hook: kernel + 1024 * column slices, 0 = the choice below
bool f8_force_kernel(int kernel) {
    bool known = kernel == 0;
    for (const F8KernelShape& k : kShapes) known |= kernel % 1024 == k.kernel && (kernel < 1024 || k.kernel > kSlices64);
    if (known) g_forced = kernel;
    return known;
}
static bool makes(const F8KernelShape& k, bool exact) {
    if (exact) return k.kernel < kTile128Wide;   // the operands as fp16 leave no registers for the larger tiles' sums
    // 1851 x 384 x 2048 in fp32: 14.3 us, 128 x 64 16.2; in 16 bits, where that has half the work, it is faster: 1920 x 272 x 1024 9.4, 7.9
    return k.kernel != kSlices64;
}

// Duration in microseconds.  The constants were fitted to timings of every kernel on 88 products (1 to 3660 rows, 256 to 28672 x 512 to 14336, up to 64
// experts, all types): what they choose is 1.2 to 1.4 % slower than the fastest, in the mean of two runs, 16 % at most
// (profiles/f8_kernel_choice.txt).
static double f8_time_us(const F8KernelShape& k, int slices, int rows, int out, int kb, int experts, bool grouped, bool exact, bool ws_f32) {
    // tiles of y's rows that have any: a group fills its last one by half, in the mean
    const int groups = grouped ? std::min(rows, experts) : 1;
    const double mt = grouped ? std::max<double>(groups, double(rows) / k.toks + 0.5 * groups) : (rows + k.toks - 1) / k.toks;
    const double tiles = mt * ((out + k.rows - 1) / k.rows), rounds = tiles * slices / 256;
    // the weights once, from memory, at the rate that a kernel was found to take them at most
    const double stream = 4.0 + double(groups) * out * kb * 128 / (k.kernel == kSlices64 ? 2.7e6 : 5.4e6);
    const double passes = (kb + 7) / 8, steps = (kb + slices - 1) / slices;
    double us = 4.15;
    switch (k.kernel) {
        case kSlices16: {   // up to four workgroups on a compute unit
            const double whole = std::floor(rounds / 4), rest = rounds - 4 * whole;
            us = 3.5 + passes * (whole * 4.46 + (rest > 0 ? 0.14 + 1.15 * rest : 0.0));
            break;
        }
        case kSlices16Wide: us = 4.0 + passes * std::max(1.93, 0.9 + (exact ? 3.08 : 2.48) * rounds); break;   // two
        case kSlices32: us = 4.0 + passes * std::max(2.3, 0.9 + (exact ? 3.86 : 3.08) * rounds); break;
        case kSlices64: us = 4.0 + passes * std::ceil(rounds) * 4.47; break;
        case kTile64: {   // two, which take less than twice as long as one
            const double one = exact ? 0.88 : 0.542, two = exact ? 1.47 : 0.905, whole = std::floor(rounds / 2), rest = rounds - 2 * whole;
            us += steps * (whole * two + (rest > 1 ? two : rest > 0 ? one : 0.0));
            break;
        }
        case kTile128: us += steps * std::ceil(rounds) * (exact ? 1.46 : 0.78); break;
        case kTile128Wide: us += steps * std::ceil(rounds) * 1.08; break;
        default: us += steps * std::ceil(rounds) * (ws_f32 ? 1.87 : 1.61);
    }
    return std::max(us, stream) + (slices > 1 ? 4.0 + slices * tiles * k.rows * k.toks * 8 / 6.3e6 : 0.0);
}

// Kernel and column slices of a product, from sizes alone, and from the room for the partial sums where that is too small for the fastest
F8Plan f8_plan(int rows, int out, int in, int experts, bool grouped, bool exact, bool ws_f32, size_t room) {
    const int forced = g_forced.load(), kb = (in + 127) / 128;
    auto plan_of = [&](const F8KernelShape& k, int slices) {
        const int each = (kb + slices - 1) / slices;
        F8Plan plan{k.kernel, (kb + each - 1) / each, k.toks, 0, 0, 0};   // none of the slices empty
        // every group's rows, rounded up to tiles, and those of the rows past the last group
        plan.n_tiles = grouped ? rows / k.toks + 1 + std::min(rows, experts) : (rows + k.toks - 1) / k.toks;
        const size_t tiles = size_t((out + k.rows - 1) / k.rows) * plan.n_tiles;
        plan.tiles = int(std::min<size_t>(tiles, 0x7fffffff));
        if (plan.slices > 1) plan.part_bytes = plan.slices * tiles * (k.rows * k.toks * 4);
        return plan;
    };
    auto fits = [&](const F8Plan& plan) { return plan.slices == 1 || (grouped ? plan.n_tiles * sizeof(F8Tile) + 256 : 0) + plan.part_bytes <= room; };
    for (const F8KernelShape& k : kShapes)
        if (forced && k.kernel == forced % 1024 && makes(k, exact)) return plan_of(k, std::max(1, std::min(forced / 1024, kb)));
    F8Plan plan = plan_of(kShapes[0], 1);
    double best = 1e30;
    for (const F8KernelShape& k : kShapes) {
        if (rows <= 16 && k.toks > 16) break;   // never faster
        if (!makes(k, exact)) continue;
        for (int slices : {1, 2, 3, 4, 5, 6, 7, 8, 12, 16}) {
            if (slices > 1 && (k.kernel <= kSlices64 || slices > kb / 4)) continue;
            const double us = f8_time_us(k, slices, rows, out, kb, experts, grouped, exact, ws_f32);
            if (us >= best) continue;
            const F8Plan this_one = plan_of(k, slices);
            if (!f8_launchable(this_one) || !fits(this_one)) continue;
            best = us;
            plan = this_one;
        }
    }
    return plan;
}
hipError_t launch_f8_product(const F8Params& args, const F8Plan& plan, hipStream_t st) {
    F8Params p = args;
    p.slices = plan.slices;
    p.slice_blocks = (p.kb + plan.slices - 1) / plan.slices;
    p.n_tiles = plan.n_tiles;
    const bool exact = p.y_dtype == BITSTACK_T_F32;
    switch (plan.kernel) {
        case kSlices16: return slices<1, 1, 2>(p, st);
        case kSlices16Wide: return slices<4, 1, 1>(p, st);
        case kSlices32: return slices<4, 2, 1>(p, st);
        case kSlices64:
            slices_as<4, 4, 1, kModeExact, BITSTACK_T_F8>(p, st);
            return hipGetLastError();
        case kTile64:
            if (exact) return tiles<2, 2, 4, 2, kModeExact>(p, st);
            return p.ws_f32 ? tiles<2, 2, 4, 2, kModeF32>(p, st) : tiles<2, 2, 4, 2, kModeE8M0>(p, st);
        case kTile128:
            if (exact) return tiles<2, 4, 4, 2, kModeExact>(p, st);
            return p.ws_f32 ? tiles<2, 4, 4, 2, kModeF32>(p, st) : tiles<2, 4, 4, 2, kModeE8M0>(p, st);
        case kTile128Wide:
            return p.ws_f32 ? tiles<4, 4, 4, 2, kModeF32>(p, st) : tiles<4, 4, 4, 2, kModeE8M0>(p, st);
        default: return p.ws_f32 ? tiles256<kModeF32>(p, st) : tiles256<kModeE8M0>(p, st);
    }
}

}  // namespace bitstack
