// Activations and weights into 8-bit floating point (e4m3), one power-of-two scale for each 128 columns of a row, or for each
// block of 128 x 128:
//
//     s = 2^e, e = the least with max |v| <= 448 * 2^e, at least -126;   q = v / s rounded to nearest even
//
// With a power of two the quotient is exact, so that the rounding to e4m3 is the only one.
#include <hip/hip_runtime.h>

#include "f8.h"

namespace bitstack {

// Inclusive scan of v[0 .. n) in LDS by a workgroup of 256, op associative
template <class OP>
__device__ __forceinline__ void scan256(int* v, int n, OP op) {
    __shared__ int part[256];
    const int i = threadIdx.x, each = (n + 255) / 256, first = i * each, last = min(first + each, n);
    for (int k = first + 1; k < last; ++k) v[k] = op(v[k - 1], v[k]);
    part[i] = first < last ? v[last - 1] : v[n - 1];
    __syncthreads();
    const int parts = (n + each - 1) / each;
    for (int d = 1; d < parts; d <<= 1) {
        const int mine = i >= d ? op(part[i - d], part[i]) : part[i];
        __syncthreads();
        part[i] = mine;
        __syncthreads();
    }
    if (i > 0)
        for (int k = first; k < last; ++k) v[k] = op(part[i - 1], v[k]);
    __syncthreads();
}

// The tiles of the groups, by a workgroup of 256: group e has the rows [end[e - 1], end[e]), cut into pieces of tile_rows; the rows past the last group
// are one more group, of zeros.  Offsets that fall, or pass the last row, are held to the rows there are.
__device__ void make_work_list(const F8WorkList& l) {
    __shared__ int end[kMaxExperts + 1], upto[kMaxExperts + 1];
    const int i = threadIdx.x;
    for (int e = i; e < l.experts; e += 256) end[e] = min(max(l.offsets[e + 1], 0), l.rows);
    __syncthreads();
    scan256(end, l.experts, [](int a, int b) { return max(a, b); });
    if (i == 0) end[l.experts] = l.rows;
    __syncthreads();
    for (int e = i; e <= l.experts; e += 256) upto[e] = (end[e] - (e ? end[e - 1] : 0) + l.tile_rows - 1) / l.tile_rows;
    __syncthreads();
    scan256(upto, l.experts + 1, [](int a, int b) { return a + b; });
    for (int t = i; t < l.n_tiles; t += 256) {
        int lo = 0, hi = l.experts + 1;   // the first group with upto > t
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (upto[mid] > t) hi = mid;
            else lo = mid + 1;
        }
        F8Tile tile = {-1, 0, 0, upto[l.experts]};
        if (lo <= l.experts) {
            const int first = (lo ? end[lo - 1] : 0) + (t - (lo ? upto[lo - 1] : 0)) * l.tile_rows;
            tile = {lo < l.experts ? lo : -1, first, min(l.tile_rows, end[lo] - first), upto[l.experts]};
        }
        l.tiles[t] = tile;
    }
}

// Sixteen lanes bring a block of 128 columns to 8 bits, eight columns each: a wavefront has four blocks of a row, whose scales are one word, WORDS
// times over.  Bound by memory: x is read once and q written once, 16 and 8 bytes a lane and word: 2048 x 8192 in fp16, from memory, 12.9 us, 3.9 TB/s.  Gated rows
// have the gate's instructions beside that (f8_gate: 16 and two of a quarter of the rate): 2048 of 2 x 14336 41.7 us, 3.5 TB/s, 37.2 with six and two.  The first
// workgroup makes the work list where there is one: a launch less.
template <int T, bool GATED, int WORDS>
__global__ __launch_bounds__(256) void k_f8_quantise(const typename Elem<T>::type* x, size_t ld, int rows, int in, unsigned char* q,
                                                     unsigned* s, int kp, F8WorkList list) {
    if (list.offsets && blockIdx.x == 0) {
        make_work_list(list);
        return;
    }
    const int lane = threadIdx.x & 63;
    const int per_row = (kp + 512 * WORDS - 1) / (512 * WORDS);   // wavefronts
    const size_t wave = (size_t(blockIdx.x - (list.offsets ? 1 : 0)) * 256 + threadIdx.x) >> 6;
    const int row = int(wave / per_row), word0 = int(wave % per_row) * WORDS;
    if (row >= rows) return;
    float v[WORDS][8], u[GATED ? WORDS : 1][8];
#pragma unroll
    for (int k = 0; k < WORDS; ++k) {   // all requests first
        const int col = (word0 + k) * 512 + lane * 8;
        const typename Elem<T>::type* const from = x + size_t(row) * ld + col;
        load_elems<T, 8>(from, in - col, v[k]);
        if constexpr (GATED) load_elems<T, 8>(from + in, in - col, u[k]);
    }
#pragma unroll
    for (int k = 0; k < WORDS; ++k) {
        const int word = word0 + k, col = word * 512 + lane * 8;
        if (word * 512 >= kp) break;
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (GATED) v[k][i] = f8_gate(v[k][i], u[k][i]);
            m = max(m, f8_magnitude(v[k][i]));
        }
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) m = max(m, unsigned(__shfl_xor(int(m), d, 16)));
        const bool bad = m >= 0x7f800000u;   // a NaN or an infinity in the block: NaN
        const int e = bad ? 127 : f8_exponent(__uint_as_float(m));
        const float r = f8_inverse(e);
        const uint2 bytes = bad ? make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu)
                                : make_uint2(f8_x4(v[k][0] * r, v[k][1] * r, v[k][2] * r, v[k][3] * r), f8_x4(v[k][4] * r, v[k][5] * r, v[k][6] * r, v[k][7] * r));
        if (col < kp) *reinterpret_cast<uint2*>(q + size_t(row) * kp + col) = bytes;
        const unsigned four = unsigned(__builtin_amdgcn_readlane(e, 0)) | unsigned(__builtin_amdgcn_readlane(e, 16)) << 8 |
                              unsigned(__builtin_amdgcn_readlane(e, 32)) << 16 | unsigned(__builtin_amdgcn_readlane(e, 48)) << 24;
        if (lane == 0) s[size_t(word) * rows + row] = four;
    }
}

// A workgroup brings a block of 128 rows x 128 columns to 8 bits: sixteen lanes a row, sixteen rows a pass, the values in registers between
// the maximum and the rounding, so that w is read once.  Bound by memory: 28672 x 8192 in fp16 132 us, 5.4 TB/s.
template <int T>
__global__ __launch_bounds__(256) void k_f8_quantise_weight(const typename Elem<T>::type* w, size_t ld, int out, int in,
                                                            unsigned char* q, size_t ld_q, int q_cols, unsigned char* s, int kb) {
    __shared__ unsigned most[4];
    const int kblock = blockIdx.x % kb, nblock = blockIdx.x / kb;
    const int col = kblock * kF8Block + (threadIdx.x & 15) * 8;
    float v[8][8];
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = nblock * kF8Block + i * 16 + (threadIdx.x >> 4);
        load_elems<T, 8>(w + size_t(row) * ld + col, row < out ? in - col : 0, v[i]);
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, f8_magnitude(v[i][k]));
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = max(m, unsigned(__shfl_xor(int(m), d)));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(most[0], most[1]), max(most[2], most[3]));
    const bool bad = m >= 0x7f800000u;
    const int e = bad ? 127 : f8_exponent(__uint_as_float(m));
    const float r = f8_inverse(e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = nblock * kF8Block + i * 16 + (threadIdx.x >> 4);
        if (row >= out || col >= q_cols) continue;
        const uint2 bytes = bad ? make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu)
                                : make_uint2(f8_x4(v[i][0] * r, v[i][1] * r, v[i][2] * r, v[i][3] * r),
                                             f8_x4(v[i][4] * r, v[i][5] * r, v[i][6] * r, v[i][7] * r));
        *reinterpret_cast<uint2*>(q + size_t(row) * ld_q + col) = bytes;
    }
    if (threadIdx.x == 0) s[size_t(nblock) * kb + kblock] = (unsigned char)e;
}

template <int T>
static void quantise(const void* x, size_t ld, int rows, int in, bool gated, unsigned char* q, unsigned char* s, const F8WorkList& list, hipStream_t st) {
    typedef typename Elem<T>::type E;
    const int kp = (in + 127) / 128 * 128;
    unsigned* const words = reinterpret_cast<unsigned*>(s);
    // Gated rows, whose arithmetic hides no latency: four words a wavefront where that leaves enough wavefronts
    const int each = gated && size_t(rows) * ((kp + 2047) / 2048) >= 4096 ? 4 : 1;
    const size_t waves = size_t(rows) * ((kp + 512 * each - 1) / (512 * each));
    const unsigned grid = unsigned((waves + 3) / 4) + (list.offsets ? 1 : 0);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, static_cast<const E*>(x), ld, rows, in, q, words, kp, list); };
    if (gated) each == 4 ? go(&k_f8_quantise<T, true, 4>) : go(&k_f8_quantise<T, true, 1>);
    else go(&k_f8_quantise<T, false, 1>);
}

hipError_t launch_f8_quantise(const void* x, int dtype, size_t ld, int rows, int in, bool gated, unsigned char* q, unsigned char* s,
                              const F8WorkList& list, hipStream_t st) {
    if (dtype == BITSTACK_T_F16) quantise<BITSTACK_T_F16>(x, ld, rows, in, gated, q, s, list, st);
    else if (dtype == BITSTACK_T_BF16) quantise<BITSTACK_T_BF16>(x, ld, rows, in, gated, q, s, list, st);
    else quantise<BITSTACK_T_F32>(x, ld, rows, in, gated, q, s, list, st);
    return hipGetLastError();
}

template <int T>
static void quantise_weight(const void* w, size_t ld, int out, int in, unsigned char* q, size_t ld_q, unsigned char* s, hipStream_t st) {
    typedef typename Elem<T>::type E;
    const int kb = (in + 127) / 128, nb = (out + 127) / 128;
    const int q_cols = int(ld_q < size_t(kb) * 128 ? ld_q : size_t(kb) * 128);   // written: what lies past `in` as zero
    hipLaunchKernelGGL((k_f8_quantise_weight<T>), dim3(unsigned(size_t(kb) * nb)), dim3(256), 0, st, static_cast<const E*>(w), ld, out, in,
                       q, ld_q, q_cols, s, kb);
}

hipError_t launch_f8_quantise_weight(const void* w, int dtype, size_t ld, int out, int in, unsigned char* q, size_t ld_q,
                                     unsigned char* s, hipStream_t st) {
    if (dtype == BITSTACK_T_F16) quantise_weight<BITSTACK_T_F16>(w, ld, out, in, q, ld_q, s, st);
    else if (dtype == BITSTACK_T_BF16) quantise_weight<BITSTACK_T_BF16>(w, ld, out, in, q, ld_q, s, st);
    else quantise_weight<BITSTACK_T_F32>(w, ld, out, in, q, ld_q, s, st);
    return hipGetLastError();
}

}  // namespace bitstack
