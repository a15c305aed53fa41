// Around the products grouped by expert (f8_product.h): which experts a token goes to and where its rows lie, and the
// weighted sums of a token's rows.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "f8.h"
#include "route.h"

namespace bitstack {

// inclusive scan of v[0 .. n) in LDS by the whole workgroup (n <= blockDim.x), OP associative
template <class OP>
__device__ __forceinline__ void scan_lds(int* v, int n, OP op) {
    const int i = threadIdx.x;
    for (int d = 1; d < n; d <<= 1) {
        const int mine = i < n ? (i >= d ? op(v[i - d], v[i]) : v[i]) : 0;
        __syncthreads();
        if (i < n) v[i] = mine;
        __syncthreads();
    }
}

// ---- routing.  Tokens are cut into chunks, one workgroup each, worked through 64 tokens at a time.  k_route_choose takes the top_k of every
// token, a wavefront a token, and counts a chunk's rows by expert; k_route_place adds up the counts before its own chunk and ranks its
// rows.  Ranks are counted with ballots, in order, so the places do not depend on the order in which anything runs.  One chunk: one launch.
//   A choice is a maximum over the wavefront (six dependent row operations) and a ballot, top_k of them in a chain for each token; four tokens to a
// wavefront, whose logits are under way together.  57 tokens, 8 experts: 6.3 us, bound by that chain.  16384 tokens, 8 of 128 experts: 13.8 and 8.2 us, of which reading
// the logits would be 1; 16 wavefronts on every compute unit choose for 64 tokens at a time, with 271 vector instructions a token, whose issue takes
// 58 % of k_route_choose's clocks; in k_route_place it is 40 %.
constexpr int kRouteStep = 64, kRouteChunks = 256;
__host__ __device__ inline int route_steps(int tokens) { return tokens / kRouteStep + (tokens % kRouteStep ? 1 : 0); }   // any number of tokens

// A token's keys, NL to a lane
template <int T, int NL>
__device__ __forceinline__ void load_keys(const RouteParams& p, int token, int lane, unsigned (&key)[NL]) {
    const typename Elem<T>::type* const l = static_cast<const typename Elem<T>::type*>(p.logits) + size_t(token) * p.ld;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int e = i * 64 + lane;
        key[i] = e < p.experts ? route_key(float(l[e])) : 0;
    }
}

struct RouteLds {
    int base[kMaxExperts];                     // where an expert's rows of this step begin
    int count[kMaxExperts];
    short chosen[kRouteStep * kMaxTopK];
    unsigned short before[];                   // [top_k][experts]: an expert's rows in the 64-entry groups before
};

template <int T, int NL>
__device__ __forceinline__ void choose_step(const RouteParams& p, RouteLds& s, int token0) {
    // four tokens a wavefront; their logits are requested together where registers allow
    constexpr int kEach = kRouteStep / 16, kTogether = NL <= 4 ? kEach : 1;
    const int lane = threadIdx.x & 63, t0 = (threadIdx.x >> 6) * kEach;
#pragma unroll
    for (int g = 0; g < kEach; g += kTogether) {
        unsigned key[kTogether][NL];
#pragma unroll
        for (int k = 0; k < kTogether; ++k) load_keys<T, NL>(p, min(token0 + t0 + g + k, p.tokens - 1), lane, key[k]);
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
            const int t = t0 + g + k;
            if (token0 + t >= p.tokens) break;
            int expert;
            float weight;
            choose<NL>(p.top_k, p.renormalise != 0, key[k], lane, expert, weight);
            if (lane < p.top_k) {
                const size_t at = size_t(token0 + t) * p.top_k + lane;
                p.chosen[at] = expert;
                p.weights[at] = weight;
                s.chosen[t * p.top_k + lane] = short(expert);
            }
        }
    }
}

// Ranks the step's entries (s.chosen, n of them in the order of (token, j)) within their experts and writes their places; s.base moves on.
__device__ __forceinline__ void place_step(const RouteParams& p, RouteLds& s, int token0, int n) {
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x; i < p.top_k * p.experts; i += 1024) s.before[i] = 0;
    __syncthreads();
    int rank[kMaxTopK / 16];
#pragma unroll
    for (int r = 0; r < kMaxTopK / 16; ++r) {
        const int g = (threadIdx.x >> 6) + 16 * r, i = g * 64 + lane;
        if (g >= p.top_k) break;
        const int e = i < n ? s.chosen[i] : -1;
        unsigned long long same = __ballot(e >= 0);
#pragma unroll
        for (int b = 0; b < 10; ++b) {   // the lanes with the same expert
            const unsigned long long set = __ballot(e >> b & 1);
            same &= e >> b & 1 ? set : ~set;
        }
        rank[r] = __popcll(same & ((1ull << lane) - 1));
        if (e >= 0 && rank[r] == 0) s.before[g * p.experts + e] = (unsigned short)__popcll(same);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += 1024) {
        int sum = 0;
        for (int g = 0; g < p.top_k; ++g) {
            const int c = s.before[g * p.experts + e];
            s.before[g * p.experts + e] = (unsigned short)sum;
            sum += c;
        }
        s.count[e] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kMaxTopK / 16; ++r) {
        const int g = (threadIdx.x >> 6) + 16 * r, i = g * 64 + lane;
        if (g >= p.top_k) break;
        if (i >= n) continue;
        const int e = s.chosen[i];
        int slot = -1;
        if (e >= 0) {
            slot = s.base[e] + s.before[g * p.experts + e] + rank[r];
            p.index[slot] = token0 + i / p.top_k;
        }
        p.slots[size_t(token0) * p.top_k + i] = slot;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.experts; e += 1024) s.base[e] += s.count[e];
    __syncthreads();
}

// s.count[e]: all rows of expert e; s.base[e]: its rows in earlier chunks.  Afterwards s.base[e] is where its next row goes.  The first
// workgroup writes the offsets; all of them share the entries past the last row.
__device__ __forceinline__ void bases(const RouteParams& p, RouteLds& s) {
    scan_lds(s.count, p.experts, [](int a, int b) { return a + b; });
    const int e = threadIdx.x;
    if (e < p.experts) {
        s.base[e] += e ? s.count[e - 1] : 0;
        if (blockIdx.x == 0) {
            p.offsets[e + 1] = s.count[e];
            if (e == 0) p.offsets[0] = 0;
        }
    }
    const int rows = s.count[p.experts - 1];
    for (size_t i = size_t(rows) + blockIdx.x * 1024 + threadIdx.x; i < size_t(p.tokens) * p.top_k; i += size_t(gridDim.x) * 1024) p.index[i] = -1;
    __syncthreads();
}

template <int T, int NL, bool ALONE>
__global__ __launch_bounds__(1024) void k_route_choose(RouteParams p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    RouteLds& s = *reinterpret_cast<RouteLds*>(smem);
    for (int e = threadIdx.x; e < p.experts; e += 1024) s.count[e] = s.base[e] = 0;
    const int steps = route_steps(p.tokens), per_chunk = (steps + p.chunks - 1) / p.chunks;
    for (int step = blockIdx.x * per_chunk; step < min(steps, int(blockIdx.x + 1) * per_chunk); ++step) {
        __syncthreads();
        choose_step<T, NL>(p, s, step * kRouteStep);
        __syncthreads();
        const int n = min(kRouteStep, p.tokens - step * kRouteStep) * p.top_k;
        for (int i = threadIdx.x; i < n; i += 1024)
            if (s.chosen[i] >= 0) atomicAdd(&s.count[s.chosen[i]], 1);   // whole numbers: the order does not matter
    }
    __syncthreads();
    if constexpr (ALONE) {   // one step
        bases(p, s);
        place_step(p, s, 0, p.tokens * p.top_k);
    } else {
        for (int e = threadIdx.x; e < p.experts; e += 1024) p.counts[size_t(blockIdx.x) * p.experts + e] = s.count[e];
    }
}

__global__ __launch_bounds__(1024) void k_route_place(RouteParams p) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    RouteLds& s = *reinterpret_cast<RouteLds*>(smem);
    for (int e = threadIdx.x; e < p.experts; e += 1024) s.count[e] = s.base[e] = 0;
    __syncthreads();
    // the counts of all chunks: as many threads as there are experts to a row of them, eight requests at a time
    const int parts = max(1, 1024 / p.experts);
    for (int e = threadIdx.x % p.experts, part = threadIdx.x / p.experts; part < parts && e < p.experts; part += parts) {
        int all = 0, before = 0;
        for (int c0 = part; c0 < p.chunks; c0 += 8 * parts) {
            int c[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) c[k] = c0 + k * parts < p.chunks ? p.counts[size_t(c0 + k * parts) * p.experts + e] : 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                all += c[k];
                before += c0 + k * parts < int(blockIdx.x) ? c[k] : 0;
            }
        }
        atomicAdd(&s.count[e], all);   // whole numbers: the order does not matter
        atomicAdd(&s.base[e], before);
    }
    __syncthreads();
    bases(p, s);
    const int steps = route_steps(p.tokens), per_chunk = (steps + p.chunks - 1) / p.chunks;
    for (int step = blockIdx.x * per_chunk; step < min(steps, int(blockIdx.x + 1) * per_chunk); ++step) {
        const int token0 = step * kRouteStep, n = min(kRouteStep, p.tokens - token0) * p.top_k;
        for (int i = threadIdx.x; i < n; i += 1024) s.chosen[i] = short(p.chosen[size_t(token0) * p.top_k + i]);
        __syncthreads();
        place_step(p, s, token0, n);
    }
}

static int route_chunks(int tokens) { return std::max(1, std::min(route_steps(tokens), kRouteChunks)); }
size_t route_workspace_bytes(int tokens, int experts) {   // the chunks' counts; one chunk has them in LDS
    return tokens <= kRouteStep ? 1 : size_t(route_chunks(tokens)) * experts * 4;
}

template <int T, int NL>
static hipError_t route(const RouteParams& p, hipStream_t st) {
    const unsigned lds = unsigned(sizeof(RouteLds)) + unsigned(p.top_k * p.experts * 2);
    const bool alone = p.tokens <= kRouteStep;
    const void* const kernels[] = {reinterpret_cast<const void*>(&k_route_choose<T, NL, true>), reinterpret_cast<const void*>(&k_route_choose<T, NL, false>),
                                   reinterpret_cast<const void*>(&k_route_place)};
    if (lds > 65536)
        for (const void* k : kernels) {
            const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
            if (e != hipSuccess) return e;
        }
    if (alone) {
        hipLaunchKernelGGL((k_route_choose<T, NL, true>), dim3(1), dim3(1024), lds, st, p);
    } else {
        hipLaunchKernelGGL((k_route_choose<T, NL, false>), dim3(unsigned(p.chunks)), dim3(1024), lds, st, p);
        hipLaunchKernelGGL(k_route_place, dim3(unsigned(p.chunks)), dim3(1024), lds, st, p);
    }
    return hipGetLastError();
}

template <int T>
static hipError_t route_of(const RouteParams& p, hipStream_t st) {
    if (p.experts <= 64) return route<T, 1>(p, st);
    if (p.experts <= 128) return route<T, 2>(p, st);
    if (p.experts <= 256) return route<T, 4>(p, st);
    return route<T, 16>(p, st);
}

hipError_t launch_route(RouteParams p, int dtype, void* workspace, hipStream_t st) {
    p.counts = static_cast<int*>(workspace);
    p.chunks = route_chunks(p.tokens);
    if (dtype == BITSTACK_T_F16) return route_of<BITSTACK_T_F16>(p, st);
    if (dtype == BITSTACK_T_BF16) return route_of<BITSTACK_T_BF16>(p, st);
    return route_of<BITSTACK_T_F32>(p, st);
}

// ---- y[t] = sum_j weights[t][j] h[slots[t][j]]: eight columns a thread, 16 bytes a load, sums in fp32 in the order of j.  Bound by memory: 2048 tokens x 6 rows
// of 4096 in bf16 22.5 us, 5.2 TB/s, what a large copy reaches; 57 x 2 rows 2.9 us, a launch and two dependent loads.
template <int T>
__global__ __launch_bounds__(256) void k_combine(CombineParams p) {
    typedef typename Elem<T>::type E;
    const int token = blockIdx.x, col = (blockIdx.y * 256 + threadIdx.x) * 8;
    if (col >= p.width) return;
    float sum[8] = {};
    for (int j = 0; j < p.top_k; ++j) {
        const int slot = p.slots[size_t(token) * p.top_k + j];
        if (unsigned(slot) >= unsigned(p.h_rows)) continue;
        const float w = p.weights[size_t(token) * p.top_k + j];
        float v[8];
        load_elems<T, 8>(static_cast<const E*>(p.h) + size_t(slot) * p.ld_h + col, p.width - col, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = fmaf(w, v[i], sum[i]);
    }
    E* const y = static_cast<E*>(p.y) + size_t(token) * p.ld_y + col;
    if (p.width - col >= 8) {
#pragma unroll
        for (int i = 0; i < 8 / Elem<T>::kPer16; ++i) {
            typename Piece<T>::type u;
#pragma unroll
            for (int e = 0; e < Elem<T>::kPer16; ++e) u[e] = E(sum[i * Elem<T>::kPer16 + e]);
            reinterpret_cast<typename Piece<T>::loose*>(y)[i] = u;
        }
    } else {
        for (int i = 0; i < 8 && col + i < p.width; ++i) y[i] = E(sum[i]);
    }
}

template <int T>
static void combine(CombineParams p, hipStream_t st) {
    constexpr int kMost = 1 << 23;   // workgroups: a launch takes fewer than 2^32 threads
    for (; p.tokens > 0; p.tokens -= kMost) {
        hipLaunchKernelGGL((k_combine<T>), dim3(unsigned(std::min(p.tokens, kMost)), unsigned((p.width + 2047) / 2048)), dim3(256), 0, st, p);
        p.slots += size_t(kMost) * p.top_k;
        p.weights += size_t(kMost) * p.top_k;
        p.y = static_cast<typename Elem<T>::type*>(p.y) + size_t(kMost) * p.ld_y;
    }
}

hipError_t launch_combine(const CombineParams& p, int dtype, hipStream_t st) {
    if (dtype == BITSTACK_T_F16) combine<BITSTACK_T_F16>(p, st);
    else if (dtype == BITSTACK_T_BF16) combine<BITSTACK_T_BF16>(p, st);
    else combine<BITSTACK_T_F32>(p, st);
    return hipGetLastError();
}

}  // namespace bitstack
