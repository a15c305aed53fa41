// The products in 8-bit floating point with nothing after them, and the choice of kernel for all of them (kernels: f8_product.h).
#include <cmath>

#include "f8_product.h"

namespace bitstack {

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
F8Plan f8_plan_parts(int rows, int out, int in, bool exact, bool ws_f32, size_t room) {
    const int forced = g_forced.load(), kb = (in + 127) / 128;
    auto plan_of = [&](const F8KernelShape& k, int slices) {
        const int each = (kb + slices - 1) / slices, n_tiles = (rows + k.toks - 1) / k.toks;
        const size_t tiles = size_t((out + k.rows - 1) / k.rows) * n_tiles;
        return F8Plan{k.kernel, (kb + each - 1) / each, k.toks, n_tiles, int(std::min<size_t>(tiles, 0x7fffffff)), size_t((kb + each - 1) / each) * tiles * (k.rows * k.toks * 4)};
    };
    auto makes_parts = [&](const F8KernelShape& k) { return k.kernel > kSlices64 && makes(k, exact); };
    for (const F8KernelShape& k : kShapes)
        if (forced && k.kernel == forced % 1024 && makes_parts(k)) return plan_of(k, std::max(1, std::min(forced / 1024, kb)));
    F8Plan plan{};
    double best = 1e30;
    for (const F8KernelShape& k : kShapes) {
        if (!makes_parts(k)) continue;
        for (int slices : {1, 2, 3, 4, 5, 6, 7, 8, 12, 16}) {
            if (slices > 1 && slices > kb / 4) continue;
            const F8Plan this_one = plan_of(k, slices);
            // the sums are written and read whatever the slices
            const double tiles = double((out + k.rows - 1) / k.rows) * this_one.n_tiles;
            const double us = f8_time_us(k, slices, rows, out, kb, 1, false, exact, ws_f32) + (slices == 1 ? 4.0 + tiles * k.rows * k.toks * 8 / 6.3e6 : 0.0);
            if (plan.kernel && (us >= best || !f8_launchable(this_one) || this_one.part_bytes > room)) continue;   // the smallest tiles in one slice if nothing fits
            best = f8_launchable(this_one) && this_one.part_bytes <= room ? us : 1e30;
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
    if (p.epi == kEpiGated && !p.parts_only) return launch_f8_gated(p, plan, st);
    if (p.epi != kEpiNone) return launch_f8_epilogue(p, plan, st);
    return launch_f8_kernel<kEpiNone>(p, plan, st);
}

}  // namespace bitstack
