// Host side of include/bitstack_f8.h: argument checks, the layout of the workspace, dispatch.
#include <hip/hip_runtime.h>

#include "../../include/bitstack_f8.h"
#include "expert_layer.h"
#include "f8.h"
#include "layout.h"

using namespace bitstack;

namespace {

constexpr int kMaxIn = 1 << 20, kMaxOut = 1 << 24;
constexpr size_t kMaxLd = size_t(1) << 22;               // bytes between two rows of a weight: a tile of 256 is reached by 31-bit offsets
constexpr size_t kMaxRowBytes = (size_t(1) << 31) - 1;   // 8-bit activations: reached by 31-bit offsets

bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }
bool real_type(int t) { return t == BITSTACK_T_F16 || t == BITSTACK_T_F32 || t == BITSTACK_T_BF16; }
size_t type_size(int t) { return t == BITSTACK_T_F32 ? 4 : 2; }
bool columns_ok(int in) { return in >= 1 && in <= kMaxIn; }

// What a call needs of the workspace.  `raw`: the product itself brings the activations to 8 bits.
struct Workspace {
    size_t q, scales, list, part, total;
};
Workspace workspace_of(int x_rows, int in, const F8Plan& plan, bool raw, bool grouped) {
    Workspace w;
    w.q = 0;
    w.scales = raw ? 0 : align256(size_t(x_rows) * bitstack_f8_row_bytes(in));
    w.list = raw ? 0 : w.scales + align256(size_t(x_rows) * bitstack_f8_row_scales(in));
    w.part = w.list + (grouped ? align256(size_t(plan.n_tiles) * sizeof(F8Tile)) : 0);
    w.total = w.part + align256(plan.part_bytes);
    return w;
}
// The least that calls with up to so many rows run in, whichever their kernels: the work list of the smallest tiles, no partial sums
size_t least_workspace(int x_rows, int in, int y_rows, int experts) {
    F8Plan plan{};
    plan.n_tiles = y_rows / 16 + 1 + (y_rows < experts ? y_rows : experts);
    return workspace_of(x_rows, in, plan, false, true).total;
}

int check_rows(const bitstack_f8_rows_t& x, int in) {
    if (x.rows < 0) return BITSTACK_E_RANGE;
    if (size_t(x.rows) * bitstack_f8_row_bytes(in) > kMaxRowBytes) return BITSTACK_E_RANGE;
    if (x.dtype == BITSTACK_T_F8) {
        if (x.rows && (!x.x || !x.scales)) return BITSTACK_E_NULL;
        if (misaligned(x.x, 16) || misaligned(x.scales, 4)) return BITSTACK_E_ALIGN;
        return BITSTACK_OK;
    }
    if (!real_type(x.dtype) || (x.gated != 0 && x.gated != 1)) return BITSTACK_E_ARG;
    if (x.rows && !x.x) return BITSTACK_E_NULL;
    if (misaligned(x.x, type_size(x.dtype))) return BITSTACK_E_ALIGN;
    if (x.rows > 1 && x.ld < size_t(in) << x.gated) return BITSTACK_E_SHAPE;
    return BITSTACK_OK;
}

int check_call(const bitstack_f8_rows_t* x, const bitstack_f8_weight_t* w, int y_rows, int y_dtype) {
    if (y_rows < 0) return BITSTACK_E_RANGE;
    if (!columns_ok(w->in) || w->out < 1 || w->out > kMaxOut || w->experts < 1 || w->experts > kMaxExperts) return BITSTACK_E_SHAPE;
    if (w->scale_type != BITSTACK_S_E8M0 && w->scale_type != BITSTACK_S_F32) return BITSTACK_E_ARG;
    if (!real_type(y_dtype)) return BITSTACK_E_ARG;
    return check_rows(*x, w->in);
}

// Does the product bring the activations to 8 bits itself?  A few rows of 16 bits, not gated, in no groups (their work list is made by the launch that
// quantises), in whole 16-byte pieces within reach of 31-bit offsets.  Every workgroup converts all columns anew, kb blocks for each tile of
// 16 or 64 rows of the weight: up to 64 blocks on a compute unit (measurements at k_f8_slices; fp32 rows and gated ones take two to six times as
// long there as a launch more).
bool raw_rows(const bitstack_f8_rows_t& x, const bitstack_f8_weight_t& w, int y_rows, const F8Plan& plan, bool grouped) {
    if (grouped || x.gated || (x.dtype != BITSTACK_T_F16 && x.dtype != BITSTACK_T_BF16) || y_rows > 16 || plan.tile_rows != 16 || w.in % 16 != 0) return false;
    if (size_t(plan.tiles) * ((w.in + kF8Block - 1) / kF8Block) > 64 * 256) return false;
    return !misaligned(x.x, 16) && (x.rows == 1 || (x.ld % 8 == 0 && x.ld <= kMaxRowBytes / 2)) && (size_t(x.rows - 1) * x.ld + w.in) * 2 <= kMaxRowBytes;
}

// What follows the product.  Gates and values meet inside it where their rows do not share blocks of 128 and one descriptor reaches both by 31-bit offsets;
// otherwise they are joined from partial sums of all rows.
bool is_gated(const bitstack_f8_epilogue_t* e) { return e && e->activation == BITSTACK_ACT_SILU_GATED; }
bool any_epilogue(const bitstack_f8_epilogue_t* e) { return e && (e->bias || e->residual || e->activation != BITSTACK_ACT_NONE); }
bool parts_only(const bitstack_f8_epilogue_t* e, int out, size_t ld) {
    return is_gated(e) && (out / 2 % kF8Block != 0 || (size_t(out / 2) + 256) * ld > kMaxRowBytes);
}
F8Plan plan_of(const bitstack_f8_epilogue_t* e, int rows, const bitstack_f8_weight_t& w, bool grouped, bool exact, size_t room = ~size_t(0)) {
    const bool ws_f32 = w.scale_type == BITSTACK_S_F32;
    return parts_only(e, w.out, w.ld) ? f8_plan_parts(rows, w.out, w.in, exact, ws_f32, room) : f8_plan(rows, w.out, w.in, w.experts, grouped, exact, ws_f32, room);
}
int check_epilogue(const bitstack_f8_epilogue_t& e, const bitstack_f8_weight_t& w, int rows, int y_dtype) {
    if (e.activation < BITSTACK_ACT_NONE || e.activation > BITSTACK_ACT_SILU_GATED) return BITSTACK_E_ARG;
    if (e.bias && !real_type(e.bias_dtype)) return BITSTACK_E_ARG;
    const bool gated = is_gated(&e);
    if (gated && w.out % 2 != 0) return BITSTACK_E_SHAPE;
    if (gated && w.out / 2 % kF8Block == 0 && w.ld <= kMaxLd && size_t(w.out / 2) * w.ld >> 32) return BITSTACK_E_RANGE;   // as documented
    if (e.bias && misaligned(e.bias, type_size(e.bias_dtype))) return BITSTACK_E_ALIGN;
    if (misaligned(e.residual, type_size(y_dtype))) return BITSTACK_E_ALIGN;
    if (e.residual && rows > 1 && e.ld_residual < size_t(gated ? w.out / 2 : w.out)) return BITSTACK_E_SHAPE;
    return BITSTACK_OK;
}

// Do rows of a and of b, so many bytes long and so far apart, share memory?
struct Rows {
    const void* p;
    size_t ld, bytes;
};
bool share_memory(const Rows& a, const Rows& b, int rows) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    if (a0 + (rows - 1) * a.ld + a.bytes <= b0 || b0 + (rows - 1) * b.ld + b.bytes <= a0) return false;
    for (int i = 0; i < rows; ++i)   // they may lie between each other
        for (int j = 0; j < rows; ++j)
            if (a0 + i * a.ld < b0 + j * b.ld + b.bytes && b0 + j * b.ld < a0 + i * a.ld + a.bytes) return true;
    return false;
}

int product(const bitstack_f8_rows_t* x, const bitstack_f8_weight_t* w, const int32_t* offsets, const int32_t* index, int y_rows, const bitstack_f8_epilogue_t* epi,
            void* y, int y_dtype, size_t ld_y, void* workspace, size_t workspace_bytes, bitstack_stream_t stream) {
    int rc = check_call(x, w, y_rows, y_dtype);
    if (rc == BITSTACK_OK && epi) rc = check_epilogue(*epi, *w, y_rows, y_dtype);
    if (rc) return rc;
    const int cols = is_gated(epi) ? w->out / 2 : w->out;
    if (y_rows == 0) return BITSTACK_OK;
    if (!w->q || !w->scales || !y) return BITSTACK_E_NULL;
    if (misaligned(w->q, 16) || w->ld % 16 || (w->scale_type == BITSTACK_S_F32 && misaligned(w->scales, 4))) return BITSTACK_E_ALIGN;
    if (w->ld < size_t(w->in) || w->ld > kMaxLd || (y_rows > 1 && ld_y < size_t(cols))) return BITSTACK_E_SHAPE;
    if (misaligned(y, type_size(y_dtype))) return BITSTACK_E_ALIGN;
    auto plan_in = [&](size_t room) {
        return plan_of(epi, y_rows, *w, offsets != nullptr, y_dtype == BITSTACK_T_F32, room);
    };
    F8Plan plan = plan_in(~size_t(0));
    if (!f8_launchable(plan)) return BITSTACK_E_RANGE;   // with any kernel's tiles
    if (parts_only(epi, w->out, w->ld) && plan.part_bytes >> 37) return BITSTACK_E_RANGE;   // joining them is one launch, 32 bytes to a thread
    const bool quantised = x->dtype == BITSTACK_T_F8;
    // Where every workgroup reads x for itself, one may have written its outputs before another one reads: not over x
    bool raw = raw_rows(*x, *w, y_rows, plan, offsets != nullptr);
    if (raw && plan.tiles > 1) {
        const size_t size = type_size(y_dtype);
        raw = !share_memory({x->x, x->rows > 1 ? x->ld * 2 : 0, size_t(w->in) * 2}, {y, y_rows > 1 ? ld_y * size : 0, cols * size}, y_rows);
    }
    Workspace at = workspace_of(x->rows, w->in, plan, quantised || raw, offsets != nullptr);
    if (at.total) {
        if (!workspace) return BITSTACK_E_NULL;
        if (misaligned(workspace, 256)) return BITSTACK_E_ALIGN;
        if (workspace_bytes < at.total && plan.part_bytes) {   // made for more rows, whose columns need not be sliced: as many slices as fit
            plan = plan_in(workspace_bytes < at.list ? 0 : workspace_bytes - at.list);
            at = workspace_of(x->rows, w->in, plan, quantised, offsets != nullptr);
        }
        if (workspace_bytes < at.total) return BITSTACK_E_BUFSIZE;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    F8WorkList list;
    if (offsets) list = {offsets, w->experts, y_rows, plan.tile_rows, plan.n_tiles, reinterpret_cast<F8Tile*>(ws + at.list)};
    F8Params p{};
    p.x_dtype = BITSTACK_T_F8;
    p.x_bytes = unsigned(size_t(x->rows) * bitstack_f8_row_bytes(w->in));
    const bool rows_here = !quantised && !raw && x->rows > 0;
    if (rows_here || offsets) {
        const hipError_t e = launch_f8_quantise(x->x, rows_here ? x->dtype : int(BITSTACK_T_F16), x->ld, rows_here ? x->rows : 0, w->in, x->gated != 0, ws + at.q,
                                                ws + at.scales, list, st);
        if (e != hipSuccess) return hip_error(e);
    }
    p.x = ws + at.q;
    p.xs = ws + at.scales;
    if (quantised) {
        p.x = static_cast<const unsigned char*>(x->x);
        p.xs = static_cast<const unsigned char*>(x->scales);
    } else if (raw) {
        p.x = static_cast<const unsigned char*>(x->x);
        p.x_dtype = x->dtype;
        p.x_bytes = unsigned((size_t(x->rows - 1) * x->ld + w->in) * 2);
        p.x_ld = x->rows > 1 ? unsigned(x->ld * 2) : 0;
    }
    p.w = static_cast<const unsigned char*>(w->q);
    p.ws = w->scales;
    p.y = y;
    p.index = index;
    p.tiles = list.tiles;
    p.part = reinterpret_cast<float*>(ws + at.part);
    p.ldw = w->ld;
    p.ldy = ld_y;
    p.out = w->out;
    p.in = w->in;
    p.kb = (w->in + kF8Block - 1) / kF8Block;
    p.kp = p.kb * kF8Block;
    p.ks = int(bitstack_f8_row_scales(w->in));
    p.x_rows = x->rows;
    p.rows = y_rows;
    p.y_dtype = y_dtype;
    p.ws_f32 = w->scale_type == BITSTACK_S_F32;
    if (any_epilogue(epi)) {
        p.epi = is_gated(epi) ? kEpiGated : kEpiPlain;
        p.act = epi->activation;
        p.cols = cols;
        p.bias = epi->bias;
        p.bias_dtype = epi->bias_dtype;
        p.residual = epi->residual;
        p.ld_r = epi->ld_residual;
        p.parts_only = parts_only(epi, w->out, w->ld);
    }
    const hipError_t e = launch_f8_product(p, plan, st);
    return e == hipSuccess ? BITSTACK_OK : hip_error(e);
}

// The workspace of a layer of experts
struct LayerWorkspace {
    size_t list, row_weight, row_token, arrived, h, part, total;
};
// bytes of h: the rows, or fragments of 16 tokens of every entry of the list; whole blocks of columns
size_t h_bytes_of(const LayerPlan& plan, size_t rows, int width, int h_parts) {
    return (plan.pack ? rows : size_t(plan.most) * plan.fragments * 16) * ((size_t(width) + 127) / 128) * h_parts * 256;
}
LayerWorkspace layer_workspace(int tokens, int hidden, int width, int experts, int top_k, int h_parts) {
    const LayerPlan plan = layer_plan(tokens, hidden, width, experts, top_k, h_parts == 3);
    const size_t rows = size_t(tokens) * top_k;
    LayerWorkspace w;
    w.list = 256;
    w.row_weight = w.list + align256(size_t(plan.most) * sizeof(LayerExpert));
    w.row_token = w.row_weight + align256(rows * 4);
    w.arrived = w.row_token + align256(rows);
    w.h = w.arrived + align256(size_t(plan.tiles_down) * 4);
    w.part = w.h + align256(h_bytes_of(plan, rows, width, h_parts));
    w.total = w.part + (plan.splits > 1 ? align256(size_t(plan.tiles_down) * plan.splits * tokens * plan.down_rows * 4) : 0);
    return w;
}
bool layer_sizes_ok(int hidden, int width, int experts, int top_k) {
    return hidden >= 8 && columns_ok(hidden) && columns_ok(width) && experts >= 1 && experts <= kMaxExperts && top_k >= 1 && top_k <= kMaxTopK && top_k <= experts;
}
int check_weight(const bitstack_f8_weight_t& w) {
    if (w.scale_type != BITSTACK_S_E8M0 && w.scale_type != BITSTACK_S_F32) return BITSTACK_E_ARG;
    if (!w.q || !w.scales) return BITSTACK_E_NULL;
    if (misaligned(w.q, 16) || w.ld % 16 || (w.scale_type == BITSTACK_S_F32 && misaligned(w.scales, 4))) return BITSTACK_E_ALIGN;
    if (w.ld < size_t(w.in) || w.ld > kMaxLd) return BITSTACK_E_SHAPE;
    return BITSTACK_OK;
}

}  // namespace

extern "C" {

size_t bitstack_f8_row_bytes(int in) { return columns_ok(in) ? (size_t(in) + 127) / 128 * 128 : 0; }
size_t bitstack_f8_row_scales(int in) { return columns_ok(in) ? ((size_t(in) + 127) / 128 + 3) / 4 * 4 : 0; }

int bitstack_f8_quantise(const void* x, int x_dtype, size_t ld, int rows, int in, int gated, void* q, void* scales,
                         bitstack_stream_t stream) {
    if (!columns_ok(in)) return BITSTACK_E_SHAPE;
    if (x_dtype == BITSTACK_T_F8) return BITSTACK_E_ARG;
    const bitstack_f8_rows_t r = {x, nullptr, ld, x_dtype, rows, gated};
    const int rc = check_rows(r, in);
    if (rc) return rc;
    if (rows == 0) return BITSTACK_OK;
    if (!q || !scales) return BITSTACK_E_NULL;
    if (misaligned(q, 16) || misaligned(scales, 4)) return BITSTACK_E_ALIGN;
    const hipError_t e = launch_f8_quantise(x, x_dtype, ld, rows, in, gated != 0, static_cast<unsigned char*>(q),
                                            static_cast<unsigned char*>(scales), F8WorkList{}, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? BITSTACK_OK : hip_error(e);
}

int bitstack_f8_quantise_weight(const void* w, int w_dtype, size_t ld, int out, int in, void* q, size_t ld_q, void* scales,
                                bitstack_stream_t stream) {
    if (!columns_ok(in) || out < 1 || out > kMaxOut) return BITSTACK_E_SHAPE;
    if (!real_type(w_dtype)) return BITSTACK_E_ARG;
    if (!w || !q || !scales) return BITSTACK_E_NULL;
    if (misaligned(w, type_size(w_dtype)) || misaligned(q, 16) || ld_q % 16) return BITSTACK_E_ALIGN;
    if ((out > 1 && ld < size_t(in)) || ld_q < size_t(in) || ld_q > kMaxLd) return BITSTACK_E_SHAPE;
    const hipError_t e = launch_f8_quantise_weight(w, w_dtype, ld, out, in, static_cast<unsigned char*>(q), ld_q,
                                                   static_cast<unsigned char*>(scales), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? BITSTACK_OK : hip_error(e);
}

size_t bitstack_f8_workspace_bytes(int x_rows, int in, int y_rows, int out, int experts) {
    if (x_rows < 0 || y_rows < 0 || !columns_ok(in) || out < 1 || out > kMaxOut || experts < 1 || experts > kMaxExperts) return 0;
    if (size_t(x_rows) * bitstack_f8_row_bytes(in) > kMaxRowBytes) return 0;
    size_t most = least_workspace(x_rows, in, y_rows, experts);
    for (int k = 0; k < 8; ++k)
        if (y_rows) {
            const size_t n = workspace_of(x_rows, in, f8_plan(y_rows, out, in, experts, k & 1, k >> 1 & 1, k >> 2), false, true).total;
            most = n > most ? n : most;
        }
    return most;
}

size_t bitstack_f8_call_workspace_bytes(const bitstack_f8_rows_t* x, const bitstack_f8_weight_t* w, int y_rows, int y_dtype, int grouped) {
    if (!x || !w || check_call(x, w, y_rows, y_dtype) || y_rows == 0) return 0;
    const F8Plan plan = f8_plan(y_rows, w->out, w->in, w->experts, grouped != 0, y_dtype == BITSTACK_T_F32, w->scale_type == BITSTACK_S_F32);
    return workspace_of(x->rows, w->in, plan, x->dtype == BITSTACK_T_F8 || raw_rows(*x, *w, y_rows, plan, grouped != 0), grouped != 0).total;
}

int bitstack_f8_linear(const bitstack_f8_rows_t* x, const bitstack_f8_weight_t* w, void* y, int y_dtype, size_t ld_y,
                       void* workspace, size_t workspace_bytes, bitstack_stream_t stream) {
    if (!x || !w) return BITSTACK_E_NULL;
    if (w->experts != 1) return BITSTACK_E_SHAPE;
    return product(x, w, nullptr, nullptr, x->rows, nullptr, y, y_dtype, ld_y, workspace, workspace_bytes, stream);
}

int bitstack_f8_grouped_linear(const bitstack_f8_rows_t* x, const bitstack_f8_weight_t* w, const int32_t* offsets,
                               const int32_t* index, int y_rows, void* y, int y_dtype, size_t ld_y, void* workspace,
                               size_t workspace_bytes, bitstack_stream_t stream) {
    if (!x || !w || !offsets || (!index && y_rows > 0 && y_rows > x->rows)) return !x || !w || !offsets ? BITSTACK_E_NULL : BITSTACK_E_RANGE;
    if (misaligned(offsets, 4) || misaligned(index, 4)) return BITSTACK_E_ALIGN;
    return product(x, w, offsets, index, y_rows, nullptr, y, y_dtype, ld_y, workspace, workspace_bytes, stream);
}

size_t bitstack_f8_epilogue_workspace_bytes(int rows, int in, int out, int activation) {
    if (activation < BITSTACK_ACT_NONE || activation > BITSTACK_ACT_SILU_GATED || (activation == BITSTACK_ACT_SILU_GATED && out % 2 != 0)) return 0;
    size_t most = bitstack_f8_workspace_bytes(rows, in, rows, out, 1);
    const bitstack_f8_epilogue_t e = {nullptr, 0, activation, nullptr, 0};
    if (!most || !rows || !parts_only(&e, out, bitstack_f8_row_bytes(in))) return most;
    for (int k = 0; k < 4; ++k) {
        const size_t n = workspace_of(rows, in, f8_plan_parts(rows, out, in, k & 1, k >> 1), false, false).total;
        most = n > most ? n : most;
    }
    return most;
}

size_t bitstack_f8_epilogue_call_workspace_bytes(const bitstack_f8_rows_t* x, const bitstack_f8_weight_t* w, const bitstack_f8_epilogue_t* epilogue, int y_dtype) {
    if (!x || !w || w->experts != 1 || check_call(x, w, x->rows, y_dtype) || (epilogue && check_epilogue(*epilogue, *w, x->rows, y_dtype)) || x->rows == 0) return 0;
    const F8Plan plan = plan_of(epilogue, x->rows, *w, false, y_dtype == BITSTACK_T_F32);
    return workspace_of(x->rows, w->in, plan, x->dtype == BITSTACK_T_F8 || raw_rows(*x, *w, x->rows, plan, false), false).total;
}

int bitstack_f8_linear_epilogue(const bitstack_f8_rows_t* x, const bitstack_f8_weight_t* w, const bitstack_f8_epilogue_t* epilogue, void* y, int y_dtype,
                                size_t ld_y, void* workspace, size_t workspace_bytes, bitstack_stream_t stream) {
    if (!x || !w || !epilogue) return BITSTACK_E_NULL;
    if (w->experts != 1) return BITSTACK_E_SHAPE;
    return product(x, w, nullptr, nullptr, x->rows, epilogue, y, y_dtype, ld_y, workspace, workspace_bytes, stream);
}

size_t bitstack_route_workspace_bytes(int tokens, int experts, int top_k) {
    if (tokens < 0 || experts < 1 || experts > kMaxExperts || top_k < 1 || top_k > kMaxTopK || top_k > experts) return 0;
    return align256(route_workspace_bytes(tokens, experts));
}

int bitstack_route(const void* logits, int dtype, size_t ld, int tokens, int experts, int top_k, int renormalise,
                   int32_t* chosen, float* weights, int32_t* slots, int32_t* index, int32_t* offsets, void* workspace,
                   size_t workspace_bytes, bitstack_stream_t stream) {
    if (tokens < 0 || size_t(tokens) * size_t(top_k > 0 ? top_k : 0) > 0x7fffffffu) return BITSTACK_E_RANGE;
    if (experts < 1 || experts > kMaxExperts || top_k < 1 || top_k > kMaxTopK || top_k > experts) return BITSTACK_E_SHAPE;
    if (!real_type(dtype) || (renormalise != 0 && renormalise != 1)) return BITSTACK_E_ARG;
    if (!offsets || !workspace || (tokens && (!logits || !chosen || !weights || !slots || !index))) return BITSTACK_E_NULL;
    if (misaligned(logits, type_size(dtype)) || misaligned(chosen, 4) || misaligned(weights, 4) || misaligned(slots, 4) || misaligned(index, 4) ||
        misaligned(offsets, 4) || misaligned(workspace, 256))
        return BITSTACK_E_ALIGN;
    if (tokens > 1 && ld < size_t(experts)) return BITSTACK_E_SHAPE;
    if (workspace_bytes < bitstack_route_workspace_bytes(tokens, experts, top_k)) return BITSTACK_E_BUFSIZE;
    RouteParams p{logits, ld, tokens, experts, top_k, renormalise, chosen, weights, slots, index, offsets, nullptr, 0};
    const hipError_t e = launch_route(p, dtype, workspace, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? BITSTACK_OK : hip_error(e);
}

int bitstack_combine(const void* h, int dtype, size_t ld_h, int h_rows, int width, const int32_t* slots,
                     const float* weights, int tokens, int top_k, void* y, size_t ld_y, bitstack_stream_t stream) {
    if (h_rows < 0 || tokens < 0) return BITSTACK_E_RANGE;
    if (width < 1 || width > kMaxOut || top_k < 1 || top_k > kMaxTopK) return BITSTACK_E_SHAPE;
    if (!real_type(dtype)) return BITSTACK_E_ARG;
    if (tokens == 0) return BITSTACK_OK;
    if ((h_rows && !h) || !slots || !weights || !y) return BITSTACK_E_NULL;
    const size_t size = type_size(dtype);
    if (misaligned(h, size) || misaligned(y, size) || misaligned(slots, 4) || misaligned(weights, 4)) return BITSTACK_E_ALIGN;
    if ((h_rows > 1 && ld_h < size_t(width)) || (tokens > 1 && ld_y < size_t(width))) return BITSTACK_E_SHAPE;
    const CombineParams p{h, y, slots, weights, ld_h, ld_y, h_rows, width, tokens, top_k};
    const hipError_t e = launch_combine(p, dtype, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? BITSTACK_OK : hip_error(e);
}

size_t bitstack_f8_expert_layer_workspace_bytes(int tokens, int hidden, int width, int experts, int top_k) {
    if (tokens < 0 || tokens > kLayerTokens || !layer_sizes_ok(hidden, width, experts, top_k)) return 0;
    size_t most = 256;
    for (int t = 1; t <= tokens; ++t)
        for (int parts = 2; parts <= 3; ++parts) {
            const size_t n = layer_workspace(t, hidden, width, experts, top_k, parts).total;
            most = n > most ? n : most;
        }
    return most;
}

int bitstack_f8_expert_layer(const void* x, int dtype, size_t ld_x, const void* logits, int logits_dtype, size_t ld_logits, int tokens, int top_k,
                             int renormalise, const bitstack_f8_weight_t* w1, const bitstack_f8_weight_t* w2, const void* residual,
                             size_t ld_residual, void* y, size_t ld_y, void* workspace, size_t workspace_bytes, bitstack_stream_t stream) {
    if (!w1 || !w2) return BITSTACK_E_NULL;
    if (tokens < 0 || tokens > kLayerTokens) return BITSTACK_E_RANGE;
    const int hidden = w1->in, width = w2->in, experts = w1->experts;
    if (!layer_sizes_ok(hidden, width, experts, top_k) || w2->experts != experts || w1->out != 2 * width || w2->out != hidden) return BITSTACK_E_SHAPE;
    if (!real_type(dtype) || !real_type(logits_dtype) || (renormalise != 0 && renormalise != 1)) return BITSTACK_E_ARG;
    int rc = check_weight(*w1);
    if (rc == BITSTACK_OK) rc = check_weight(*w2);
    if (rc) return rc;
    if (tokens == 0) return BITSTACK_OK;
    if (!x || !logits || !y || !workspace) return BITSTACK_E_NULL;
    const size_t size = type_size(dtype);
    if (misaligned(x, size) || misaligned(y, size) || misaligned(residual, size) || misaligned(logits, type_size(logits_dtype)) || misaligned(workspace, 256))
        return BITSTACK_E_ALIGN;
    if (tokens > 1 && (ld_x < size_t(hidden) || ld_y < size_t(hidden) || (residual && ld_residual < size_t(hidden)) || ld_logits < size_t(experts)))
        return BITSTACK_E_SHAPE;
    const int h_parts = dtype == BITSTACK_T_F32 ? 3 : 2;
    const LayerPlan plan = layer_plan(tokens, hidden, width, experts, top_k, h_parts == 3);
    const size_t rows = size_t(tokens) * top_k, h_bytes = h_bytes_of(plan, rows, width, h_parts);
    // reached by 32-bit offsets (h by 31-bit ones)
    if (size_t(w1->out - 1) * w1->ld + (size_t(hidden) + 15) / 16 * 16 > 0xffffffffu || h_bytes > kMaxRowBytes) return BITSTACK_E_RANGE;
    const LayerWorkspace at = layer_workspace(tokens, hidden, width, experts, top_k, h_parts);
    if (workspace_bytes < at.total) return BITSTACK_E_BUFSIZE;
    unsigned char* const ws = static_cast<unsigned char*>(workspace);
    LayerParams p{};
    p.x = x;
    p.logits = logits;
    p.w1 = static_cast<const unsigned char*>(w1->q);
    p.s1 = static_cast<const unsigned char*>(w1->scales);
    p.w2 = static_cast<const unsigned char*>(w2->q);
    p.s2 = static_cast<const unsigned char*>(w2->scales);
    p.residual = residual;
    p.y = y;
    p.ld_x = ld_x;
    p.ld_logits = ld_logits;
    p.ld_w1 = w1->ld;
    p.ld_w2 = w2->ld;
    p.ld_r = ld_residual;
    p.ld_y = ld_y;
    p.dtype = dtype;
    p.logits_dtype = logits_dtype;
    p.s1_f32 = w1->scale_type == BITSTACK_S_F32;
    p.s2_f32 = w2->scale_type == BITSTACK_S_F32;
    p.tokens = tokens;
    p.top_k = top_k;
    p.renormalise = renormalise;
    p.experts = experts;
    p.hidden = hidden;
    p.width = width;
    p.fragments = plan.fragments;
    p.most = plan.most;
    p.up_few = plan.up_few;
    p.pack = plan.pack;
    p.count = reinterpret_cast<int*>(ws);
    p.list = reinterpret_cast<LayerExpert*>(ws + at.list);
    p.row_weight = reinterpret_cast<float*>(ws + at.row_weight);
    p.row_token = ws + at.row_token;
    p.arrived = reinterpret_cast<unsigned*>(ws + at.arrived);
    p.h = reinterpret_cast<unsigned short*>(ws + at.h);
    p.part = reinterpret_cast<float*>(ws + at.part);
    p.h_bytes = unsigned(h_bytes);
    p.h_parts = h_parts;
    p.down_rows = plan.down_rows;
    p.tiles_down = plan.tiles_down;
    p.splits = plan.splits;
    const hipError_t e = launch_expert_layer(p, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? BITSTACK_OK : hip_error(e);
}

}  // extern "C"
