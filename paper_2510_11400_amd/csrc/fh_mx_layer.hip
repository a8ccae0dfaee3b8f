// A linear layer's training step in microscaled form, each half by one call: an optional layer norm, the operands' storage and the
// products, with everything in between in two buffers of the caller's.
#include "fh_norm.hpp"

namespace fh {
namespace {

inline size_t whole(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
inline size_t larger(size_t a, size_t b) { return a > b ? a : b; }

// Offsets into the two buffers.  kept: from the forward call until the backward one; scratch: within a call.
struct Parts {
    size_t mean, rstd, x_columns, w_columns, kept;
    size_t x_rows, w_rows, forward_work, forward;
    size_t dy_rows, dy_columns, dh, backward_work, backward;
};
constexpr int32_t kNeeds = FH_MX_NEEDS_INPUT | FH_MX_NEEDS_WEIGHT;
// `wide`: with the gradient of a norm's output in binary32, in the place of dy's columns, which only the product before it reads.
// `kept_for`, `stats`: what there is room for in `kept`.
Parts parts_of(int64_t tokens, int64_t features, int64_t out, bool wide, int32_t kept_for, bool stats)
{
    Parts p;
    p.mean = 0;
    p.rstd = stats ? whole((size_t)tokens * 4) : 0;
    p.x_columns = p.rstd * 2;
    p.w_columns = p.x_columns + (kept_for & FH_MX_NEEDS_WEIGHT ? whole(mx_bytes(features, tokens)) : 0);
    p.kept = p.w_columns + (kept_for & FH_MX_NEEDS_INPUT ? whole(mx_bytes(features, out)) : 0);
    p.x_rows = 0;
    p.w_rows = whole(mx_bytes(tokens, features));
    p.forward_work = p.w_rows + whole(mx_bytes(out, features));
    p.forward = p.forward_work + whole(fh_mx_matmul_workspace_bytes(tokens, out, features));
    p.dy_rows = 0;
    p.dy_columns = whole(mx_bytes(tokens, out));
    p.dh = p.dy_columns;
    p.backward_work = p.dy_columns + larger(whole(mx_bytes(out, tokens)), wide ? whole((size_t)tokens * (size_t)features * 4) : 0);
    p.backward = p.backward_work + whole(larger(larger(fh_mx_matmul_workspace_bytes(tokens, features, out), fh_mx_matmul_workspace_bytes(out, features, tokens)),
                                                larger(fh_layer_norm_backward_workspace_bytes(tokens, features), (size_t)mx_tile_rows(tokens) * (size_t)out * 4)));
    return p;
}

bool shape_ok(int64_t tokens, int64_t features, int64_t out)
{
    constexpr int64_t kMostSummed = (int64_t)1 << 24;             // each of the three is summed over by one of the products
    return tokens >= 0 && features >= 1 && out >= 1 && tokens <= kMostSummed && features <= kMostSummed && out <= kMostSummed;
}

fh_status check(const fh_mx_layer* l)
{
    if (!l) return FH_ERR_NULL;
    if (!is_dtype(l->dtype) || !is_dtype(l->p_dtype)) return FH_ERR_BAD_DTYPE;
    if (l->rounding != FH_ROUND_NEAREST && l->rounding != FH_ROUND_STOCHASTIC) return FH_ERR_BAD_ROUND;
    if (!shape_ok(l->tokens, l->features, l->out_features) || l->x_stride < l->features || l->weight_stride < l->features ||
        l->dy_stride < l->out_features || l->x_stride > kMostStride || l->weight_stride > kMostStride || l->dy_stride > kMostStride)
        return FH_ERR_BAD_SHAPE;
    if ((l->norm != 0 && l->norm != 1) || (l->wide_gradient != 0 && l->wide_gradient != 1)) return FH_ERR_BAD_PARAM;
    if ((l->kept_for & ~kNeeds) != 0 || (l->kept_for && (l->needs & ~l->kept_for) != 0)) return FH_ERR_BAD_PARAM;
    if ((l->needs & ~kNeeds) != 0 || l->reserved != 0 || (l->norm && !(l->eps >= 0.0f))) return FH_ERR_BAD_PARAM;
    return FH_OK;
}

bool is_wide(const fh_mx_layer& l) { return l.wide_gradient && l.norm && (l.needs & FH_MX_NEEDS_INPUT) && l.dtype != FH_F32; }
Parts parts_of(const fh_mx_layer& l)
{
    return parts_of(l.tokens, l.features, l.out_features, is_wide(l), l.kept_for ? l.kept_for : kNeeds, l.norm || !l.kept_for);
}

uint8_t* at(void* p, size_t offset) { return static_cast<uint8_t*>(p) + offset; }

}  // namespace
}  // namespace fh

extern "C" {

size_t fh_mx_layer_kept_bytes(int64_t tokens, int64_t features, int64_t out_features)
{
    return fh::shape_ok(tokens, features, out_features) ? fh::parts_of(tokens, features, out_features, false, fh::kNeeds, true).kept : 0;
}

size_t fh_mx_layer_scratch_bytes(int64_t tokens, int64_t features, int64_t out_features)
{
    if (!fh::shape_ok(tokens, features, out_features)) return 0;
    const fh::Parts p = fh::parts_of(tokens, features, out_features, false, fh::kNeeds, true);
    return fh::larger(p.forward, p.backward);
}

fh_status fh_mx_layer_sizes(const fh_mx_layer* l, size_t* kept, size_t* forward_scratch, size_t* backward_scratch)
{
    using namespace fh;
    if (!kept || !forward_scratch || !backward_scratch) return FH_ERR_NULL;
    const fh_status ok = check(l);
    if (ok != FH_OK) return ok;
    const Parts p = parts_of(*l);
    *kept = l->needs ? p.kept : 0;
    *forward_scratch = p.forward;
    *backward_scratch = p.backward;
    return FH_OK;
}

fh_status fh_mx_layer_forward(const fh_mx_layer* l, void* stream)
{
    using namespace fh;
    const fh_status ok = check(l);
    if (ok != FH_OK || l->tokens == 0) return ok;
    const Parts p = parts_of(*l);
    const size_t size = dtype_size(l->dtype), p_size = dtype_size(l->p_dtype);
    const bool keeps = l->needs != 0;
    if (!l->x || !l->weight || !l->y || !l->scratch || (keeps && !l->kept)) return FH_ERR_NULL;
    if (!is_aligned(l->x, size) || !is_aligned(l->y, size) || !is_aligned(l->weight, p_size) || !is_aligned(l->bias, p_size) ||
        !is_aligned(l->norm_weight, p_size) || !is_aligned(l->norm_bias, p_size) || !is_aligned(l->kept, 16) || !is_aligned(l->scratch, 16))
        return FH_ERR_ALIGNMENT;
    if (l->scratch_cap < p.forward || (keeps && l->kept_cap < p.kept)) return FH_ERR_BUFFER_TOO_SMALL;

    const fh_dtype dtype = (fh_dtype)l->dtype, p_dtype = (fh_dtype)l->p_dtype;
    uint8_t *x_rows = at(l->scratch, p.x_rows), *w_rows = at(l->scratch, p.w_rows);
    uint8_t* x_columns = l->needs & FH_MX_NEEDS_WEIGHT ? at(l->kept, p.x_columns) : nullptr;
    uint8_t* w_columns = l->needs & FH_MX_NEEDS_INPUT ? at(l->kept, p.w_columns) : nullptr;
    const size_t x_bytes = mx_bytes(l->tokens, l->features), w_bytes = mx_bytes(l->out_features, l->features);
    fh_status s;
    if (l->norm)
        s = fh_layer_norm_mx(l->x, dtype, l->tokens, l->features, l->x_stride, l->norm_weight, l->norm_bias, p_dtype, l->eps, FH_ROUND_NEAREST, 0, 0,
                             x_rows, x_bytes, x_columns, mx_bytes(l->features, l->tokens), keeps ? at(l->kept, p.mean) : nullptr, keeps ? at(l->kept, p.rstd) : nullptr,
                             stream);
    else
        s = fh_mx_quantize(l->x, dtype, l->tokens, l->features, l->x_stride, FH_ROUND_NEAREST, 0, 0, x_rows, x_bytes, x_columns,
                           mx_bytes(l->features, l->tokens), stream);
    if (s != FH_OK) return s;
    s = fh_mx_quantize(l->weight, p_dtype, l->out_features, l->features, l->weight_stride, FH_ROUND_NEAREST, 0, 0, w_rows, w_bytes, w_columns,
                       mx_bytes(l->features, l->out_features), stream);
    if (s != FH_OK) return s;
    const fh_mx_product y = {x_rows, x_bytes, w_rows, w_bytes, l->tokens, l->out_features, l->features, l->bias, l->p_dtype, l->dtype, l->y,
                             l->out_features, (size_t)l->tokens * (size_t)l->out_features * size, at(l->scratch, p.forward_work),
                             l->scratch_cap - p.forward_work, 0};
    return fh_mx_matmul(&y, stream);
}

fh_status fh_mx_layer_backward(const fh_mx_layer* l, void* stream)
{
    using namespace fh;
    const fh_status ok = check(l);
    if (ok != FH_OK || (!l->needs && !l->dbias)) return ok;
    const Parts p = parts_of(*l);
    const size_t size = dtype_size(l->dtype), p_size = dtype_size(l->p_dtype);
    const bool input = l->needs & FH_MX_NEEDS_INPUT, weight = l->needs & FH_MX_NEEDS_WEIGHT;
    if ((l->needs && p.kept && !l->kept) || (p.backward && !l->scratch) || (weight && !l->dweight)) return FH_ERR_NULL;
    if (l->tokens > 0 && (!l->dy || (input && !l->dx) || (input && l->norm && !l->x))) return FH_ERR_NULL;
    if (!is_aligned(l->x, size) || !is_aligned(l->dy, size) || !is_aligned(l->dx, size) || !is_aligned(l->dweight, p_size) ||
        !is_aligned(l->norm_weight, p_size) || !is_aligned(l->dnorm_weight, p_size) || !is_aligned(l->dnorm_bias, p_size) ||
        !is_aligned(l->dbias, p_size) || !is_aligned(l->kept, 16) || !is_aligned(l->scratch, 16)) return FH_ERR_ALIGNMENT;
    if (l->scratch_cap < p.backward || (l->needs && l->kept_cap < p.kept)) return FH_ERR_BUFFER_TOO_SMALL;

    uint8_t *dy_rows = input ? at(l->scratch, p.dy_rows) : nullptr, *dy_columns = weight ? at(l->scratch, p.dy_columns) : nullptr;
    const size_t rows_bytes = mx_bytes(l->tokens, l->out_features), columns_bytes = mx_bytes(l->out_features, l->tokens);
    void* work = at(l->scratch, p.backward_work);
    const size_t work_bytes = l->scratch_cap - p.backward_work;
    fh_status s;
    if (l->dbias) {                                              // in the workspace until the sums are joined, ahead of the products
        const hipStream_t hs = static_cast<hipStream_t>(stream);
        float* sums = static_cast<float*>(work);
        if (l->tokens > 0 && launch_mx_tiles(l->dy, l->dtype, l->tokens, l->out_features, l->dy_stride, nullptr, sums, l->rounding == FH_ROUND_STOCHASTIC, l->seed,
                                             l->tensor_id, dy_rows, dy_columns, hs) != hipSuccess) return FH_ERR_LAUNCH;
        if (launch_join(sums, mx_tile_rows(l->tokens), l->out_features, 1, l->p_dtype, l->dbias, nullptr, hs) != hipSuccess) return FH_ERR_LAUNCH;
        if (!l->needs) return FH_OK;
    } else {
        s = fh_mx_quantize(l->dy, (fh_dtype)l->dtype, l->tokens, l->out_features, l->dy_stride, l->rounding, l->seed, l->tensor_id,
                           dy_rows, rows_bytes, dy_columns, columns_bytes, stream);
        if (s != FH_OK) return s;
    }
    if (weight) {
        const fh_mx_product dw = {dy_columns, columns_bytes, at(l->kept, p.x_columns), mx_bytes(l->features, l->tokens), l->out_features, l->features,
                                  l->tokens, nullptr, l->p_dtype, l->p_dtype, l->dweight, l->features,
                                  (size_t)l->out_features * (size_t)l->features * p_size, work, work_bytes, 0};
        if ((s = fh_mx_matmul(&dw, stream)) != FH_OK) return s;
    }
    if (!input) return FH_OK;
    // With a norm its output's gradient stays in binary32 on the way, or is rounded to dtype as between two layers of their own: in bf16 dx is then
    // 0.0024 of its norm from the exact one instead of 0.0017, the norm's parameters have sums of rounded values for gradients, and 8192 x 768 values
    // go through memory as 25 MB instead of 50 (a step of 8192 x 768 tokens to 2304: 97.5 and 102.3 us).
    const bool wide = is_wide(*l);
    const int32_t dh_dtype = wide ? FH_F32 : l->dtype;
    void* dh = wide ? at(l->scratch, p.dh) : l->dx;
    const size_t values = (size_t)l->tokens * (size_t)l->features;
    const fh_mx_product dx = {dy_rows, rows_bytes, at(l->kept, p.w_columns), mx_bytes(l->features, l->out_features), l->tokens, l->features,
                              l->out_features, nullptr, l->p_dtype, dh_dtype, dh, l->features, values * dtype_size(dh_dtype), work, work_bytes, 0};
    if ((s = fh_mx_matmul(&dx, stream)) != FH_OK || !l->norm) return s;
    const fh_norm_backward n = {dh, l->x, l->features, l->x_stride, at(l->kept, p.mean), at(l->kept, p.rstd), l->norm_weight, l->tokens, l->features,
                                l->dtype, l->p_dtype, l->dx, l->features, values * size, l->dnorm_weight, l->dnorm_bias, work, work_bytes};
    return norm_backward(n, dh_dtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"
