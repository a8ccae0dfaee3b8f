// Products of matrices in 8-bit integers: the plain one, and the gated projection.
#include "fh_product.hpp"

namespace fh {
namespace {

template <Made MADE>
hipError_t q8_product(const ProductArgs& p, int32_t out_dtype, hipStream_t s)
{
    if (few_rows_of_bytes(p.m, MADE != Made::linear)) return out_dtype == FH_F32 ? product_rows<OfQ8, MADE, float>(p, s) : product_rows<OfQ8, MADE, Bf16>(p, s);
    const ProductTile tile = product_tile(p.m, MADE == Made::linear ? p.n : 2 * (int64_t)p.n, p.chunks, false);
    return out_dtype == FH_F32 ? product_by<OfQ8, MADE, float>(tile, p, s) : product_by<OfQ8, MADE, Bf16>(tile, p, s);
}

bool q8_product_shape_ok(int64_t m, int64_t n, int64_t k) { return q8_shape_ok(m, k) && q8_shape_ok(n, k) && k <= kQ8MostSummed; }

ProductArgs q8_args(const void* a, int64_t m, int64_t n, int64_t k, void* out, int64_t stride)
{
    ProductArgs p = {};
    p.a = static_cast<const uint8_t*>(a);
    p.a_pitch = p.b_pitch = p.b2_pitch = (uint32_t)(q8_chunks(k) * kQ8Chunk);
    p.chunks = p.chunks_each = (uint32_t)q8_chunks(k);
    p.tail = kChunkBytes;
    p.parts = 1;
    p.m = (uint32_t)m;
    p.n = (uint32_t)n;
    p.out = out;
    p.stride = stride;
    return p;
}

}  // namespace
}  // namespace fh

extern "C" {

// No kernel here lays anything out: a workspace is taken, as by the other products, and left alone.
size_t fh_q8_matmul_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }
size_t fh_q8_gated_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

fh_status fh_q8_matmul(const fh_q8_product* q, void* stream)
{
    using namespace fh;
    if (!q) return FH_ERR_NULL;
    if (!is_dtype(q->out_dtype) || !is_dtype(q->bias_dtype)) return FH_ERR_BAD_DTYPE;
    if (!q8_product_shape_ok(q->m, q->n, q->k) || q->stride < q->n || q->stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (q->reserved != 0) return FH_ERR_BAD_PARAM;
    if (q->m == 0 || q->n == 0) return FH_OK;
    if (!q->out || (q->k > 0 && (!q->a || !q->b))) return FH_ERR_NULL;
    const size_t size = dtype_size(q->out_dtype);
    if (!is_aligned(q->a, 16) || !is_aligned(q->b, 16) || !is_aligned(q->out, size) || !is_aligned(q->bias, dtype_size(q->bias_dtype)) ||
        !is_aligned(q->workspace, 16)) return FH_ERR_ALIGNMENT;
    if (q->a_cap < q8_bytes(q->m, q->k) || q->b_cap < q8_bytes(q->n, q->k) || q->out_cap < strided_elements(q->m, q->n, q->stride) * size)
        return FH_ERR_BUFFER_TOO_SMALL;
    ProductArgs p = q8_args(q->a, q->m, q->n, q->k, q->out, q->stride);
    p.b = static_cast<const uint8_t*>(q->b);
    p.bias = q->bias;
    p.bias_dtype = (int16_t)q->bias_dtype;
    return q8_product<Made::linear>(p, q->out_dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

fh_status fh_q8_gated(const fh_q8_gated_product* q, void* stream)
{
    using namespace fh;
    if (!q) return FH_ERR_NULL;
    if (!is_dtype(q->out_dtype) || !is_dtype(q->bias_dtype)) return FH_ERR_BAD_DTYPE;
    if (!q8_product_shape_ok(q->m, q->n, q->k) || q->stride < q->n || q->stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (!is_activation(q->activation) || q->reserved != 0 || q->reserved2 != 0) return FH_ERR_BAD_PARAM;
    if (q->m == 0 || q->n == 0) return FH_OK;
    if (!q->out || (q->k > 0 && (!q->x || !q->gate || !q->up))) return FH_ERR_NULL;
    const size_t size = dtype_size(q->out_dtype), bias = dtype_size(q->bias_dtype);
    if (!is_aligned(q->x, 16) || !is_aligned(q->gate, 16) || !is_aligned(q->up, 16) || !is_aligned(q->out, size) || !is_aligned(q->gate_bias, bias) ||
        !is_aligned(q->up_bias, bias) || !is_aligned(q->workspace, 16)) return FH_ERR_ALIGNMENT;
    if (q->x_cap < q8_bytes(q->m, q->k) || q->gate_cap < q8_bytes(q->n, q->k) || q->up_cap < q8_bytes(q->n, q->k) ||
        q->out_cap < strided_elements(q->m, q->n, q->stride) * size) return FH_ERR_BUFFER_TOO_SMALL;
    ProductArgs p = q8_args(q->x, q->m, q->n, q->k, q->out, q->stride);
    p.b = static_cast<const uint8_t*>(q->gate);
    p.b2 = static_cast<const uint8_t*>(q->up);
    p.bias = q->gate_bias;
    p.bias2 = q->up_bias;
    p.bias_dtype = (int16_t)q->bias_dtype;
    p.act = (int16_t)q->activation;
    return q8_product<Made::gated>(p, q->out_dtype, static_cast<hipStream_t>(stream)) == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

}  // extern "C"
