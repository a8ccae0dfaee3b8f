// The gated projection h = act(x Wg^T + bg) * (x Wu^T + bu) of dense matrices, and its backward pass.
//
// Backward, from x, the weights and dh alone, by three products:
//   D  = [dg | du]: the forward product again, and in its epilogue dg = dh up act'(gate), du = dh act(gate); rounded to the layer's type, in which
//        the products behind take it (a relative 2^-9 a value in bf16, as much as the results' own rounding);
//   dx = D [Wg; Wu]
//   [dWg; dWu] = D^T x
// and the biases' gradients are sums of D's columns before that rounding: partial sums by tiles of rows, joined in order.
#include "fh_product.hpp"

namespace fh {
namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 21, kMostFeatures = (int64_t)1 << 20;   // 256 rows are addressed with 32 bits
constexpr int64_t kMostPitch = (int64_t)1 << 23;                                    // bytes

int64_t chunk_values(int32_t dtype) { return kChunkBytes / (int64_t)dtype_size(dtype); }
int64_t padded_bytes(int64_t cols, int32_t dtype) { return (cols * (int64_t)dtype_size(dtype) + kChunkBytes - 1) / kChunkBytes * kChunkBytes; }
size_t aligned(size_t n) { return (n + 255) & ~(size_t)255; }

// ---- operands as the products want them ----------------------------------------------------------
// Rows of any alignment and length to rows of whole chunks, zeros behind their ends.  Sixteen bytes a thread.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(const T* x, uint32_t cols, int64_t stride, uint8_t* out, uint32_t pitch, uint32_t rows, uint32_t first)
{
    constexpr int kRun = 16 / sizeof(T);
    const uint32_t pieces = pitch / 16, row = first + blockIdx.x;
    for (uint32_t i = threadIdx.x; i < pieces; i += 256) {
        Run<T, kRun> v;
        v.load(x + (int64_t)row * stride + (int64_t)i * kRun, (int64_t)cols - (int64_t)i * kRun);
        *reinterpret_cast<u32x4*>(out + (int64_t)row * pitch + i * 16) = u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
    }
}
// The transposed matrix: out[c][r] = x[r][c], row c from byte c * pitch on; r goes to `padded` with zeros behind `rows`.  Tiles of 64 x 64.
template <typename T>
__global__ __launch_bounds__(256) void transpose_kernel(const T* x, uint32_t rows, uint32_t cols, int64_t stride, T* out, int64_t out_stride, uint32_t padded,
                                                        uint32_t across, uint32_t first)
{
    __shared__ T s_tile[64][65];
    const uint32_t tile = first + blockIdx.x, r0 = tile / across * 64, c0 = tile % across * 64;
    for (uint32_t i = threadIdx.x; i < 64 * 64; i += 256) {
        const uint32_t r = i / 64, c = i % 64;
        s_tile[r][c] = r0 + r < rows && c0 + c < cols ? x[(int64_t)(r0 + r) * stride + c0 + c] : T{};
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 64 * 64; i += 256) {
        const uint32_t c = i / 64, r = i % 64;
        if (c0 + c < cols && r0 + r < padded) out[(int64_t)(c0 + c) * out_stride + r0 + r] = s_tile[r][c];
    }
}
// Columns from..to of every row: zeros.
template <typename T>
__global__ __launch_bounds__(64) void clear_columns_kernel(T* out, int64_t stride, uint32_t from, uint32_t to)
{
    for (uint32_t c = from + threadIdx.x; c < to; c += 64) out[(int64_t)blockIdx.x * stride + c] = T{};
}

template <typename T>
hipError_t pack(const void* x, int64_t rows, int64_t cols, int64_t stride, void* out, hipStream_t s)
{
    const uint32_t pitch = (uint32_t)padded_bytes(cols, sizeof(T) == 4 ? FH_F32 : FH_BF16);
    return in_parts(rows, 256, [&](int64_t first, int64_t count) {
        return launch(pack_kernel<T>, dim3((uint32_t)count), dim3(256), s, static_cast<const T*>(x), (uint32_t)cols, stride, static_cast<uint8_t*>(out), pitch,
                      (uint32_t)rows, (uint32_t)first);
    });
}
template <typename T>
hipError_t transpose(const void* x, int64_t rows, int64_t cols, int64_t stride, T* out, int64_t out_stride, int64_t padded, hipStream_t s)
{
    const int64_t across = (cols + 63) / 64, tiles = (padded + 63) / 64 * across;
    return in_parts(tiles, 256, [&](int64_t first, int64_t count) {
        return launch(transpose_kernel<T>, dim3((uint32_t)count), dim3(256), s, static_cast<const T*>(x), (uint32_t)rows, (uint32_t)cols, stride, out, out_stride,
                      (uint32_t)padded, (uint32_t)across, (uint32_t)first);
    });
}

// A matrix as an operand: as it lies, or packed.
struct Rows { const void* p; int64_t rows, cols, stride; };
bool lies_well(const Rows& r, int32_t dtype)
{
    const int64_t size = (int64_t)dtype_size(dtype), pitch = r.stride * size;
    return is_aligned(r.p, 16) && r.cols * size % kChunkBytes == 0 && (r.rows <= 1 || (pitch % 16 == 0 && pitch <= kMostPitch));
}
size_t packed_bytes(const Rows& r, int32_t dtype) { return lies_well(r, dtype) ? 0 : aligned((size_t)r.rows * (size_t)padded_bytes(r.cols, dtype)); }

struct Forward { Rows x, gate, up; };
Forward forward_rows(const fh_gated_layer& l)
{
    return {{l.x, l.tokens, l.features, l.x_stride}, {l.w_gate, l.hidden, l.features, l.w_gate_stride}, {l.w_up, l.hidden, l.features, l.w_up_stride}};
}
size_t forward_bytes(const fh_gated_layer& l)
{
    const Forward f = forward_rows(l);
    return packed_bytes(f.x, l.dtype) + packed_bytes(f.gate, l.dtype) + packed_bytes(f.up, l.dtype);
}

// Pieces of the workspace in turn.
struct Space {
    uint8_t* p;
    uint8_t* take(size_t n)
    {
        uint8_t* at = p;
        p += aligned(n);
        return at;
    }
};

template <typename T> struct OpOf;
template <> struct OpOf<float> { typedef OfF32 type; };
template <> struct OpOf<Bf16> { typedef OfBf16 type; };

template <Made MADE, typename T>
hipError_t gated_product(const typename ArgsOf<MADE>::type& p, hipStream_t s)
{
    return product_of<typename OpOf<T>::type, MADE, T>(p, s);
}

// The operands of the forward product.
template <typename T>
hipError_t forward_operands(const fh_gated_layer& l, ProductArgs& p, Space& space, hipStream_t s)
{
    const Forward f = forward_rows(l);
    const auto take = [&](const Rows& r, const uint8_t*& at, uint32_t& pitch) -> hipError_t {
        if (lies_well(r, l.dtype)) {
            at = static_cast<const uint8_t*>(r.p);
            pitch = r.rows <= 1 ? 0u : (uint32_t)(r.stride * (int64_t)sizeof(T));
            return hipSuccess;
        }
        uint8_t* to = space.take(packed_bytes(r, l.dtype));
        at = to;
        pitch = (uint32_t)padded_bytes(r.cols, l.dtype);
        return pack<T>(r.p, r.rows, r.cols, r.stride, to, s);
    };
    hipError_t e = take(f.x, p.a, p.a_pitch);
    if (e == hipSuccess) e = take(f.gate, p.b, p.b_pitch);
    if (e == hipSuccess) e = take(f.up, p.b2, p.b2_pitch);
    p.chunks = (uint32_t)(padded_bytes(l.features, l.dtype) / kChunkBytes);
    p.m = (uint32_t)l.tokens;
    p.n = (uint32_t)l.hidden;
    p.bias = l.b_gate;
    p.bias2 = l.b_up;
    p.bias_dtype = (int16_t)l.dtype;
    p.act = (int16_t)l.activation;
    return e;
}

template <typename T>
hipError_t forward_of(const fh_gated_layer& l, hipStream_t s)
{
    ProductArgs p = {};
    Space space = {static_cast<uint8_t*>(l.workspace)};
    const hipError_t e = forward_operands<T>(l, p, space, s);
    if (e != hipSuccess) return e;
    p.out = l.h;
    p.stride = l.h_stride;
    return gated_product<Made::gated, T>(p, s);
}

// What the backward call lays out in its workspace.
struct Backward {
    int64_t d_values;                  // of a row of D
    int64_t tokens_padded;             // of a row of D^T and x^T
    int64_t tile_rows;                 // rows that a partial sum of the biases' gradients stands for
    size_t d, d_turned, x_turned, w_turned, sums, forward;
    size_t bytes() const { return d + d_turned + x_turned + w_turned + sums + forward; }
};
Backward backward_of(const fh_gated_layer& l)
{
    const size_t size = dtype_size(l.dtype);
    Backward b = {};
    b.d_values = padded_bytes(2 * l.hidden, l.dtype) / (int64_t)size;
    b.tokens_padded = padded_bytes(l.tokens, l.dtype) / (int64_t)size;
    b.tile_rows = product_sum_rows(product_plan(l.tokens, 2 * l.hidden, padded_bytes(l.features, l.dtype) / kChunkBytes, l.dtype == FH_F32));
    b.d = aligned((size_t)l.tokens * (size_t)b.d_values * size);
    if (l.needs & FH_GATED_NEEDS_WEIGHT) {
        b.d_turned = aligned((size_t)(2 * l.hidden) * (size_t)b.tokens_padded * size);
        b.x_turned = aligned((size_t)l.features * (size_t)b.tokens_padded * size);
    }
    if (l.needs & FH_GATED_NEEDS_INPUT) b.w_turned = aligned((size_t)l.features * (size_t)b.d_values * size);
    if (l.db_gate || l.db_up) b.sums = aligned((size_t)((l.tokens + b.tile_rows - 1) / b.tile_rows) * 2u * (size_t)l.hidden * 4u);
    b.forward = forward_bytes(l);
    return b;
}

// Zeros to `n` values: the gradients of no tokens.
template <typename T>
hipError_t clear(void* out, int64_t rows, int64_t cols, hipStream_t s)
{
    if (!out) return hipSuccess;
    return in_parts(rows, 64, [&](int64_t first, int64_t count) {
        return launch(clear_columns_kernel<T>, dim3((uint32_t)count), dim3(64), s, static_cast<T*>(out) + first * cols, cols, 0u, (uint32_t)cols);
    });
}

template <typename T>
hipError_t backward_of(const fh_gated_layer& l, hipStream_t s)
{
    constexpr int64_t size = sizeof(T);
    hipError_t e = hipSuccess;
    if (l.tokens == 0) {
        if (l.needs & FH_GATED_NEEDS_WEIGHT) {
            e = clear<T>(l.dw_gate, l.hidden, l.features, s);
            if (e == hipSuccess) e = clear<T>(l.dw_up, l.hidden, l.features, s);
        }
        if (e == hipSuccess) e = clear<T>(l.db_gate, 1, l.hidden, s);
        if (e == hipSuccess) e = clear<T>(l.db_up, 1, l.hidden, s);
        return e;
    }
    const Backward b = backward_of(l);
    Space space = {static_cast<uint8_t*>(l.workspace)};
    T* d = reinterpret_cast<T*>(space.take(b.d));
    T* d_turned = reinterpret_cast<T*>(space.take(b.d_turned));
    T* x_turned = reinterpret_cast<T*>(space.take(b.x_turned));
    T* w_turned = reinterpret_cast<T*>(space.take(b.w_turned));
    float* sums = reinterpret_cast<float*>(space.take(b.sums));

    BackwardArgs p = {};
    e = forward_operands<T>(l, p, space, s);
    if (e != hipSuccess) return e;
    p.out = d;
    p.stride = b.d_values;
    p.dh = l.dh;
    p.dh_stride = l.dh_stride;
    p.up_at = l.hidden;
    p.sums = b.sums ? sums : nullptr;
    e = gated_product<Made::gated_backward, T>(p, s);
    if (e == hipSuccess && b.sums)
        e = launch_join(sums, (l.tokens + b.tile_rows - 1) / b.tile_rows, l.hidden, 2, l.dtype, l.db_gate, l.db_up, s);

    if (e == hipSuccess && (l.needs & FH_GATED_NEEDS_INPUT)) {
        if (b.d_values > 2 * l.hidden)
            e = in_parts(l.tokens, 64, [&](int64_t first, int64_t count) {
                return launch(clear_columns_kernel<T>, dim3((uint32_t)count), dim3(64), s, d + first * b.d_values, b.d_values, (uint32_t)(2 * l.hidden), (uint32_t)b.d_values);
            });
        if (e == hipSuccess) e = transpose<T>(l.w_gate, l.hidden, l.features, l.w_gate_stride, w_turned, b.d_values, l.hidden, s);
        if (e == hipSuccess) e = transpose<T>(l.w_up, l.hidden, l.features, l.w_up_stride, w_turned + l.hidden, b.d_values, b.d_values - l.hidden, s);
        ProductArgs q = {};
        q.a = reinterpret_cast<const uint8_t*>(d);
        q.b = reinterpret_cast<const uint8_t*>(w_turned);
        q.a_pitch = q.b_pitch = (uint32_t)(b.d_values * size);
        q.chunks = q.a_pitch / kChunkBytes;
        q.m = (uint32_t)l.tokens;
        q.n = (uint32_t)l.features;
        q.out = l.dx;
        q.stride = l.features;
        if (e == hipSuccess) e = gated_product<Made::linear, T>(q, s);
    }
    if (e == hipSuccess && (l.needs & FH_GATED_NEEDS_WEIGHT)) {
        e = transpose<T>(d, l.tokens, 2 * l.hidden, b.d_values, d_turned, b.tokens_padded, b.tokens_padded, s);
        if (e == hipSuccess) e = transpose<T>(l.x, l.tokens, l.features, l.x_stride, x_turned, b.tokens_padded, b.tokens_padded, s);
        ProductArgs q = {};
        q.a = reinterpret_cast<const uint8_t*>(d_turned);
        q.b = reinterpret_cast<const uint8_t*>(x_turned);
        q.a_pitch = q.b_pitch = (uint32_t)(b.tokens_padded * size);
        q.chunks = q.a_pitch / kChunkBytes;
        q.n = (uint32_t)l.features;
        q.stride = l.features;
        // both weights' gradients at once where they lie one behind the other
        const bool one = static_cast<T*>(l.dw_up) == static_cast<T*>(l.dw_gate) + l.hidden * l.features;
        q.m = (uint32_t)(one ? 2 * l.hidden : l.hidden);
        q.out = l.dw_gate;
        if (e == hipSuccess) e = gated_product<Made::linear, T>(q, s);
        if (!one) {
            q.a += l.hidden * (int64_t)q.a_pitch;
            q.out = l.dw_up;
            if (e == hipSuccess) e = gated_product<Made::linear, T>(q, s);
        }
    }
    return e;
}

fh_status check(const fh_gated_layer* l)
{
    if (!l) return FH_ERR_NULL;
    if (!is_dtype(l->dtype)) return FH_ERR_BAD_DTYPE;
    if (l->tokens < 0 || l->tokens > kMostTokens || l->features < 1 || l->features > kMostFeatures || l->hidden < 1 || l->hidden > kMostFeatures) return FH_ERR_BAD_SHAPE;
    if (l->x_stride < l->features || l->w_gate_stride < l->features || l->w_up_stride < l->features || l->x_stride > kMostStride || l->w_gate_stride > kMostStride ||
        l->w_up_stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (!is_activation(l->activation) || (l->needs & ~(FH_GATED_NEEDS_INPUT | FH_GATED_NEEDS_WEIGHT)) || l->reserved != 0) return FH_ERR_BAD_PARAM;
    return FH_OK;
}
fh_status check_inputs(const fh_gated_layer& l)
{
    if (!l.x || !l.w_gate || !l.w_up) return FH_ERR_NULL;
    for (const void* p : {l.x, l.w_gate, l.w_up, l.b_gate, l.b_up})
        if (!is_aligned(p, dtype_size(l.dtype))) return FH_ERR_ALIGNMENT;
    return FH_OK;
}
fh_status check_workspace(const fh_gated_layer& l, size_t need)
{
    if (need && !l.workspace) return FH_ERR_NULL;
    if (!is_aligned(l.workspace, 16)) return FH_ERR_ALIGNMENT;
    return l.workspace_cap < need ? FH_ERR_BUFFER_TOO_SMALL : FH_OK;
}

}  // namespace
}  // namespace fh

extern "C" {

size_t fh_gated_workspace_bytes(const fh_gated_layer* l, int32_t backward)
{
    using namespace fh;
    if (check(l) != FH_OK || l->tokens == 0) return 0;
    return backward ? backward_of(*l).bytes() : forward_bytes(*l);
}

fh_status fh_gated(const fh_gated_layer* l, void* stream)
{
    using namespace fh;
    fh_status status = check(l);
    if (status != FH_OK) return status;
    if (l->h_stride < l->hidden || l->h_stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (l->tokens == 0) return FH_OK;
    if ((status = check_inputs(*l)) != FH_OK) return status;
    if (!l->h) return FH_ERR_NULL;
    if (!is_aligned(l->h, dtype_size(l->dtype))) return FH_ERR_ALIGNMENT;
    if (l->h_cap < strided_elements(l->tokens, l->hidden, l->h_stride) * dtype_size(l->dtype)) return FH_ERR_BUFFER_TOO_SMALL;
    if ((status = check_workspace(*l, forward_bytes(*l))) != FH_OK) return status;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return (l->dtype == FH_F32 ? forward_of<float>(*l, s) : forward_of<Bf16>(*l, s)) == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

fh_status fh_gated_backward(const fh_gated_layer* l, void* stream)
{
    using namespace fh;
    fh_status status = check(l);
    if (status != FH_OK) return status;
    if (l->dh_stride < l->hidden || l->dh_stride > kMostStride) return FH_ERR_BAD_SHAPE;
    const bool input = l->needs & FH_GATED_NEEDS_INPUT, weight = l->needs & FH_GATED_NEEDS_WEIGHT;
    if (!input && !weight && !l->db_gate && !l->db_up) return FH_OK;
    if (weight && (!l->dw_gate || !l->dw_up)) return FH_ERR_NULL;
    for (const void* p : {(const void*)l->dw_gate, (const void*)l->dw_up, (const void*)l->db_gate, (const void*)l->db_up, (const void*)l->dx, l->dh})
        if (!is_aligned(p, dtype_size(l->dtype))) return FH_ERR_ALIGNMENT;
    if (l->tokens > 0) {
        if ((status = check_inputs(*l)) != FH_OK) return status;
        if (!l->dh || (input && !l->dx)) return FH_ERR_NULL;
        if ((status = check_workspace(*l, backward_of(*l).bytes())) != FH_OK) return status;
    }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    return (l->dtype == FH_F32 ? backward_of<float>(*l, s) : backward_of<Bf16>(*l, s)) == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

}  // extern "C"
