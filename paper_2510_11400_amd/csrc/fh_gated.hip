// The gated projection h = act(x Wg^T + bg) * (x Wu^T + bu) of dense matrices, and its backward pass.
//
// Backward, from x, the weights and dh alone, by three products:
//   D  = [dg | du]: the forward product again, and in its epilogue dg = dh up act'(gate), du = dh act(gate); rounded to the layer's type, in which
//        the products behind take it (up to a relative 2^-8 a value in bf16, as much as the results' own rounding; small layers keep what it leaves);
//   dx = D [Wg; Wu]
//   [dWg; dWu] = D^T x
// and the biases' gradients are sums of D's columns before that rounding: partial sums by tiles of rows, joined in order.  Operands whose rows are the
// summed dimension (the weights of dx, D and x of dW) are read as they lie and transposed on their way from LDS to registers; copying them to the other
// order first took 8192 tokens of 768 -> 2048 in bf16 70 us of 283.  dW has few outputs and a sum over all tokens: several workgroups share a tile's.
#include "fh_product.hpp"

namespace fh {
namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 21, kMostFeatures = (int64_t)1 << 20;   // 256 rows are addressed with 32 bits
constexpr int64_t kMostPitch = (int64_t)1 << 23;                                    // bytes

int64_t chunk_values(int32_t dtype) { return kChunkBytes / (int64_t)dtype_size(dtype); }
int64_t padded_bytes(int64_t cols, int32_t dtype) { return (cols * (int64_t)dtype_size(dtype) + kChunkBytes - 1) / kChunkBytes * kChunkBytes; }
size_t aligned(size_t n) { return (n + 255) & ~(size_t)255; }

// ---- operands as the products want them ----------------------------------------------------------
// Rows of any alignment and length to rows of whole chunks, zeros behind their ends: up to three matrices of as many columns, a workgroup a row, sixteen
// bytes a thread.  (A launch for each took 333 x 515 -> 1001 in fp32, a step, 8 us longer; this one takes 4.3 us for 9.6 MB read and written.)
struct PackArgs {
    const void* x[3];
    uint8_t*    out[3];
    int64_t     stride[3];
    uint32_t    end[3];                // workgroups of the matrices up to this one
    uint32_t    cols, pitch, first;
};
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackArgs p)
{
    constexpr int kRun = 16 / sizeof(T);
    const uint32_t number = p.first + blockIdx.x, which = (number >= p.end[0]) + (number >= p.end[1]);
    const uint32_t row = number - (which == 0 ? 0u : which == 1 ? p.end[0] : p.end[1]);
    const T* x = static_cast<const T*>(which == 0 ? p.x[0] : which == 1 ? p.x[1] : p.x[2]) + (int64_t)row * (which == 0 ? p.stride[0] : which == 1 ? p.stride[1] : p.stride[2]);
    uint8_t* out = (which == 0 ? p.out[0] : which == 1 ? p.out[1] : p.out[2]) + (int64_t)row * p.pitch;
    for (uint32_t i = threadIdx.x; i < p.pitch / 16; i += 256) {
        Run<T, kRun> v;
        v.load(x + (int64_t)i * kRun, (int64_t)p.cols - (int64_t)i * kRun);
        *reinterpret_cast<u32x4*>(out + i * 16) = u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
    }
}
template <typename T>
__global__ __launch_bounds__(64) void clear_rows_kernel(T* out, uint32_t cols)
{
    for (uint32_t c = threadIdx.x; c < cols; c += 64) out[(int64_t)blockIdx.x * cols + c] = T{};
}
// The parts of a shared sum, each `hidden_padded` + hidden rows of cols, added up in their order: the first `hidden` rows and the last.  Bound by the memory
// that the parts come from, the memory-side cache as a rule: two parts of 4096 x 768 to bf16 take 6.6 us, 4.8 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void join_weights_kernel(const float* parts, uint32_t count, uint32_t hidden, uint32_t hidden_padded, uint32_t cols, uint32_t runs, T* gate, T* up)
{
    const uint32_t at = blockIdx.x * 256 + threadIdx.x, number = at / runs, col = (at - number * runs) * 4;
    if (number >= 2 * hidden) return;
    const uint32_t second = number >= hidden, row = second ? number - hidden : number, all = hidden_padded + hidden;
    const float* from = parts + (int64_t)(second ? hidden_padded + row : row) * cols + col;
    float v[4] = {};
    for (uint32_t k = 0; k < count; ++k) {
        float w[4];
        load4(from + (int64_t)k * all * cols, (int64_t)cols - col, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += w[i];
    }
    store4((second ? up : gate) + (int64_t)row * cols + col, (int64_t)cols - col, v);
}

// A matrix as an operand: as it lies, or packed.  As it lies where every row, and its end, is at a multiple of 16 bytes.
struct Rows { const void* p; int64_t rows, cols, stride; };
bool lies_well(const Rows& r, int32_t dtype)
{
    const int64_t size = (int64_t)dtype_size(dtype), pitch = r.stride * size;
    return is_aligned(r.p, 16) && r.cols * size % 16 == 0 && (r.rows <= 1 || (pitch % 16 == 0 && pitch <= kMostPitch));
}
size_t packed_bytes(const Rows& r, int32_t dtype) { return lies_well(r, dtype) ? 0 : aligned((size_t)r.rows * (size_t)padded_bytes(r.cols, dtype)); }

struct Forward { Rows x, gate, up; };
Forward forward_rows(const fh_gated_layer& l)
{
    return {{l.x, l.tokens, l.features, l.x_stride}, {l.w_gate, l.hidden, l.features, l.w_gate_stride}, {l.w_up, l.hidden, l.features, l.w_up_stride}};
}
size_t forward_bytes(const fh_gated_layer& l)                    // of the products that want their operands laid out
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

// The kernel of the products of a layer's pairs of sums.
ProductTile pair_tile(const fh_gated_layer& l, ProductTile last = ProductTile::square256)
{
    return product_tile(l.tokens, 2 * l.hidden, padded_bytes(l.features, l.dtype) / kChunkBytes, l.dtype == FH_F32, last);
}

// The chunks of rows of `values`.
template <typename T>
void set_summed(ProductArgs& p, int64_t values)
{
    const int64_t bytes = values * (int64_t)sizeof(T);
    p.chunks = p.chunks_each = (uint32_t)((bytes + kChunkBytes - 1) / kChunkBytes);
    p.tail = (uint32_t)((bytes + 15) / 16 * 16 - (int64_t)(p.chunks - 1) * kChunkBytes);
    p.parts = 1;
}

template <typename T>
void set_layer(const fh_gated_layer& l, ProductArgs& p)
{
    set_summed<T>(p, l.features);
    p.m = (uint32_t)l.tokens;
    p.n = (uint32_t)l.hidden;
    p.bias = l.b_gate;
    p.bias2 = l.b_up;
    p.bias_dtype = (int16_t)l.dtype;
    p.act = (int16_t)l.activation;
}
// Whether a few tokens' forward product takes its operands as they lie, at any alignment; its arguments hold strides in 32 bits.
bool forward_as_it_lies(const fh_gated_layer& l)
{
    const int64_t most = ((int64_t)1 << 32) / (int64_t)dtype_size(l.dtype);
    return few_rows_dense(l.tokens, l.dtype == FH_F32, forward_bytes(l) > 0) && l.x_stride < most && l.w_gate_stride < most && l.w_up_stride < most;
}

// The operands of the forward product.
template <typename T>
hipError_t forward_operands(const fh_gated_layer& l, ProductArgs& p, Space& space, hipStream_t s)
{
    const Forward f = forward_rows(l);
    PackArgs q = {};
    q.cols = (uint32_t)l.features;
    q.pitch = (uint32_t)padded_bytes(l.features, l.dtype);
    int count = 0;
    uint32_t all = 0;
    const auto take = [&](const Rows& r, const uint8_t*& at, uint32_t& pitch) {
        if (lies_well(r, l.dtype)) {
            at = static_cast<const uint8_t*>(r.p);
            pitch = (uint32_t)((r.rows <= 1 ? r.cols : r.stride) * (int64_t)sizeof(T));
            return;
        }
        uint8_t* to = space.take(packed_bytes(r, l.dtype));
        at = to;
        pitch = q.pitch;
        q.x[count] = r.p;
        q.out[count] = to;
        q.stride[count] = r.stride;
        all += (uint32_t)r.rows;
        for (int i = count++; i < 3; ++i) q.end[i] = all;
    };
    take(f.x, p.a, p.a_pitch);
    take(f.gate, p.b, p.b_pitch);
    take(f.up, p.b2, p.b2_pitch);
    const hipError_t e = in_parts(all, 256, [&](int64_t first, int64_t some) {
        q.first = (uint32_t)first;
        return launch(pack_kernel<T>, dim3((uint32_t)some), dim3(256), s, q);
    });
    set_layer<T>(l, p);
    return e;
}

template <typename T>
hipError_t forward_of(const fh_gated_layer& l, hipStream_t s)
{
    ProductArgs p = {};
    Space space = {static_cast<uint8_t*>(l.workspace)};
    p.out = l.h;
    p.stride = l.h_stride;
    if (forward_as_it_lies(l)) {
        const Forward f = forward_rows(l);
        const auto pitch = [](const Rows& r) { return r.rows <= 1 ? 0u : (uint32_t)(r.stride * (int64_t)sizeof(T)); };
        p.a = static_cast<const uint8_t*>(f.x.p);
        p.b = static_cast<const uint8_t*>(f.gate.p);
        p.b2 = static_cast<const uint8_t*>(f.up.p);
        p.a_pitch = pitch(f.x);
        p.b_pitch = pitch(f.gate);
        p.b2_pitch = pitch(f.up);
        set_layer<T>(l, p);
        p.tail = (uint32_t)(l.features * (int64_t)sizeof(T) - (int64_t)(p.chunks - 1) * kChunkBytes);
        return product_rows<typename OpOf<T>::type, Made::gated, T>(p, s);
    }
    const hipError_t e = forward_operands<T>(l, p, space, s);
    if (e != hipSuccess) return e;
    return product_by<typename OpOf<T>::type, Made::gated, T>(pair_tile(l), p, s);
}

// What the backward call lays out in its workspace.
struct Backward {
    int64_t hidden_padded;             // columns of D's halves: whole chunks, so that the products over them have no tails, zeros behind the last
    bool rests;                        // D's rows are [dg | du | what their rounding left of each]
    int64_t d_columns;                 // of a row of D
    ProductTile pair, last;            // the first product's kernel; the last one that the products may take
    int64_t sum_rows;                  // rows that a partial sum of the biases' gradients stands for
    ProductPlan weights;
    size_t d, sums, parts, forward;
    size_t bytes() const { return d + sums + parts + forward; }
};
Backward backward_of(const fh_gated_layer& l)
{
    const size_t size = dtype_size(l.dtype);
    Backward b = {};
    b.hidden_padded = padded_bytes(l.hidden, l.dtype) / (int64_t)size;
    b.rests = product_with_rests(l.tokens, l.features, l.hidden, l.dtype == FH_F32);
    b.last = product_last(b.rests);
    b.pair = pair_tile(l, b.last);
    b.sum_rows = product_sum_rows(b.pair);
    b.d_columns = (b.rests ? 4 : 2) * b.hidden_padded;
    b.d = aligned((size_t)l.tokens * (size_t)b.d_columns * size);
    if (l.db_gate || l.db_up) b.sums = aligned((size_t)((l.tokens + b.sum_rows - 1) / b.sum_rows) * 2u * (size_t)l.hidden * 4u);
    if (l.needs & FH_GATED_NEEDS_WEIGHT) {
        const int64_t m = b.hidden_padded + l.hidden;
        b.weights = product_plan(m, l.features, (b.rests ? 2 : 1) * padded_bytes(l.tokens, l.dtype) / kChunkBytes, l.dtype == FH_F32, true, b.last);
        if (b.weights.parts > 1) b.parts = aligned((size_t)b.weights.parts * (size_t)m * (size_t)l.features * 4u);
    }
    b.forward = forward_bytes(l);
    return b;
}

// Zeros to `n` values: the gradients of no tokens.
template <typename T>
hipError_t clear(void* out, int64_t rows, int64_t cols, hipStream_t s)
{
    if (!out) return hipSuccess;
    return in_parts(rows, 64, [&](int64_t first, int64_t count) {
        return launch(clear_rows_kernel<T>, dim3((uint32_t)count), dim3(64), s, static_cast<T*>(out) + first * cols, (uint32_t)cols);
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
    float* sums = reinterpret_cast<float*>(space.take(b.sums));
    float* parts = reinterpret_cast<float*>(space.take(b.parts));
    typedef typename OpOf<T>::type Op;

    BackwardArgs p = {};
    e = forward_operands<T>(l, p, space, s);
    if (e != hipSuccess) return e;
    p.out = d;
    p.stride = b.d_columns;
    p.dh = l.dh;
    p.dh_stride = l.dh_stride;
    p.up_at = b.hidden_padded;
    p.rest_at = b.rests ? 2 * b.hidden_padded : 0;
    p.sums = b.sums ? sums : nullptr;
    e = product_by<Op, Made::gated_backward, T>(b.pair, p, s);
    if (e == hipSuccess && b.sums) e = launch_join(sums, (l.tokens + b.sum_rows - 1) / b.sum_rows, l.hidden, 2, l.dtype, l.db_gate, l.db_up, s);

    if (e == hipSuccess && (l.needs & FH_GATED_NEEDS_INPUT)) {
        TurnedArgs q = {};
        q.a = reinterpret_cast<const uint8_t*>(d);
        q.a_pitch = (uint32_t)(b.d_columns * size);
        set_summed<T>(q, b.d_columns);
        q.b = p.b;
        q.b2 = p.b2;
        q.b_pitch = p.b_pitch;
        q.b2_pitch = p.b2_pitch;
        q.summed = (uint32_t)l.hidden;
        q.halves = b.rests;
        q.rest = (uint32_t)(2 * b.hidden_padded * size);
        q.split = q.rest / 2 / kChunkBytes;
        q.gap_from = (uint32_t)l.tokens;
        q.m = (uint32_t)l.tokens;
        q.n = (uint32_t)l.features;
        q.out = l.dx;
        q.stride = l.features;
        e = product_by<Op, Made::linear, T, Lies::rows, Lies::columns>(product_tile(q.m, q.n, q.chunks, sizeof(T) == 4, b.last), q, s);
    }
    if (e == hipSuccess && (l.needs & FH_GATED_NEEDS_WEIGHT)) {
        TurnedArgs q = {};
        q.a = reinterpret_cast<const uint8_t*>(d);
        q.a_pitch = (uint32_t)(b.d_columns * size);
        q.b = p.a;
        q.b_pitch = p.a_pitch;
        set_summed<T>(q, l.tokens);
        q.summed = (uint32_t)l.tokens;
        q.split = q.chunks;
        q.halves = b.rests;
        if (b.rests) q.chunks = q.chunks_each = 2 * q.chunks;
        q.rest = (uint32_t)(2 * b.hidden_padded * size);
        q.n = (uint32_t)l.features;
        q.stride = l.features;
        if (b.weights.parts > 1) {
            q.m = q.gap_from = (uint32_t)(b.hidden_padded + l.hidden);
            q.parts = b.weights.parts;
            q.chunks_each = b.weights.chunks_each;
            q.out = parts;
            e = product_by<Op, Made::linear, float, Lies::columns, Lies::columns>(b.weights.tile, q, s);
            const int64_t runs = (l.features + 3) / 4;
            const auto join = [&](int64_t groups) {
                return launch(join_weights_kernel<T>, dim3((uint32_t)groups), dim3(256), s, parts, q.parts, (uint32_t)l.hidden, (uint32_t)b.hidden_padded, q.n, (uint32_t)runs,
                              static_cast<T*>(l.dw_gate), static_cast<T*>(l.dw_up));
            };
            if (e == hipSuccess) e = join((2 * l.hidden * runs + 255) / 256);
            return e;
        }
        // both weights' gradients at once where they lie one behind the other: what D has between its halves is left out
        const bool one = static_cast<T*>(l.dw_up) == static_cast<T*>(l.dw_gate) + l.hidden * l.features;
        q.m = (uint32_t)(one ? b.hidden_padded + l.hidden : l.hidden);
        q.gap_from = (uint32_t)l.hidden;
        q.gap = one ? (uint32_t)(b.hidden_padded - l.hidden) : 0u;
        q.out = l.dw_gate;
        const ProductTile tile = b.weights.tile;                 // wherever they lie: the same sums
        e = product_by<Op, Made::linear, T, Lies::columns, Lies::columns>(tile, q, s);
        if (e == hipSuccess && !one) {
            q.a += b.hidden_padded * size;
            q.out = l.dw_up;
            e = product_by<Op, Made::linear, T, Lies::columns, Lies::columns>(tile, q, s);
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
    return backward ? backward_of(*l).bytes() : forward_as_it_lies(*l) ? 0 : forward_bytes(*l);
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
    if ((status = check_workspace(*l, forward_as_it_lies(*l) ? 0 : forward_bytes(*l))) != FH_OK) return status;
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
