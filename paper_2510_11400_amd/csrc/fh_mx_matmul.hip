// The product of two microscaled matrices: out[i][j] = sum_k A[i][k] B[j][k] + bias[j].
#include "fh_norm.hpp"

namespace fh {
namespace {

constexpr int64_t kMostSummed = (int64_t)1 << 24;   // a row's codes are addressed with 32 bits

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct ProductArgs {
    MxStore      a, b;                 // m and n rows, the same number of chunks
    int64_t      m, n, chunks;
    const void*  bias;                 // may be null
    int32_t      bias_dtype;
    void*        out;
    int64_t      stride;
};

// v_mfma_scale_f32_16x16x128_f8f6f4 with 4-bit operands: lane (r = lane % 16, g = lane / 16) brings 32 values of row r of
// each operand with their scale, and gets the outputs [4g .. 4g+3][r].  Any 32 values of the sum may go to any g, the same
// for both operands: of a chunk's eight blocks a lane takes 2g and 2g+1, for one instruction each, whose codes are 32
// contiguous bytes and whose scales lie in one word.
template <int BYTE>
__device__ __forceinline__ f32x4 mx_mfma(u32x4 a, u32x4 b, uint32_t sa, uint32_t sb, f32x4 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, BYTE, (int)sa, BYTE, (int)sb);
}

template <typename T>
__device__ __forceinline__ float bias_of(const ProductArgs& p, int64_t j) { return parameter(p.bias, p.bias_dtype, j, 0.0f); }

// 16 x 16 outputs a workgroup, its waves taking chunks in turn: their sums are joined in LDS in the waves' order.
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void mx_few_rows_kernel(ProductArgs p, uint32_t n_tiles)
{
    __shared__ float s_part[WAVES][256];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const int64_t j0 = (int64_t)(blockIdx.x % n_tiles) * 16, i0 = (int64_t)(blockIdx.x / n_tiles) * 16;
    const int64_t j = j0 + r < p.n ? j0 + r : p.n - 1, i = i0 + r < p.m ? i0 + r : p.m - 1;
    const uint8_t *cb = p.b.codes + j * (p.chunks * 128) + g * 32, *ca = p.a.codes + i * (p.chunks * 128) + g * 32;
    const uint8_t *sb = p.b.scales + mx_scale_at(j, (g >> 1) * 4, p.chunks), *sa = p.a.scales + mx_scale_at(i, (g >> 1) * 4, p.chunks);
    f32x4 c = {0, 0, 0, 0};
    for (int64_t k = wave; k < p.chunks; k += WAVES) {
        const u32x4 b0 = *reinterpret_cast<const u32x4*>(cb + k * 128), b1 = *reinterpret_cast<const u32x4*>(cb + k * 128 + 16);
        const u32x4 a0 = *reinterpret_cast<const u32x4*>(ca + k * 128), a1 = *reinterpret_cast<const u32x4*>(ca + k * 128 + 16);
        const uint32_t tb = *reinterpret_cast<const uint32_t*>(sb + k * 256) >> ((g & 1) * 16);
        const uint32_t ta = *reinterpret_cast<const uint32_t*>(sa + k * 256) >> ((g & 1) * 16);
        c = mx_mfma<0>(b0, a0, tb, ta, c);
        c = mx_mfma<1>(b1, a1, tb, ta, c);
    }
    // outputs [i = r][j = 4g ..]
    *reinterpret_cast<f32x4*>(&s_part[wave][r * 16 + g * 4]) = c;
    __syncthreads();
    if (threadIdx.x < 256) {
        float sum = 0.0f;
        for (int w = 0; w < WAVES; ++w) sum += s_part[w][threadIdx.x];
        const int64_t row = i0 + (threadIdx.x >> 4), col = j0 + (threadIdx.x & 15);
        if (row < p.m && col < p.n) store1(static_cast<T*>(p.out) + row * p.stride + col, sum + bias_of<T>(p, col));
    }
}

template <typename T>
hipError_t product_of(const ProductArgs& p, hipStream_t s)
{
    const int64_t n_tiles = (p.n + 15) / 16, tiles = n_tiles * ((p.m + 15) / 16);
    if (tiles > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((mx_few_rows_kernel<T, 4>), dim3((uint32_t)tiles), dim3(256), 0, s, p, (uint32_t)n_tiles);
    return hipGetLastError();
}

}  // namespace
}  // namespace fh

extern "C" {

size_t fh_mx_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k) { return 0; }

fh_status fh_mx_matmul(const fh_mx_product* q, void* stream)
{
    using namespace fh;
    if (!q) return FH_ERR_NULL;
    if (!is_dtype(q->out_dtype) || !is_dtype(q->bias_dtype)) return FH_ERR_BAD_DTYPE;
    if (!mx_shape_ok(q->m, q->k) || !mx_shape_ok(q->n, q->k) || q->k > kMostSummed || q->stride < q->n || q->stride > kMostStride) return FH_ERR_BAD_SHAPE;
    if (q->reserved != 0) return FH_ERR_BAD_PARAM;
    if (q->m == 0 || q->n == 0) return FH_OK;
    if (!q->out || (q->k > 0 && (!q->a || !q->b))) return FH_ERR_NULL;
    const size_t size = dtype_size(q->out_dtype);
    if (!is_aligned(q->a, 16) || !is_aligned(q->b, 16) || !is_aligned(q->out, size) || !is_aligned(q->bias, dtype_size(q->bias_dtype)) ||
        !is_aligned(q->workspace, 16)) return FH_ERR_ALIGNMENT;
    if (q->a_cap < mx_bytes(q->m, q->k) || q->b_cap < mx_bytes(q->n, q->k) || q->out_cap < strided_elements(q->m, q->n, q->stride) * size)
        return FH_ERR_BUFFER_TOO_SMALL;
    const size_t workspace = fh_mx_matmul_workspace_bytes(q->m, q->n, q->k);
    if (workspace && !q->workspace) return FH_ERR_NULL;
    if (q->workspace_cap < workspace) return FH_ERR_BUFFER_TOO_SMALL;
    const ProductArgs p = {mx_store(const_cast<void*>(q->a), q->m, q->k), mx_store(const_cast<void*>(q->b), q->n, q->k), q->m, q->n,
                           mx_chunks(q->k), q->bias, q->bias_dtype, q->out, q->stride};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = q->out_dtype == FH_F32 ? product_of<float>(p, s) : product_of<Bf16>(p, s);
    return e == hipSuccess ? FH_OK : FH_ERR_LAUNCH;
}

}  // extern "C"
