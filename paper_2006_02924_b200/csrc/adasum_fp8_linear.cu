// Products of packed 8-bit matrices: a linear layer, and the gradient of its input.
//
//     y[r][n]  = sum_k x[r][k] w[n][k] + bias[n]
//     dx[r][k] = sum_n dy[r][n] w[n][k]
#include "adasum_fp8.cuh"

namespace adasum {
namespace {

constexpr int kTile = 64, kDepth = 32, kThreads = 256;
constexpr size_t kStatusBytes = 1024;

struct LinearArgs {
    const uint8_t *a, *a_steps, *w, *w_steps;
    int64_t rows, depth, wide;         // out: rows x wide, sums of `depth` products
    int64_t a_width, w_width;
    const void* bias;
    int bias_dtype;
    void* out;
    int64_t out_stride;
    int out_dtype;
};

__device__ __forceinline__ float value_at(const uint8_t* codes, const uint8_t* steps, int64_t width, int64_t row, int64_t column)
{
    const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)codes[row * width + column], __NV_E4M3);
    return __half2float(*reinterpret_cast<const __half*>(&h)) *
           fp8_step_value(steps[fp8_step_at(row, column / kFp8Block, width / kFp8Block)]);
}

// GRAD: the weights are read with the summed index as rows.
template <bool GRAD>
__global__ void __launch_bounds__(kThreads) fp8_linear_kernel(const __grid_constant__ LinearArgs a)
{
    __shared__ float left[kDepth][kTile + 1], right[kDepth][kTile + 1];
    const int64_t row0 = (int64_t)blockIdx.x * kTile, col0 = (int64_t)blockIdx.y * kTile;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float sum[4][4] = {};
    for (int64_t k0 = 0; k0 < a.depth; k0 += kDepth) {
        for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
            const int64_t row = row0 + i / kDepth, k = k0 + i % kDepth;
            left[i % kDepth][i / kDepth] = row < a.rows && k < a.depth ? value_at(a.a, a.a_steps, a.a_width, row, k) : 0.0f;
            const int d = GRAD ? i / kTile : i % kDepth, c = GRAD ? i % kTile : i / kDepth;
            const bool in = col0 + c < a.wide && k0 + d < a.depth;
            right[d][c] = !in ? 0.0f : GRAD ? value_at(a.w, a.w_steps, a.w_width, k0 + d, col0 + c)
                                            : value_at(a.w, a.w_steps, a.w_width, col0 + c, k0 + d);
        }
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum[i][j] = fmaf(left[k][ty + 16 * i], right[k][tx + 16 * j], sum[i][j]);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t row = row0 + ty + 16 * i, column = col0 + tx + 16 * j;
            if (row < a.rows && column < a.wide)
                store_from_float(a.out, a.out_dtype, row * a.out_stride + column,
                                 sum[i][j] + (a.bias ? load_as_float(a.bias, a.bias_dtype, column) : 0.0f));
        }
}

adasum_status_t linear(const void* x, const void* w, int64_t rows, int64_t features, int64_t outputs, const void* bias,
                       adasum_dtype_t bias_dtype, void* out, int64_t out_stride, adasum_dtype_t out_dtype, void* workspace,
                       size_t workspace_bytes, bool grad, void* stream_ptr)
{
    clear_error();
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs))
        return fail(ADASUM_ERR_ARG, "rows = %lld, features = %lld, outputs = %lld out of range", (long long)rows,
                    (long long)features, (long long)outputs);
    if (!operator_dtype(out_dtype) || (bias && !operator_dtype(bias_dtype)))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d: fp32, fp16 or bf16", (int)out_dtype, (int)bias_dtype);
    const int64_t depth = grad ? outputs : features, wide = grad ? features : outputs;
    if (rows == 0 || wide == 0)
        return ADASUM_OK;
    if (depth > 0 && (!x || !w))
        return fail(ADASUM_ERR_NULL, "a packed matrix is NULL");
    if (!aligned_to(x, 16) || !aligned_to(w, 16))
        return fail(ADASUM_ERR_ARG, "a packed matrix is not 16-byte aligned");
    adasum_status_t status = check_matrix(grad ? "dx" : "y", out, out_stride, wide, out_dtype);
    if (status != ADASUM_OK)
        return status;
    if (bias && !aligned_to(bias, operator_bytes(bias_dtype)))
        return fail(ADASUM_ERR_ARG, "bias is not aligned to its element size");
    const size_t need = adasum_fp8_linear_workspace_bytes(rows, features, outputs);
    if (!workspace || workspace_bytes < need)
        return fail(ADASUM_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned_to(workspace, 256))
        return fail(ADASUM_ERR_ARG, "workspace is not 256-byte aligned");
    const size_t out_bytes = matrix_span(rows, wide, out_stride, operator_bytes(out_dtype));
    const size_t x_bytes = fp8_bytes(rows, depth), w_bytes = fp8_bytes(outputs, features);
    const size_t bias_bytes = bias ? (size_t)(outputs * operator_bytes(bias_dtype)) : 0;
    if (spans_overlap(out, out_bytes, x, x_bytes) || spans_overlap(out, out_bytes, w, w_bytes) ||
        spans_overlap(out, out_bytes, bias, bias_bytes) || spans_overlap(out, out_bytes, workspace, need) ||
        spans_overlap(workspace, need, x, x_bytes) || spans_overlap(workspace, need, w, w_bytes) ||
        spans_overlap(workspace, need, bias, bias_bytes))
        return fail(ADASUM_ERR_ARG, "the output or the workspace overlaps an input or each other");
    LinearArgs a;
    a.rows = rows;
    a.depth = depth;
    a.wide = wide;
    a.a_width = fp8_width(depth);
    a.w_width = fp8_width(features);
    a.a = static_cast<const uint8_t*>(x);
    a.a_steps = a.a + rows * a.a_width;
    a.w = static_cast<const uint8_t*>(w);
    a.w_steps = a.w + outputs * a.w_width;
    a.bias = bias;
    a.bias_dtype = (int)bias_dtype;
    a.out = out;
    a.out_stride = out_stride;
    a.out_dtype = (int)out_dtype;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    const dim3 grid((unsigned)((rows + kTile - 1) / kTile), (unsigned)((wide + kTile - 1) / kTile));
    if (grid.y > 65535)
        return fail(ADASUM_ERR_ARG, "too large");
    if (grad)
        fp8_linear_kernel<true><<<grid, kThreads, 0, stream>>>(a);
    else
        fp8_linear_kernel<false><<<grid, kThreads, 0, stream>>>(a);
    ADASUM_CUDA_CHECK(cudaGetLastError());
    profile_mark(stream, ADASUM_KERNEL_FP8_LINEAR, 0, 0, false);
    return ADASUM_OK;
}

}  // namespace
}  // namespace adasum

extern "C" {

size_t adasum_fp8_linear_workspace_bytes(int64_t rows, int64_t features, int64_t outputs)
{
    using namespace adasum;
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs))
        return 0;
    return kStatusBytes;
}

adasum_status_t adasum_fp8_linear(const void* x, const void* w, int64_t rows, int64_t features, int64_t outputs,
                                  const void* bias, adasum_dtype_t bias_dtype, void* y, int64_t y_stride,
                                  adasum_dtype_t out_dtype, void* workspace, size_t workspace_bytes, void* stream_ptr)
{
    return adasum::linear(x, w, rows, features, outputs, bias, bias_dtype, y, y_stride, out_dtype, workspace, workspace_bytes,
                          false, stream_ptr);
}

adasum_status_t adasum_fp8_linear_grad(const void* dy, const void* w, int64_t rows, int64_t features, int64_t outputs,
                                       void* dx, int64_t dx_stride, adasum_dtype_t out_dtype, void* workspace,
                                       size_t workspace_bytes, void* stream_ptr)
{
    return adasum::linear(dy, w, rows, features, outputs, nullptr, out_dtype, dx, dx_stride, out_dtype, workspace, workspace_bytes,
                          true, stream_ptr);
}

adasum_status_t adasum_fp8_linear_status(const void* workspace, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    if (!workspace)
        return fail(ADASUM_ERR_NULL, "workspace is NULL");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    ADASUM_CUDA_CHECK(cudaStreamSynchronize(stream));
    return ADASUM_OK;
}

}  // extern "C"
