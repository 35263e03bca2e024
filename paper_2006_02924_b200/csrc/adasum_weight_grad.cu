// Gradients of a linear layer from the kept values of its input:
//
//     grad_weight[n][k] = scale * sum_t grad_out[t][n] * (kept x)[t][k]
//     grad_bias[n]      = scale * sum_t grad_out[t][n]
#include "adasum_operators.cuh"

namespace adasum {
namespace {

constexpr int kGroup = 32;
constexpr int kTile = 64, kDepth = 16, kPerThread = 4;

struct WeightGradArgs {
    const int8_t* codes;
    const uint8_t* steps;
    int64_t rows, features, width, outputs, stride;
    float scale;
    void* weight;
    void* bias;
    int out_dtype;
    bool accumulate;
};

__device__ __forceinline__ void write_gradient(const WeightGradArgs& a, void* dst, int64_t e, float sum)
{
    float y = sum * a.scale;
    if (a.accumulate)
        y += load_as_float(dst, a.out_dtype, e);
    store_from_float(dst, a.out_dtype, e, y);
}

// One block: a 64 x 64 tile of grad_weight, fp32 throughout.
template <typename T>
__global__ void __launch_bounds__(256) weight_grad_kernel(WeightGradArgs a, const T* __restrict__ grad)
{
    __shared__ float g[kDepth][kTile], x[kDepth][kTile];
    const int64_t k0 = (int64_t)blockIdx.x * kTile, n0 = (int64_t)blockIdx.y * kTile;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float sum[kPerThread][kPerThread] = {};
    float bias = 0.0f;
    for (int64_t t0 = 0; t0 < a.rows; t0 += kDepth) {
        for (int i = threadIdx.x; i < kDepth * kTile; i += 256) {
            const int64_t t = t0 + i / kTile, n = n0 + i % kTile, k = k0 + i % kTile;
            g[i / kTile][i % kTile] = t < a.rows && n < a.outputs ? load_one(grad + t * a.stride + n) : 0.0f;
            x[i / kTile][i % kTile] =
                t < a.rows && k < a.features
                    ? (float)a.codes[t * a.width + k] *
                          __uint_as_float((uint32_t)a.steps[t * (a.width / kGroup) + k / kGroup] << 23)
                    : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
#pragma unroll
            for (int i = 0; i < kPerThread; ++i)
#pragma unroll
                for (int j = 0; j < kPerThread; ++j)
                    sum[i][j] = fmaf(g[d][ty + 16 * i], x[d][tx + 16 * j], sum[i][j]);
            if (threadIdx.x < kTile)
                bias += g[d][threadIdx.x];
        }
        __syncthreads();
    }
    for (int i = 0; i < kPerThread; ++i)
        for (int j = 0; j < kPerThread; ++j) {
            const int64_t n = n0 + ty + 16 * i, k = k0 + tx + 16 * j;
            if (n < a.outputs && k < a.features)
                write_gradient(a, a.weight, n * a.features + k, sum[i][j]);
        }
    if (a.bias && blockIdx.x == 0 && threadIdx.x < kTile && n0 + threadIdx.x < a.outputs)
        write_gradient(a, a.bias, n0 + threadIdx.x, bias);
}

template <typename T>
void launch_weight_grad(const WeightGradArgs& a, const void* grad_out, cudaStream_t stream)
{
    // with no features the bias gradient still has its blocks
    const dim3 grid((unsigned)((a.features + kTile - 1) / kTile + (a.features == 0)),
                    (unsigned)((a.outputs + kTile - 1) / kTile));
    weight_grad_kernel<T><<<grid, 256, 0, stream>>>(a, static_cast<const T*>(grad_out));
}

}  // namespace
}  // namespace adasum

extern "C" {

size_t adasum_checkpoint_weight_grad_workspace_bytes(int64_t rows, int64_t features, int64_t outputs,
                                                     adasum_dtype_t dtype)
{
    using namespace adasum;
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs) || !operator_dtype(dtype))
        return 0;
    return 256;
}

adasum_status_t adasum_checkpoint_weight_grad(const void* checkpoint, int64_t rows, int64_t features,
                                              const void* grad_out, int64_t grad_out_stride, int64_t outputs,
                                              adasum_dtype_t dtype, float scale, void* grad_weight, void* grad_bias,
                                              adasum_dtype_t grad_dtype, int32_t accumulate, void* workspace,
                                              size_t workspace_bytes, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs))
        return fail(ADASUM_ERR_ARG, "rows = %lld, features = %lld, outputs = %lld out of range", (long long)rows,
                    (long long)features, (long long)outputs);
    if (!operator_dtype(dtype) || !operator_dtype(grad_dtype))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d: fp32, fp16 or bf16", (int)dtype, (int)grad_dtype);
    if (outputs == 0 || (features == 0 && !grad_bias) || (rows == 0 && accumulate))
        return ADASUM_OK;
    if (rows > 0 && (!grad_out || (features > 0 && !checkpoint)))
        return fail(ADASUM_ERR_NULL, "checkpoint or grad_out is NULL");
    if (features > 0 && !grad_weight)
        return fail(ADASUM_ERR_NULL, "grad_weight is NULL");
    const int64_t eb = operator_bytes(dtype), gb = operator_bytes(grad_dtype);
    if (!aligned_to(checkpoint, 16))
        return fail(ADASUM_ERR_ARG, "checkpoint is not 16-byte aligned");
    if (!aligned_to(grad_out, eb) || !aligned_to(grad_weight, gb) || !aligned_to(grad_bias, gb))
        return fail(ADASUM_ERR_ARG, "grad_out, grad_weight or grad_bias is not aligned to its element size");
    if (rows > 0 && !stride_ok(grad_out_stride, outputs))
        return fail(ADASUM_ERR_ARG, "grad_out_stride %lld is shorter than a row or out of range",
                    (long long)grad_out_stride);
    const size_t need = adasum_checkpoint_weight_grad_workspace_bytes(rows, features, outputs, dtype);
    if (!workspace || workspace_bytes < need)
        return fail(ADASUM_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace ? workspace_bytes : (size_t)0,
                    need);
    if (!aligned_to(workspace, 256))
        return fail(ADASUM_ERR_ARG, "workspace is not 256-byte aligned");
    const size_t in_bytes = matrix_span(rows, outputs, grad_out_stride, eb);
    const size_t kept_bytes = adasum_checkpoint_bytes(rows, features);
    const size_t weight_bytes = (size_t)outputs * (size_t)features * (size_t)gb;
    const size_t bias_bytes = grad_bias ? (size_t)outputs * (size_t)gb : 0;
    const struct { const void* p; size_t bytes; } inputs[] = {{checkpoint, kept_bytes}, {grad_out, in_bytes}};
    for (const auto& in : inputs)
        if (spans_overlap(in.p, in.bytes, grad_weight, weight_bytes) || spans_overlap(in.p, in.bytes, grad_bias, bias_bytes) ||
            spans_overlap(in.p, in.bytes, workspace, need))
            return fail(ADASUM_ERR_ARG, "an input overlaps a gradient or the workspace");
    if (spans_overlap(grad_weight, weight_bytes, grad_bias, bias_bytes) ||
        spans_overlap(workspace, need, grad_weight, weight_bytes) || spans_overlap(workspace, need, grad_bias, bias_bytes))
        return fail(ADASUM_ERR_ARG, "grad_weight, grad_bias and workspace overlap");

    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    WeightGradArgs a;
    a.rows = rows;
    a.features = features;
    a.width = (features + kGroup - 1) / kGroup * kGroup;
    a.codes = static_cast<const int8_t*>(checkpoint);
    a.steps = static_cast<const uint8_t*>(checkpoint) + rows * a.width;
    a.outputs = outputs;
    a.stride = grad_out_stride;
    a.scale = scale;
    a.weight = grad_weight;
    a.bias = grad_bias;
    a.out_dtype = (int)grad_dtype;
    a.accumulate = accumulate != 0;
    profile_mark(stream, -1, 0, 0, true);
    if (dtype == ADASUM_F32)
        launch_weight_grad<float>(a, grad_out, stream);
    else if (dtype == ADASUM_F16)
        launch_weight_grad<__half>(a, grad_out, stream);
    else
        launch_weight_grad<__nv_bfloat16>(a, grad_out, stream);
    ADASUM_CUDA_CHECK(cudaGetLastError());
    profile_mark(stream, ADASUM_KERNEL_WEIGHT_GRAD, 1, 0, false);
    return ADASUM_OK;
}

}  // extern "C"
