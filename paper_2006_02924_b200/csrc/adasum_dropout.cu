// Dropout, alone or on its way into the residual stream:  out = [residual +] kept * x / (1 - q).  Its gradient is the
// same call on the gradient.  One pass; a thread handles vectors of eight columns, which share one call of the
// generator.  With fp32 or a residual HBM traffic bounds it (16384 x 4096 fp32 79 us, with a residual 116 us: 6.8 TB/s), with bf16
// alone the generator's instructions (55 us, 4.9 TB/s; with a residual 64 us, 6.2 TB/s).
#include "adasum_random.cuh"
#include "adasum_vectors.cuh"

namespace adasum {
namespace {

// Vectors per thread, in as many rows.  16384 x 4096 bf16 with 1, 2, 4: 71, 57, 55 us (fp32: 78, 79, 79).
constexpr int kDropRows = 4;

template <typename T, bool VEC>
__global__ void __launch_bounds__(kStripThreads)
dropout_kernel(const __grid_constant__ Strips s, const __grid_constant__ Dropout d, const T* x, int64_t x_stride,
               const T* residual, int64_t residual_stride, T* out, int64_t out_stride)
{
    start_next_kernel();
    wait_for_previous_kernel();
    const Place p = place_of<kDropRows>(s);
    if (p.count <= 0)
        return;
    Raw<T> rx[kDropRows], rr[kDropRows];
    uint64_t vector[kDropRows];
#pragma unroll
    for (int u = 0; u < kDropRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        const int count = row < s.rows ? p.count : 0;
        rx[u] = load_vector<VEC>(x + row * x_stride + p.column, count);
        if (residual)
            rr[u] = load_vector<VEC>(residual + row * residual_stride + p.column, count);
        vector[u] = (uint64_t)row * (uint32_t)s.per_row + (uint32_t)(p.column >> 3);
    }
    uint32_t word[kDropRows][4];
    if (d.seed)
        random_words(d, *d.seed, vector, word);
#pragma unroll
    for (int u = 0; u < kDropRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        if (row >= s.rows)
            break;
        float y[8];
        values_of(decode(rx[u]), y);
        if (d.seed)
            drop(d, word[u], y);
        if (residual) {
            float r[8];
            values_of(decode(rr[u]), r);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                y[i] += r[i];
        }
        store_values<VEC>(out + row * out_stride + p.column, p.count, y);
    }
}

}  // namespace
}  // namespace adasum

extern "C" adasum_status_t adasum_dropout(const void* x, int64_t x_stride, int64_t rows, int64_t features,
                                          adasum_dtype_t dtype, const void* residual, int64_t residual_stride, float p,
                                          const uint64_t* seed, uint64_t site, void* out, int64_t out_stride,
                                          void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    if (!extent_ok(rows) || !extent_ok(features))
        return fail(ADASUM_ERR_ARG, "rows = %lld, features = %lld out of range", (long long)rows, (long long)features);
    if (!operator_dtype(dtype))
        return fail(ADASUM_ERR_DTYPE, "dtype %d is not fp32, fp16 or bf16", (int)dtype);
    Dropout d;
    adasum_status_t status = plan_dropout(p, seed, site, &d);
    if (status != ADASUM_OK || rows == 0 || features == 0)
        return status;
    if ((status = check_matrix("x", x, x_stride, features, dtype)) != ADASUM_OK ||
        (status = check_matrix("out", out, out_stride, features, dtype)) != ADASUM_OK)
        return status;
    if (residual && (status = check_matrix("residual", residual, residual_stride, features, dtype)) != ADASUM_OK)
        return status;
    const int64_t eb = operator_bytes(dtype);
    const size_t x_bytes = matrix_span(rows, features, x_stride, eb), out_bytes = matrix_span(rows, features, out_stride, eb);
    const size_t r_bytes = residual ? matrix_span(rows, features, residual_stride, eb) : 0;
    if (spans_overlap(x, x_bytes, out, out_bytes) && !(x == out && x_stride == out_stride))
        return fail(ADASUM_ERR_ARG, "out overlaps x without being the same matrix");
    if (spans_overlap(residual, r_bytes, out, out_bytes) && !(residual == out && residual_stride == out_stride))
        return fail(ADASUM_ERR_ARG, "out overlaps residual without being the same matrix");
    if (spans_overlap(d.seed, 8, out, out_bytes))
        return fail(ADASUM_ERR_ARG, "out overlaps the seed");
    Strips s;
    unsigned blocks;
    if (!plan_strips(rows, features, (features + 7) / 8, kDropRows, &s, &blocks))
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)features);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    cudaError_t err = cudaSuccess;
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const bool vec = features % 8 == 0 && rows_aligned(x, x_stride, eb) && rows_aligned(out, out_stride, eb) &&
                         (!residual || rows_aligned(residual, residual_stride, eb));
        err = launch_after(vec ? dropout_kernel<T, true> : dropout_kernel<T, false>, dim3(blocks), kStripThreads, 0, stream, s, d,
                           static_cast<const T*>(x), x_stride, static_cast<const T*>(residual), residual_stride, static_cast<T*>(out),
                           out_stride);
    });
    ADASUM_CUDA_CHECK(err);
    profile_mark(stream, ADASUM_KERNEL_DROPOUT, 0, 0, false);
    return ADASUM_OK;
}
