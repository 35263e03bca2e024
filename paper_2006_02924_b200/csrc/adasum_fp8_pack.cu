// Matrices to 8-bit floating point and back.  One pass over a matrix each, bound by HBM traffic: 16384 x 4096 to 8 bits
// from bf16 33 us (6.2 TB/s), from fp32 50 us (6.7 TB/s); weights 37 us and 51 us; back to bf16 34 us, to fp32 58 us.  Latency below
// a few MB: 37 x 1024 1.8 us.
#include "adasum_fp8.cuh"
#include "adasum_vectors.cuh"

namespace adasum {
namespace {

constexpr int kPackRows = 2;               // pairs of vectors per thread, in as many rows
// Vectors per thread, in as many rows.  16384 x 4096 to bf16 with 1, 2, 4: 41, 36, 34 us; to fp32 56, 64, 73 us.
template <typename T>
constexpr int kUnpackRows = sizeof(T) == 4 ? 1 : 4;
constexpr int kWeightThreads = 256;
constexpr int kWeightRows = kFp8Block * kFp8Block / 8 / kWeightThreads;      // vectors per thread, in as many rows

// A block kept as NaN has codes of zero, whatever it holds.
__device__ __forceinline__ uint2 codes_of(const Eight& x, uint32_t byte)
{
    const Pair inv = both(__uint_as_float((254u - min(byte, 254u)) << 23));
    float y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = values_of(x.p[i] * inv);
        y[2 * i] = f.x;
        y[2 * i + 1] = f.y;
    }
    const uint2 codes = make_uint2(fp8_encode(y[0], y[1], y[2], y[3]), fp8_encode(y[4], y[5], y[6], y[7]));
    return byte == 255u ? make_uint2(0, 0) : codes;
}

// A thread handles 16 neighbouring columns (a whole store of codes); eight neighbouring lanes hold the 128 columns of a
// block: the largest magnitude is three shuffles away.  `s` counts pairs of vectors.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kStripThreads)
fp8_pack_kernel(const __grid_constant__ Strips s, int64_t columns, const T* x, int64_t x_stride, uint8_t* codes, uint8_t* steps)
{
    start_next_kernel();             // the product sets itself up meanwhile (with 37 x 1024 9.0 -> 7.5 us)
    wait_for_previous_kernel();
    const Place p = place_of<kPackRows>(s);
    const int64_t column = 2 * (int64_t)p.column;
    const int count = p.inside ? (int)max((int64_t)0, min((int64_t)16, columns - column)) : 0;
    Raw<T> raw[kPackRows][2];
#pragma unroll
    for (int u = 0; u < kPackRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        const T* q = x + row * x_stride + column;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            raw[u][i] = load_vector<VEC>(q + 8 * i, row < s.rows ? min(8, count - 8 * i) : 0);
    }
#pragma unroll
    for (int u = 0; u < kPackRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        uint32_t top = max(largest(raw[u][0]), largest(raw[u][1]));
#pragma unroll
        for (int step = 1; step < 8; step *= 2)
            top = max(top, __shfl_xor_sync(0xffffffffu, top, step));
        const uint32_t byte = fp8_step_byte(top);
        if (p.inside && row < s.rows) {
            const uint2 low = codes_of(decode(raw[u][0]), byte), high = codes_of(decode(raw[u][1]), byte);
            *reinterpret_cast<uint4*>(codes + row * (int64_t)s.per_row * 16 + column) = make_uint4(low.x, low.y, high.x, high.y);
            if ((column & (kFp8Block - 1)) == 0)
                *reinterpret_cast<uint32_t*>(steps + fp8_step_at(row, column / kFp8Block, s.per_row / 8)) = byte * 0x01010101u;
        }
    }
}

// One block of 128 x 128 per thread block; sixteen threads per row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kWeightThreads)
fp8_pack_weight_kernel(const T* w, int64_t w_stride, int64_t rows, int64_t columns, uint32_t column_blocks, uint8_t* codes,
                       uint8_t* steps)
{
    __shared__ uint32_t warp_top[kWeightThreads / 32];
    start_next_kernel();
    wait_for_previous_kernel();
    const uint32_t row_block = blockIdx.x / column_blocks, column_block = blockIdx.x - row_block * column_blocks;
    const int64_t column = (int64_t)column_block * kFp8Block + (threadIdx.x & 15) * 8;
    const int64_t row0 = (int64_t)row_block * kFp8Block + (threadIdx.x >> 4);
    const int count = (int)max((int64_t)0, min((int64_t)8, columns - column));
    Raw<T> raw[kWeightRows];
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < kWeightRows; ++u) {
        const int64_t row = row0 + u * (kWeightThreads / 16);
        raw[u] = load_vector<VEC>(w + row * w_stride + column, row < rows ? count : 0);
    }
#pragma unroll
    for (int u = 0; u < kWeightRows; ++u)
        top = max(top, largest(raw[u]));
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0)
        warp_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWeightThreads / 32; ++i)
        top = max(top, warp_top[i]);
    const uint32_t byte = fp8_step_byte(top);
#pragma unroll
    for (int u = 0; u < kWeightRows; ++u) {
        const int64_t row = row0 + u * (kWeightThreads / 16);
        if (row < rows)
            *reinterpret_cast<uint2*>(codes + row * (int64_t)column_blocks * kFp8Block + column) = codes_of(decode(raw[u]), byte);
    }
    if (threadIdx.x < kFp8StepBytes / 4)
        reinterpret_cast<uint32_t*>(steps + (int64_t)blockIdx.x * kFp8StepBytes)[threadIdx.x] = byte * 0x01010101u;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kStripThreads)
fp8_unpack_kernel(const __grid_constant__ Strips s, const uint8_t* codes, const uint8_t* steps, int64_t width, T* out,
                  int64_t out_stride)
{
    const Place p = place_of<kUnpackRows<T>>(s);
    if (p.count <= 0)
        return;
    uint2 packed[kUnpackRows<T>];
    uint32_t byte[kUnpackRows<T>];
#pragma unroll
    for (int u = 0; u < kUnpackRows<T>; ++u) {
        const int64_t row = p.row0 + u * p.step;
        if (row < s.rows) {
            packed[u] = *reinterpret_cast<const uint2*>(codes + row * width + p.column);
            byte[u] = steps[fp8_step_at(row, p.column / kFp8Block, width / kFp8Block)];
        }
    }
#pragma unroll
    for (int u = 0; u < kUnpackRows<T>; ++u) {
        const int64_t row = p.row0 + u * p.step;
        if (row < s.rows) {
            const float step = fp8_step_value(byte[u]);
            float a[4], b[4];
            fp8_decode(packed[u].x, a);
            fp8_decode(packed[u].y, b);
            float y[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                y[i] = a[i] * step;
                y[4 + i] = b[i] * step;
            }
            store_values<VEC>(out + row * out_stride + p.column, p.count, y);
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------

adasum_status_t check_packed(const void* packed, int64_t rows, int64_t columns, adasum_dtype_t dtype)
{
    if (!extent_ok(rows) || !extent_ok(columns))
        return fail(ADASUM_ERR_ARG, "rows = %lld, columns = %lld out of range", (long long)rows, (long long)columns);
    if (!operator_dtype(dtype))
        return fail(ADASUM_ERR_DTYPE, "dtype %d is not fp32, fp16 or bf16", (int)dtype);
    if (rows == 0 || columns == 0)
        return ADASUM_OK;
    if (!packed)
        return fail(ADASUM_ERR_NULL, "packed is NULL");
    if (!aligned_to(packed, 16))
        return fail(ADASUM_ERR_ARG, "packed is not 16-byte aligned");
    return ADASUM_OK;
}

adasum_status_t pack(const void* x, int64_t x_stride, int64_t rows, int64_t columns, adasum_dtype_t dtype, void* packed,
                     bool weight, void* stream_ptr)
{
    clear_error();
    adasum_status_t status = check_packed(packed, rows, columns, dtype);
    if (status != ADASUM_OK || rows == 0 || columns == 0)
        return status;
    if ((status = check_matrix("the matrix", x, x_stride, columns, dtype)) != ADASUM_OK)
        return status;
    const int64_t eb = operator_bytes(dtype), width = fp8_width(columns);
    if (spans_overlap(x, matrix_span(rows, columns, x_stride, eb), packed, fp8_bytes(rows, columns)))
        return fail(ADASUM_ERR_ARG, "packed overlaps the matrix");
    const bool vec = columns % 8 == 0 && rows_aligned(x, x_stride, eb);
    uint8_t* codes = static_cast<uint8_t*>(packed);
    uint8_t* steps = codes + rows * width;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    Strips s;
    unsigned blocks = 0;
    if (weight) {
        const int64_t n = fp8_blocks(rows) * fp8_blocks(columns);
        if (n > 0x7fffffff)
            return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)columns);
        blocks = (unsigned)n;
    } else if (!plan_strips(rows, width / 2, width / 16, kPackRows, &s, &blocks)) {
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)columns);
    }
    profile_mark(stream, -1, 0, 0, true);
    cudaError_t err = cudaSuccess;
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const T* from = static_cast<const T*>(x);
        if (weight)
            err = launch_after(vec ? fp8_pack_weight_kernel<T, true> : fp8_pack_weight_kernel<T, false>, dim3(blocks), kWeightThreads, 0,
                               stream, from, x_stride, rows, columns, (uint32_t)fp8_blocks(columns), codes, steps);
        else
            err = launch_after(vec ? fp8_pack_kernel<T, true> : fp8_pack_kernel<T, false>, dim3(blocks), kStripThreads, 0, stream, s,
                               columns, from, x_stride, codes, steps);
    });
    ADASUM_CUDA_CHECK(err);
    profile_mark(stream, ADASUM_KERNEL_FP8_PACK, 0, 0, false);
    return ADASUM_OK;
}

}  // namespace
}  // namespace adasum

extern "C" {

size_t adasum_fp8_bytes(int64_t rows, int64_t columns)
{
    using namespace adasum;
    if (!extent_ok(rows) || !extent_ok(columns))
        return 0;
    return fp8_bytes(rows, columns);
}

adasum_status_t adasum_fp8_pack(const void* x, int64_t x_stride, int64_t rows, int64_t columns, adasum_dtype_t dtype,
                                void* packed, void* stream_ptr)
{
    return adasum::pack(x, x_stride, rows, columns, dtype, packed, false, stream_ptr);
}

adasum_status_t adasum_fp8_pack_weight(const void* w, int64_t w_stride, int64_t rows, int64_t columns,
                                       adasum_dtype_t dtype, void* packed, void* stream_ptr)
{
    return adasum::pack(w, w_stride, rows, columns, dtype, packed, true, stream_ptr);
}

adasum_status_t adasum_fp8_unpack(const void* packed, int64_t rows, int64_t columns, void* out, int64_t out_stride,
                                  adasum_dtype_t dtype, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    adasum_status_t status = check_packed(packed, rows, columns, dtype);
    if (status != ADASUM_OK || rows == 0 || columns == 0)
        return status;
    if ((status = check_matrix("out", out, out_stride, columns, dtype)) != ADASUM_OK)
        return status;
    const int64_t eb = operator_bytes(dtype), width = fp8_width(columns);
    if (spans_overlap(out, matrix_span(rows, columns, out_stride, eb), packed, fp8_bytes(rows, columns)))
        return fail(ADASUM_ERR_ARG, "packed overlaps out");
    Strips s;
    unsigned blocks;
    const int out_rows = dtype == ADASUM_F32 ? kUnpackRows<float> : kUnpackRows<__half>;
    if (!plan_strips(rows, columns, (columns + 7) / 8, out_rows, &s, &blocks))
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)columns);
    const uint8_t* codes = static_cast<const uint8_t*>(packed);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        auto* kernel = columns % 8 == 0 && rows_aligned(out, out_stride, eb) ? fp8_unpack_kernel<T, true> : fp8_unpack_kernel<T, false>;
        kernel<<<blocks, kStripThreads, 0, stream>>>(s, codes, codes + rows * width, width, static_cast<T*>(out), out_stride);
    });
    ADASUM_CUDA_CHECK(cudaGetLastError());
    profile_mark(stream, ADASUM_KERNEL_FP8_UNPACK, 0, 0, false);
    return ADASUM_OK;
}

}  // extern "C"
