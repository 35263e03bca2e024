// What the operators that produce a worker's gradients share (adasum_embedding.cu, adasum_checkpoint.cu,
// adasum_weight_grad.cu): checks of matrix arguments and access to strided rows of any supported type.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "adasum_internal.h"

namespace adasum {

// ---- host: arguments -------------------------------------------------------------------------------

inline bool operator_dtype(adasum_dtype_t dtype)
{
    return dtype == ADASUM_F32 || dtype == ADASUM_F16 || dtype == ADASUM_BF16;
}
inline int64_t operator_bytes(adasum_dtype_t dtype) { return dtype == ADASUM_F32 ? 4 : 2; }

// Bytes from the first to past the last element of a strided matrix.
inline size_t matrix_span(int64_t rows, int64_t cols, int64_t stride, int64_t elem_bytes)
{
    return rows > 0 && cols > 0 ? (size_t)((rows - 1) * stride + cols) * (size_t)elem_bytes : 0;
}
inline bool spans_overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && a_bytes && b_bytes && x < y + b_bytes && y < x + a_bytes;
}
inline bool aligned_to(const void* p, int64_t bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }
// Rows that 16-byte accesses may be used on.
inline bool rows_aligned(const void* p, int64_t stride, int64_t elem_bytes)
{
    return aligned_to(p, 16) && stride * elem_bytes % 16 == 0;
}

// Products such as rows * stride stay far inside 64 bits.
constexpr int64_t kMaxExtent = (int64_t(1) << 31) - 256;
inline bool extent_ok(int64_t n) { return n >= 0 && n <= kMaxExtent; }
inline bool stride_ok(int64_t stride, int64_t cols) { return stride >= cols && stride <= (int64_t(1) << 31); }

inline adasum_status_t check_matrix(const char* name, const void* p, int64_t stride, int64_t features, adasum_dtype_t dtype)
{
    if (!p)
        return fail(ADASUM_ERR_NULL, "%s is NULL", name);
    if (!aligned_to(p, operator_bytes(dtype)))
        return fail(ADASUM_ERR_ARG, "%s is not aligned to its element size", name);
    if (!stride_ok(stride, features))
        return fail(ADASUM_ERR_ARG, "stride %lld of %s is shorter than a row or out of range", (long long)stride, name);
    return ADASUM_OK;
}

// Multiprocessors of the current device (0: unknown), looked up once per device.
inline int device_sms()
{
    static std::atomic<int> cached[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64)
        return 0;
    if (cached[device] == 0) {
        int sms = 0;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)
            return 0;
        cached[device] = sms;
    }
    return cached[device];
}

// Division of vector indexes by the vectors of a row: q = floor(n / d) = high word of n * ceil(2^64 / d),
// exact while n * d < 2^64 (the rounding of the factor adds less than n * d / 2^64 / d < 1 / d).
struct RowDivider {
    uint64_t factor;
    uint32_t per_row;
};
inline RowDivider row_divider(int64_t per_row)
{
    return RowDivider{per_row > 1 ? ~uint64_t(0) / (uint64_t)per_row + 1 : 0, (uint32_t)per_row};
}

// How the elementwise kernels walk a matrix.  A thread handles vectors of eight consecutive elements; a warp takes a
// strip of up to 32 vectors of a row (of several rows, if rows are short) on a few rows below each other: all loads
// of a thread go out before the first is used, and its addresses are one sum apart.
constexpr int kStripThreads = 128;
// A matrix cut into strips: 2^lane_bits vectors of a row x 2^(5 - lane_bits) rows per lane row.
struct Strips {
    int64_t rows, features;
    int per_row;                         // vectors of a row
    int lane_bits;
    RowDivider strips_per_row;
    uint64_t warps;
};

inline bool plan_strips(int64_t rows, int64_t features, int64_t per_row, int rows_per_thread, Strips* s, unsigned* blocks)
{
    s->rows = rows;
    s->features = features;
    s->per_row = (int)per_row;
    s->lane_bits = 2;
    while (s->lane_bits < 5 && (1 << s->lane_bits) < s->per_row)
        ++s->lane_bits;
    const int64_t strips = (s->per_row + (1 << s->lane_bits) - 1) >> s->lane_bits;
    const int64_t band = (int64_t)rows_per_thread * (32 >> s->lane_bits);
    s->strips_per_row = row_divider(strips);
    s->warps = (uint64_t)((rows + band - 1) / band) * (uint64_t)strips;
    const uint64_t n = (s->warps + kStripThreads / 32 - 1) / (kStripThreads / 32);
    *blocks = (unsigned)n;
    return n <= 0x7fffffffu;
}

// Launches a kernel that begins with wait_for_previous_kernel(): it may be brought in while the stream's previous
// kernel still runs (one that called start_next_kernel()), which hides the launch.
template <typename... Params, typename... Args>
cudaError_t launch_after(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t shared_bytes, cudaStream_t stream,
                         Args&&... args)
{
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = shared_bytes;
    config.stream = stream;
    cudaLaunchAttribute attribute;
    attribute.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute.val.programmaticStreamSerializationAllowed = 1;
    config.attrs = &attribute;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, Params(args)...);
}

// Calls f with a value of the run-time type.
template <typename F>
void with_type(adasum_dtype_t dtype, F&& f)
{
    if (dtype == ADASUM_F32)
        f(float{});
    else if (dtype == ADASUM_F16)
        f(__half{});
    else
        f(__nv_bfloat16{});
}

// ---- device ----------------------------------------------------------------------------------------

__device__ __forceinline__ void divide_row(const RowDivider& d, uint64_t n, uint64_t& row, uint32_t& at)
{
    row = d.per_row > 1 ? __umul64hi(n, d.factor) : n;
    at = (uint32_t)(n - row * d.per_row);
}

// Until the previous kernel of the stream has ended and its writes are visible.  The first thing that every
// thread of a kernel launched by launch_after does: then "ended" also covers the kernels before that one.  Such a kernel
// reads global memory by coherent loads only: the non-coherent ones (__ldg) ask for memory that nobody writes in the
// kernel's whole life, and the previous kernel may write while this one waits.
__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// From here on the stream's next kernel may be brought in.
__device__ __forceinline__ void start_next_kernel() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <typename T>
struct TypeCode;
template <>
struct TypeCode<float> { static constexpr int value = ADASUM_F32; };
template <>
struct TypeCode<__half> { static constexpr int value = ADASUM_F16; };
template <>
struct TypeCode<__nv_bfloat16> { static constexpr int value = ADASUM_BF16; };

// Eight consecutive elements as floats; p is 16-byte aligned.  Plain loads: some callers overwrite the
// same elements afterwards (in place).
template <typename T>
__device__ __forceinline__ void load_eight(const T* p, float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        decode_vector<T>(*reinterpret_cast<const uint4*>(p), x);
    }
}
__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ float load_one(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float load_one(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// `count` (1 .. 8) elements, the rest zero.
template <typename T>
__device__ __forceinline__ void load_up_to_eight(const T* p, bool vec, int count, float (&x)[8])
{
    if (vec && count == 8) {
        load_eight(p, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[i] = i < count ? load_one(p + i) : 0.0f;
    }
}

// A thread's vectors: ROWS rows, one column.
struct Place {
    int64_t row0;            // first of the thread's rows; the next ones are `step` further
    int step;
    int column;              // first element
    int count;               // elements of the vector inside the matrix (<= 0: only padding)
    bool inside;             // the vector exists (padding included)
};
template <int ROWS>
__device__ __forceinline__ Place place_of(const Strips& s)
{
    const uint64_t warp = (uint64_t)blockIdx.x * (kStripThreads / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    uint64_t band;
    uint32_t strip;
    divide_row(s.strips_per_row, warp, band, strip);
    Place p;
    p.step = 32 >> s.lane_bits;
    p.row0 = (int64_t)band * (ROWS * p.step) + (lane >> s.lane_bits);
    const int vector = ((int)strip << s.lane_bits) + (lane & ((1 << s.lane_bits) - 1));
    p.inside = warp < s.warps && vector < s.per_row;
    p.column = vector * 8;
    p.count = p.inside ? (int)min((int64_t)8, s.features - p.column) : 0;
    return p;
}

}  // namespace adasum
