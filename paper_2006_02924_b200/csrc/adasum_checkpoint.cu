// Activations kept in 8 bits: save (with the activation's forward value), load, and the activation's
// gradient.  The gradients of a linear layer from the kept values are in adasum_weight_grad.cu.
//
// Every kernel here is one pass over a matrix, bound by HBM traffic.  A thread handles vectors of eight
// consecutive features; four neighbouring lanes hold a group of 32, so a group's largest magnitude is
// two shuffles away, and rows are filled up to whole groups, so a vector never leaves its row.  A warp takes a
// strip of up to 32 vectors of a row (of several rows, if rows are short) on kRows rows below each other: all
// loads of a thread go out before the first is used, and its addresses are one sum apart.
#include "adasum_operators.cuh"

namespace adasum {
namespace {

constexpr int kGroup = 32;                 // features that share a step
constexpr int kBlock = 256;
constexpr int kRows = 4;                   // vectors per thread, in as many rows: loads in flight

int64_t checkpoint_width(int64_t features) { return (features + kGroup - 1) / kGroup * kGroup; }

// ---- activations -------------------------------------------------------------------------------------

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInvSqrt2Pi = 0.3989422804014327f;
constexpr float kTanhScale = 0.7978845608028654f;     // sqrt(2 / pi)
constexpr float kTanhCubic = 0.044715f;

// Phi(x) and e = exp(-x^2 / 2) for 16-bit results.  Phi(-a) = e * r(a) with r(a) = erfcx(a / sqrt 2) / 2,
// and r is a polynomial of degree 6 without constant term in t = 1 / (1 + 0.31 a): a fit to r on
// 0 <= a <= 14 that levels out the relative error (5e-6, against 5e-4 / 2 for one rounding to fp16; beyond 14 both
// factors of the result vanish in 16 bits).  fp32 results call erfcf and expf.
__device__ __forceinline__ float normal_cdf_16(float x, float& e)
{
    const float a = fabsf(x);
    e = exp2_approx(-0.5f * kLog2e * x * x);
    const float t = reciprocal_approx(fmaf(0.31f, a, 1.0f));
    float r = -0.0739287332f;
    r = fmaf(r, t, 0.180449123f);
    r = fmaf(r, t, 0.0157461931f);
    r = fmaf(r, t, 0.133428877f);
    r = fmaf(r, t, 0.120441553f);
    r = fmaf(r, t, 0.123860669f);
    const float tail = r * t * e;
    return x < 0.0f ? tail : 1.0f - tail;
}

// s = 1 / (1 + exp(-z)), and 1 - s without the subtraction (which would leave nothing of it for large z).
template <bool WIDE>
__device__ __forceinline__ float logistic(float z, float& rest)
{
    const float e = WIDE ? expf(-fabsf(z)) : exp2_approx(-kLog2e * fabsf(z));
    const float large = WIDE ? 1.0f / (1.0f + e) : reciprocal_approx(1.0f + e), small = e * large;
    rest = z >= 0.0f ? small : large;
    return z >= 0.0f ? large : small;
}

// WIDE: the result is stored in fp32, so the accurate functions are used.
template <int ACT, bool WIDE>
__device__ __forceinline__ float activation(float x)
{
    if constexpr (ACT == ADASUM_ACT_RELU)
        return x > 0.0f ? x : 0.0f * x;
    if constexpr (ACT == ADASUM_ACT_GELU) {
        if constexpr (WIDE) {
            return x * (0.5f * erfcf(-0.70710678f * x));
        } else {
            float e;
            return x * normal_cdf_16(x, e);
        }
    }
    float rest;
    if constexpr (ACT == ADASUM_ACT_GELU_TANH)      // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        return x * logistic<WIDE>(2.0f * kTanhScale * x * fmaf(kTanhCubic * x, x, 1.0f), rest);
    if constexpr (ACT == ADASUM_ACT_SILU)
        return x * logistic<WIDE>(x, rest);
    return x;
}

template <int ACT, bool WIDE>
__device__ __forceinline__ float activation_slope(float x)
{
    if constexpr (ACT == ADASUM_ACT_RELU)
        return x > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == ADASUM_ACT_GELU) {         // Phi + x phi
        if constexpr (WIDE) {
            return fmaf(x * kInvSqrt2Pi, expf(-0.5f * x * x), 0.5f * erfcf(-0.70710678f * x));
        } else {
            float e;
            const float cdf = normal_cdf_16(x, e);
            return fmaf(x * kInvSqrt2Pi, e, cdf);
        }
    }
    float rest;
    if constexpr (ACT == ADASUM_ACT_GELU_TANH) {    // s + x s (1 - s) 2 u'
        const float s = logistic<WIDE>(2.0f * kTanhScale * x * fmaf(kTanhCubic * x, x, 1.0f), rest);
        const float du = 2.0f * kTanhScale * x * fmaf(3.0f * kTanhCubic * x, x, 1.0f);
        return fmaf(s * rest, du, s);
    }
    if constexpr (ACT == ADASUM_ACT_SILU) {
        const float s = logistic<WIDE>(x, rest);
        return fmaf(s * rest, x, s);
    }
    return 1.0f;
}

// ---- codes -------------------------------------------------------------------------------------------

// Step byte of a group from the bits of its largest magnitude (as an integer NaN > Inf > every number).
__device__ __forceinline__ uint32_t step_byte(uint32_t top_bits)
{
    const uint32_t exponent = top_bits >> 23;                // E + 127 (0: zero or subnormal)
    return exponent == 255 ? 255u : (uint32_t)max((int)exponent - 6, 1);
}
// 2^(byte - 127); Inf for 255, whose codes are 0, so that code * step is NaN.
__device__ __forceinline__ float step_value(uint32_t byte) { return __uint_as_float(byte << 23); }

// Four codes of x[0 .. 3] packed; inv = 1 / step.  Adding 1.5 * 2^23 rounds to an integer, ties to even,
// and leaves it in the low bits.  LIMIT: a magnitude may round to 128.
template <bool LIMIT>
__device__ __forceinline__ uint32_t pack_codes(const float* x, float inv)
{
    constexpr float kMagic = 12582912.0f;
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float r = fmaf(x[i], inv, kMagic);
        if constexpr (LIMIT)
            r = fminf(fmaxf(r, kMagic - 127.0f), kMagic + 127.0f);
        b[i] = __float_as_uint(r);
    }
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}
// Values of four packed codes: byte + 128 placed in the low bits of 2^23, 2^23 + 128 taken off again
// (exact), times the step (exact).
__device__ __forceinline__ void unpack_codes(uint32_t packed, float step, float* x)
{
    const uint32_t u = packed ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[i] = (__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540 + i)) - 8388736.0f) * step;
}

// ---- kernels -----------------------------------------------------------------------------------------

// A matrix cut into strips: 2^lane_bits vectors of a row x 2^(5 - lane_bits) rows per lane row.
struct Strips {
    int64_t rows, features, width;       // width: features filled up to whole groups
    int per_row;                         // vectors of a row, a multiple of 4
    int lane_bits;
    RowDivider strips_per_row;
    uint64_t warps;
};

struct Place {
    int64_t row0;            // first of the thread's rows; the next ones are `step` further
    int step;
    int column;              // first feature
    int count;               // features of the vector inside the matrix (<= 0: only padding)
    bool inside;             // the vector exists (padding included)
};
__device__ __forceinline__ Place place_of(const Strips& s)
{
    const uint64_t warp = (uint64_t)blockIdx.x * (kBlock / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    uint64_t band;
    uint32_t strip;
    divide_row(s.strips_per_row, warp, band, strip);
    Place p;
    p.step = 32 >> s.lane_bits;
    p.row0 = (int64_t)band * (kRows * p.step) + (lane >> s.lane_bits);
    const int vector = ((int)strip << s.lane_bits) + (lane & ((1 << s.lane_bits) - 1));
    p.inside = warp < s.warps && vector < s.per_row;
    p.column = vector * 8;
    p.count = p.inside ? (int)min((int64_t)8, s.features - p.column) : 0;
    return p;
}

// VEC: every row of x, y, grad and out starts on 16 bytes and features is a multiple of 8, so each vector is
// either whole or only padding.
template <bool VEC, typename T>
__device__ __forceinline__ void load_vector(const T* p, int count, float (&x)[8])
{
    if constexpr (VEC) {
        if (count > 0) {
            load_eight(p, x);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = 0.0f;
        }
    } else {
        load_up_to_eight(p, false, count, x);
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store_vector(T* p, int count, const float (&y)[8])
{
    if constexpr (VEC) {
        if (count > 0)
            store_vector_from_float<8>(p, TypeCode<T>::value, 0, y);
    } else {
        store_up_to_eight(p, false, count, y);
    }
}

template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(kBlock)
checkpoint_save_kernel(const __grid_constant__ Strips s, const T* x, int64_t x_stride, T* y, int64_t y_stride,
                       int8_t* codes, uint8_t* steps)
{
    constexpr bool WIDE = sizeof(T) == 4;
    const Place p = place_of(s);
    float v[kRows][8];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        load_vector<VEC>(x + row * x_stride + p.column, row < s.rows ? p.count : 0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            top = max(top, __float_as_uint(v[u][i]) & 0x7fffffffu);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const uint32_t byte = step_byte(top);
        const float inv = __uint_as_float((254u - min(byte, 254u)) << 23);
        uint2 packed;
        if ((top & 0x7fffffu) < 0x7f0000u) {     // the largest magnitude is below 127 steps (or a power of two less)
            packed = make_uint2(pack_codes<false>(v[u], inv), pack_codes<false>(v[u] + 4, inv));
        } else {
            packed = make_uint2(pack_codes<true>(v[u], inv), pack_codes<true>(v[u] + 4, inv));
        }
        if (byte == 255u)
            packed = make_uint2(0, 0);
        if (p.inside && row < s.rows) {
            const int64_t at = row * s.width + p.column;
            *reinterpret_cast<uint2*>(codes + at) = packed;
            if ((p.column & (kGroup - 1)) == 0)
                steps[at / kGroup] = (uint8_t)byte;
            if (y) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[u][i] = activation<ACT, WIDE>(v[u][i]);
                store_vector<VEC>(y + row * y_stride + p.column, p.count, v[u]);
            }
        }
    }
}

// ACT < 0: the values kept themselves; else out = grad * slope(kept value).
template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(kBlock)
checkpoint_apply_kernel(const __grid_constant__ Strips s, const int8_t* codes, const uint8_t* steps, const T* grad,
                        int64_t grad_stride, T* out, int64_t out_stride)
{
    constexpr bool WIDE = sizeof(T) == 4;
    const Place p = place_of(s);
    if (p.count <= 0)
        return;
    uint2 packed[kRows];
    uint32_t byte[kRows];
    float g[kRows][8];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        if (row < s.rows) {
            const int64_t at = row * s.width + p.column;
            packed[u] = *reinterpret_cast<const uint2*>(codes + at);
            byte[u] = steps[at / kGroup];
            if constexpr (ACT >= 0)
                load_vector<VEC>(grad + row * grad_stride + p.column, p.count, g[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        if (row < s.rows) {
            float x[8];
            unpack_codes(packed[u].x, step_value(byte[u]), x);
            unpack_codes(packed[u].y, step_value(byte[u]), x + 4);
            if constexpr (ACT >= 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    x[i] = g[u][i] * activation_slope<ACT, WIDE>(x[i]);
            }
            store_vector<VEC>(out + row * out_stride + p.column, p.count, x);
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------

adasum_status_t check_checkpoint(const void* checkpoint, int64_t rows, int64_t features, adasum_dtype_t dtype)
{
    if (!extent_ok(rows) || !extent_ok(features))
        return fail(ADASUM_ERR_ARG, "rows = %lld, features = %lld out of range", (long long)rows, (long long)features);
    if (!operator_dtype(dtype))
        return fail(ADASUM_ERR_DTYPE, "dtype %d is not fp32, fp16 or bf16", (int)dtype);
    if (rows == 0 || features == 0)
        return ADASUM_OK;
    if (!checkpoint)
        return fail(ADASUM_ERR_NULL, "checkpoint is NULL");
    if (!aligned_to(checkpoint, 16))
        return fail(ADASUM_ERR_ARG, "checkpoint is not 16-byte aligned");
    return ADASUM_OK;
}

adasum_status_t check_matrix(const char* name, const void* p, int64_t stride, int64_t features, adasum_dtype_t dtype)
{
    if (!p)
        return fail(ADASUM_ERR_NULL, "%s is NULL", name);
    if (!aligned_to(p, operator_bytes(dtype)))
        return fail(ADASUM_ERR_ARG, "%s is not aligned to its element size", name);
    if (!stride_ok(stride, features))
        return fail(ADASUM_ERR_ARG, "stride %lld of %s is shorter than a row or out of range", (long long)stride, name);
    return ADASUM_OK;
}

bool plan_strips(int64_t rows, int64_t features, Strips* s, unsigned* blocks)
{
    s->rows = rows;
    s->features = features;
    s->width = checkpoint_width(features);
    s->per_row = (int)(s->width / 8);
    s->lane_bits = 2;
    while (s->lane_bits < 5 && (1 << s->lane_bits) < s->per_row)
        ++s->lane_bits;
    const int64_t strips = (s->per_row + (1 << s->lane_bits) - 1) >> s->lane_bits;
    const int64_t band = (int64_t)kRows * (32 >> s->lane_bits);
    s->strips_per_row = row_divider(strips);
    s->warps = (uint64_t)((rows + band - 1) / band) * (uint64_t)strips;
    const uint64_t n = (s->warps + kBlock / 32 - 1) / (kBlock / 32);
    *blocks = (unsigned)n;
    return n <= 0x7fffffffu;
}

// Calls f with a value of the run-time type, the constant of the run-time activation, or of a truth value.
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
template <int N>
struct Constant { static constexpr int value = N; };
template <typename F>
void with_activation(adasum_activation_t act, F&& f)
{
    switch (act) {
    case ADASUM_ACT_NONE: f(Constant<ADASUM_ACT_NONE>{}); break;
    case ADASUM_ACT_RELU: f(Constant<ADASUM_ACT_RELU>{}); break;
    case ADASUM_ACT_GELU: f(Constant<ADASUM_ACT_GELU>{}); break;
    case ADASUM_ACT_GELU_TANH: f(Constant<ADASUM_ACT_GELU_TANH>{}); break;
    case ADASUM_ACT_SILU: f(Constant<ADASUM_ACT_SILU>{}); break;
    }
}
template <typename F>
void with_flag(bool flag, F&& f)
{
    if (flag)
        f(Constant<1>{});
    else
        f(Constant<0>{});
}

template <typename T, int ACT>
void launch_apply(const void* checkpoint, const Strips& s, unsigned blocks, const void* grad, int64_t grad_stride,
                  void* out, int64_t out_stride, cudaStream_t stream)
{
    const int8_t* codes = static_cast<const int8_t*>(checkpoint);
    const bool vec = s.features % 8 == 0 && rows_aligned(grad, grad_stride, sizeof(T)) && rows_aligned(out, out_stride, sizeof(T));
    with_flag(vec, [&](auto v) {
        checkpoint_apply_kernel<T, ACT, decltype(v)::value != 0><<<blocks, kBlock, 0, stream>>>(
            s, codes, reinterpret_cast<const uint8_t*>(codes + s.rows * s.width), static_cast<const T*>(grad), grad_stride,
            static_cast<T*>(out), out_stride);
    });
}

bool known_activation(int act) { return act >= ADASUM_ACT_NONE && act <= ADASUM_ACT_SILU; }

adasum_status_t launched(cudaStream_t stream, int kernel)
{
    ADASUM_CUDA_CHECK(cudaGetLastError());
    profile_mark(stream, kernel, 0, 0, false);
    return ADASUM_OK;
}

}  // namespace
}  // namespace adasum

extern "C" {

size_t adasum_checkpoint_bytes(int64_t rows, int64_t features)
{
    using namespace adasum;
    if (!extent_ok(rows) || !extent_ok(features))
        return 0;
    const int64_t width = checkpoint_width(features);
    return (size_t)(rows * width + rows * (width / kGroup));
}

adasum_status_t adasum_checkpoint_save(const void* x, int64_t x_stride, int64_t rows, int64_t features,
                                       adasum_dtype_t dtype, adasum_activation_t act, void* y, int64_t y_stride,
                                       void* checkpoint, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    adasum_status_t status = check_checkpoint(checkpoint, rows, features, dtype);
    if (status != ADASUM_OK)
        return status;
    if (!known_activation(act))
        return fail(ADASUM_ERR_ARG, "unknown activation %d", (int)act);
    if (rows == 0 || features == 0)
        return ADASUM_OK;
    if ((status = check_matrix("x", x, x_stride, features, dtype)) != ADASUM_OK)
        return status;
    if (y && (status = check_matrix("y", y, y_stride, features, dtype)) != ADASUM_OK)
        return status;
    const size_t x_bytes = matrix_span(rows, features, x_stride, operator_bytes(dtype));
    const size_t y_bytes = y ? matrix_span(rows, features, y_stride, operator_bytes(dtype)) : 0;
    const size_t c_bytes = adasum_checkpoint_bytes(rows, features);
    if (spans_overlap(x, x_bytes, y, y_bytes) && !(x == y && x_stride == y_stride))
        return fail(ADASUM_ERR_ARG, "y overlaps x without being the same matrix");
    if (spans_overlap(checkpoint, c_bytes, x, x_bytes) || spans_overlap(checkpoint, c_bytes, y, y_bytes))
        return fail(ADASUM_ERR_ARG, "checkpoint overlaps x or y");
    Strips s;
    unsigned blocks;
    if (!plan_strips(rows, features, &s, &blocks))
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)features);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    with_type(dtype, [&](auto t) {
        with_activation(act, [&](auto a) {
            using T = decltype(t);
            const bool vec = features % 8 == 0 && rows_aligned(x, x_stride, sizeof(T)) && rows_aligned(y, y_stride, sizeof(T));
            int8_t* codes = static_cast<int8_t*>(checkpoint);
            with_flag(vec, [&](auto v) {
                checkpoint_save_kernel<T, decltype(a)::value, decltype(v)::value != 0><<<blocks, kBlock, 0, stream>>>(
                    s, static_cast<const T*>(x), x_stride, static_cast<T*>(y), y_stride, codes,
                    reinterpret_cast<uint8_t*>(codes + s.rows * s.width));
            });
        });
    });
    return launched(stream, ADASUM_KERNEL_CHECKPOINT_SAVE);
}

adasum_status_t adasum_checkpoint_load(const void* checkpoint, int64_t rows, int64_t features, void* out,
                                       int64_t out_stride, adasum_dtype_t dtype, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    adasum_status_t status = check_checkpoint(checkpoint, rows, features, dtype);
    if (status != ADASUM_OK || rows == 0 || features == 0)
        return status;
    if ((status = check_matrix("out", out, out_stride, features, dtype)) != ADASUM_OK)
        return status;
    if (spans_overlap(checkpoint, adasum_checkpoint_bytes(rows, features), out,
                      matrix_span(rows, features, out_stride, operator_bytes(dtype))))
        return fail(ADASUM_ERR_ARG, "checkpoint overlaps out");
    Strips s;
    unsigned blocks;
    if (!plan_strips(rows, features, &s, &blocks))
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)features);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    with_type(dtype, [&](auto t) { launch_apply<decltype(t), -1>(checkpoint, s, blocks, nullptr, 0, out, out_stride, stream); });
    return launched(stream, ADASUM_KERNEL_CHECKPOINT_LOAD);
}

adasum_status_t adasum_checkpoint_act_grad(const void* checkpoint, int64_t rows, int64_t features,
                                           adasum_activation_t act, const void* grad_out, int64_t grad_out_stride,
                                           adasum_dtype_t dtype, void* grad_in, int64_t grad_in_stride,
                                           void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    adasum_status_t status = check_checkpoint(checkpoint, rows, features, dtype);
    if (status != ADASUM_OK)
        return status;
    if (!known_activation(act))
        return fail(ADASUM_ERR_ARG, "unknown activation %d", (int)act);
    if (rows == 0 || features == 0)
        return ADASUM_OK;
    if ((status = check_matrix("grad_out", grad_out, grad_out_stride, features, dtype)) != ADASUM_OK ||
        (status = check_matrix("grad_in", grad_in, grad_in_stride, features, dtype)) != ADASUM_OK)
        return status;
    const size_t out_bytes = matrix_span(rows, features, grad_out_stride, operator_bytes(dtype));
    const size_t in_bytes = matrix_span(rows, features, grad_in_stride, operator_bytes(dtype));
    if (spans_overlap(grad_out, out_bytes, grad_in, in_bytes) &&
        !(grad_out == grad_in && grad_out_stride == grad_in_stride))
        return fail(ADASUM_ERR_ARG, "grad_in overlaps grad_out without being the same matrix");
    if (spans_overlap(checkpoint, adasum_checkpoint_bytes(rows, features), grad_in, in_bytes))
        return fail(ADASUM_ERR_ARG, "checkpoint overlaps grad_in");
    Strips s;
    unsigned blocks;
    if (!plan_strips(rows, features, &s, &blocks))
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)features);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    with_type(dtype, [&](auto t) {
        with_activation(act, [&](auto a) {
            launch_apply<decltype(t), decltype(a)::value>(checkpoint, s, blocks, grad_out, grad_out_stride, grad_in,
                                                          grad_in_stride, stream);
        });
    });
    return launched(stream, ADASUM_KERNEL_ACT_GRAD);
}

}  // extern "C"
