// Activations kept in 8 bits: save (with the activation's forward value), load, and the activation's
// gradient.  The gradients of a linear layer from the kept values are in adasum_weight_grad.cu.
//
// Every kernel here is one pass over a matrix, bound by HBM traffic.  A thread handles vectors of eight
// consecutive features; four neighbouring lanes hold a group of 32, so a group's largest magnitude is
// two shuffles away, and rows are filled up to whole groups, so a vector never leaves its row.
#include "adasum_vectors.cuh"

namespace adasum {
namespace {

constexpr int kGroup = 32;                 // features that share a step
// Vectors per thread, in as many rows: loads in flight.  Measured on 16384 x 4096 bf16 (1, 2, 4, 8 rows): saving with
// GELU 80, 72, 70, 82 us; GELU's gradient 78, 78, 82, 121 us (72 us with two rows and registers for 16 blocks per
// multiprocessor); loading 43, 41, 45, 55 us.
constexpr int kSaveRows = 4;
constexpr int kApplyRows = 2;

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
__device__ __forceinline__ Pair negative(Pair a) { return Pair{a.v ^ 0x8000000080000000ull}; }
__device__ __forceinline__ Pair magnitude(Pair a) { return Pair{a.v & 0x7fffffff7fffffffull}; }

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eLow = (float)(1.4426950408889634 - (double)kLog2e);
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInvSqrt2Pi = 0.3989422804014327f;
constexpr float kTanhScale = 0.7978845608028654f;     // sqrt(2 / pi)
constexpr float kTanhCubic = 0.044715f;

// The normal distribution function's tail: Phi(-a) = e * r(a) for a >= 0, with e = exp(-a^2 / 2) and
// r(a) = erfcx(a / sqrt 2) / 2.  r is a polynomial without constant term in t = 1 / (1 + p a), fitted to r on
// 0 <= a <= 14 so that the relative error is level: for 16-bit results p = 0.31 and degree 6 (5e-6, against 5e-4 / 2 for one
// rounding to fp16), for fp32 p = 0.34 and degree 9 (3e-8; 3e-7 as evaluated, what erfcf has, at half its cost).
// Beyond 14 the tail vanishes in either type.  Returns r.
template <bool WIDE>
__device__ __forceinline__ Pair normal_tail(Pair a, Pair& e)
{
    if constexpr (WIDE) {
        // a^2 / 2 log2(e) with its rounding errors (twice 2^-24 of up to 100), which the exponential would multiply
        const Pair scale = both(-0.5f * kLog2e), square = a * a;
        const Pair y = square * scale;
        const Pair square_low = fma2(a, a, negative(square));
        const Pair low = fma2(square_low, scale, fma2(square, both(-0.5f * kLog2eLow), fma2(square, scale, negative(y))));
        e = each(y, exp2_approx);
        e = fma2(e, low * both(kLn2), e);
        const Pair t = each(fma2(both(0.34f), a, both(1.0f)), reciprocal_approx);
        Pair r = both(-0.026122383f);
        r = fma2(r, t, both(0.139508666f));
        r = fma2(r, t, both(-0.273151377f));
        r = fma2(r, t, both(0.202203477f));
        r = fma2(r, t, both(-0.0447323639f));
        r = fma2(r, t, both(0.115364844f));
        r = fma2(r, t, both(0.115196281f));
        r = fma2(r, t, both(0.136112377f));
        r = fma2(r, t, both(0.135620494f));
        return r * t;
    }
    e = each(a * a * both(-0.5f * kLog2e), exp2_approx);
    const Pair t = each(fma2(both(0.31f), a, both(1.0f)), reciprocal_approx);
    Pair r = both(-0.0739287332f);
    r = fma2(r, t, both(0.180449123f));
    r = fma2(r, t, both(0.0157461931f));
    r = fma2(r, t, both(0.133428877f));
    r = fma2(r, t, both(0.120441553f));
    r = fma2(r, t, both(0.123860669f));
    return r * t;
}
// |x|, for fp32 results up to 40 only (the square of a large one would not be a number); NaN stays.
template <bool WIDE>
__device__ __forceinline__ Pair tail_argument(Pair x)
{
    if constexpr (!WIDE)
        return magnitude(x);
    return each(magnitude(x), [](float a) {
        float m;
        asm("min.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(40.0f));
        return m;
    });
}
// x < 0: tail; else 1 - tail, as side * tail + (1 - side) / 2 with side = -sign(x).
__device__ __forceinline__ Pair tail_or_rest(Pair x, Pair tail)
{
    const Pair side{((~x.v) & 0x8000000080000000ull) | 0x3f8000003f800000ull};
    return fma2(side, tail, fma2(side, both(-0.5f), both(0.5f)));
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
template <bool WIDE>
__device__ __forceinline__ Pair logistic(Pair z, Pair& rest)
{
    const float2 v = values_of(z);
    float2 s, r;
    s.x = logistic<WIDE>(v.x, r.x);
    s.y = logistic<WIDE>(v.y, r.y);
    rest = pair_of(r.x, r.y);
    return pair_of(s.x, s.y);
}

// WIDE: the result is stored in fp32, so the accurate functions are used.
template <int ACT, bool WIDE>
__device__ __forceinline__ Pair activation(Pair x)
{
    if constexpr (ACT == ADASUM_ACT_RELU)
        return each(x, [](float a) {
            float m;                                // NaN stays
            asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(0.0f));
            return m;
        });
    if constexpr (ACT == ADASUM_ACT_GELU) {
        Pair e;
        const Pair r = normal_tail<WIDE>(tail_argument<WIDE>(x), e);
        return x * tail_or_rest(x, r * e);
    }
    Pair rest;
    if constexpr (ACT == ADASUM_ACT_GELU_TANH)      // (1 + tanh u) / 2 = 1 / (1 + exp(-2 u))
        return x * logistic<WIDE>(both(2.0f * kTanhScale) * x * fma2(both(kTanhCubic) * x, x, both(1.0f)), rest);
    if constexpr (ACT == ADASUM_ACT_SILU)
        return x * logistic<WIDE>(x, rest);
    return x;
}

// x: a kept value whose step is at most slope_step().
template <int ACT, bool WIDE>
__device__ __forceinline__ Pair activation_slope(Pair x)
{
    if constexpr (ACT == ADASUM_ACT_RELU)
        return each(x, [](float a) { return a > 0.0f ? 1.0f : 0.0f * fabsf(a); });      // NaN stays
    if constexpr (ACT == ADASUM_ACT_GELU) {         // Phi + x phi; at -a: e (r - a / sqrt(2 pi)), at a: 1 minus that
        Pair e;
        const Pair a = tail_argument<WIDE>(x), r = normal_tail<WIDE>(a, e);
        return tail_or_rest(x, fma2(a, both(-kInvSqrt2Pi), r) * e);
    }
    Pair rest;
    if constexpr (ACT == ADASUM_ACT_GELU_TANH && WIDE) {
        // s + s (1 - s) x z', with z = x (a + b x^2); at -|x|, where s is small and has no rounding near 1 in it, and from
        // there to |x| as 1 minus that (error 4.3e-8 of the norm, against 6.4e-8 from s and 1 - s at x itself)
        constexpr float a = 2.0f * kTanhScale, b = 2.0f * kTanhScale * kTanhCubic;
        const Pair m = magnitude(x), square = m * m, z = m * fma2(both(b), square, both(a));
        const Pair e = each(z, [](float v) { return expf(-v); });
        const Pair large = each(e, [](float v) { return 1.0f / (1.0f + v); }), small = e * large;
        return tail_or_rest(x, fma2(small * large, m * fma2(both(-3.0f * b), square, both(-a)), small));
    }
    if constexpr (ACT == ADASUM_ACT_GELU_TANH) {    // with z = v (1 + c x^2): x z' = 3 z - 2 v
        const Pair v = both(2.0f * kTanhScale) * x, z = v * fma2(both(kTanhCubic) * x, x, both(1.0f));
        const Pair s = logistic<WIDE>(z, rest);
        return fma2(s * rest, fma2(both(3.0f), z, both(-2.0f) * v), s);
    }
    if constexpr (ACT == ADASUM_ACT_SILU) {
        const Pair s = logistic<WIDE>(x, rest);
        return fma2(s * rest, x, s);
    }
    return both(1.0f);
}

// ---- codes -------------------------------------------------------------------------------------------

// Step byte of a group from the bits of its largest magnitude.
__device__ __forceinline__ uint32_t step_byte(uint32_t top_bits)
{
    const uint32_t exponent = top_bits >> 23;                // E + 127 (0: zero or subnormal)
    return exponent == 255 ? 255u : (uint32_t)max((int)exponent - 6, 1);
}
// 2^(byte - 127); Inf for 255, whose codes are 0, so that code * step is NaN.
__device__ __forceinline__ float step_value(uint32_t byte) { return __uint_as_float(byte << 23); }
// The step that a group's slopes are computed with.  tanh-GELU has powers of x that would overflow beside factors that
// have become zero, and make NaN of the slope: a step of more than 2^30 is taken for 2^30, which leaves a code of 0
// at 0 and all others at magnitudes (2^30 .. 2^37) where the slope is 1 or 0.
template <int ACT>
__device__ __forceinline__ float slope_step(uint32_t byte)
{
    return step_value(ACT == ADASUM_ACT_GELU_TANH && byte != 255u ? min(byte, 127u + 30u) : byte);
}

// Four codes of two pairs packed; inv = 1 / step.  Adding 1.5 * 2^23 rounds to an integer, ties to even,
// and leaves it in the low bits.  LIMIT: a magnitude may round to 128.
template <bool LIMIT>
__device__ __forceinline__ uint32_t pack_codes(Pair x, Pair y, Pair inv)
{
    constexpr float kMagic = 12582912.0f;
    float2 a = values_of(fma2(x, inv, both(kMagic))), b = values_of(fma2(y, inv, both(kMagic)));
    if constexpr (LIMIT) {
        auto limit = [](float r) { return fminf(fmaxf(r, kMagic - 127.0f), kMagic + 127.0f); };
        a = make_float2(limit(a.x), limit(a.y));
        b = make_float2(limit(b.x), limit(b.y));
    }
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                       __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
}
// Values of four packed codes: byte + 128 placed in the low bits of 2^23, 2^23 + 128 taken off again
// (exact), times the step (exact).
__device__ __forceinline__ void unpack_codes(uint32_t packed, Pair step, Pair& x, Pair& y)
{
    const uint32_t u = packed ^ 0x80808080u;
    auto value = [&](uint32_t selector) { return __uint_as_float(__byte_perm(u, 0x4b000000u, selector)); };
    const Pair offset = both(-8388736.0f);
    x = (pair_of(value(0x7540), value(0x7541)) + offset) * step;
    y = (pair_of(value(0x7542), value(0x7543)) + offset) * step;
}

// ---- kernels -----------------------------------------------------------------------------------------

// 16384 x 4096 bf16: GELU 70 us (4.8 TB/s, 77 % of the issue slots: bound by both), ReLU 55 us (6.1 TB/s); fp32 GELU
// 96 us (6.3 TB/s).
template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(kStripThreads)
checkpoint_save_kernel(const __grid_constant__ Strips s, const T* x, int64_t x_stride, T* y, int64_t y_stride,
                       int8_t* codes, uint8_t* steps)
{
    constexpr bool WIDE = sizeof(T) == 4;
    const Place p = place_of<kSaveRows>(s);
    Raw<T> raw[kSaveRows];
#pragma unroll
    for (int u = 0; u < kSaveRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        raw[u] = load_vector<VEC>(x + row * x_stride + p.column, row < s.rows ? p.count : 0);
    }
#pragma unroll
    for (int u = 0; u < kSaveRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        uint32_t top = largest(raw[u]);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const uint32_t byte = step_byte(top);
        const Pair inv = both(__uint_as_float((254u - min(byte, 254u)) << 23));
        Eight v = decode(raw[u]);
        uint2 packed;
        if ((top & 0x7fffffu) < 0x7f0000u) {     // the largest magnitude is below 127 steps
            packed = make_uint2(pack_codes<false>(v.p[0], v.p[1], inv), pack_codes<false>(v.p[2], v.p[3], inv));
        } else {
            packed = make_uint2(pack_codes<true>(v.p[0], v.p[1], inv), pack_codes<true>(v.p[2], v.p[3], inv));
        }
        if (byte == 255u)
            packed = make_uint2(0, 0);
        if (p.inside && row < s.rows) {
            const int64_t at = row * (int64_t)s.per_row * 8 + p.column;
            *reinterpret_cast<uint2*>(codes + at) = packed;
            if ((p.column & (kGroup - 1)) == 0)
                steps[at / kGroup] = (uint8_t)byte;
            if (y) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v.p[i] = activation<ACT, WIDE>(v.p[i]);
                store_vector<VEC>(y + row * y_stride + p.column, p.count, v);
            }
        }
    }
}

// ACT < 0: the values kept themselves; else out = grad * slope(kept value).  16384 x 4096 bf16: load 41 us (5 TB/s,
// two thirds of it writes), GELU 73 us (4.6 TB/s, instruction issue), ReLU 55 us (6.1 TB/s); fp32 GELU 111 us
// (5.5 TB/s).
template <typename T, int ACT, bool VEC>
__global__ void __launch_bounds__(kStripThreads, sizeof(T) == 2 && VEC ? 16 : 8)
checkpoint_apply_kernel(const __grid_constant__ Strips s, const int8_t* codes, const uint8_t* steps, const T* grad,
                        int64_t grad_stride, T* out, int64_t out_stride)
{
    constexpr bool WIDE = sizeof(T) == 4;
    const Place p = place_of<kApplyRows>(s);
    if (p.count <= 0)
        return;
    uint2 packed[kApplyRows];
    uint32_t byte[kApplyRows];
    Raw<T> g[kApplyRows];
#pragma unroll
    for (int u = 0; u < kApplyRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        if (row < s.rows) {
            const int64_t at = row * (int64_t)s.per_row * 8 + p.column;
            packed[u] = *reinterpret_cast<const uint2*>(codes + at);
            byte[u] = steps[at / kGroup];
            if constexpr (ACT >= 0)
                g[u] = load_vector<VEC>(grad + row * grad_stride + p.column, p.count);
        }
    }
#pragma unroll
    for (int u = 0; u < kApplyRows; ++u) {
        const int64_t row = p.row0 + u * p.step;
        if (row < s.rows) {
            const Pair step = both(slope_step<ACT>(byte[u]));
            Eight x;
            unpack_codes(packed[u].x, step, x.p[0], x.p[1]);
            unpack_codes(packed[u].y, step, x.p[2], x.p[3]);
            if constexpr (ACT >= 0) {
                const Eight d = decode(g[u]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x.p[i] = d.p[i] * activation_slope<ACT, WIDE>(x.p[i]);
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

// Calls f with the constant of the run-time activation, or of a truth value.
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
        checkpoint_apply_kernel<T, ACT, decltype(v)::value != 0><<<blocks, kStripThreads, 0, stream>>>(
            s, codes, reinterpret_cast<const uint8_t*>(codes + s.rows * (int64_t)s.per_row * 8), static_cast<const T*>(grad), grad_stride,
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
    if (!plan_strips(rows, features, checkpoint_width(features) / 8, kSaveRows, &s, &blocks))
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)features);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    with_type(dtype, [&](auto t) {
        with_activation(act, [&](auto a) {
            using T = decltype(t);
            const bool vec = features % 8 == 0 && rows_aligned(x, x_stride, sizeof(T)) && rows_aligned(y, y_stride, sizeof(T));
            int8_t* codes = static_cast<int8_t*>(checkpoint);
            with_flag(vec, [&](auto v) {
                checkpoint_save_kernel<T, decltype(a)::value, decltype(v)::value != 0><<<blocks, kStripThreads, 0, stream>>>(
                    s, static_cast<const T*>(x), x_stride, static_cast<T*>(y), y_stride, codes,
                    reinterpret_cast<uint8_t*>(codes + s.rows * (int64_t)s.per_row * 8));
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
    if (!plan_strips(rows, features, checkpoint_width(features) / 8, kApplyRows, &s, &blocks))
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
    if (!plan_strips(rows, features, checkpoint_width(features) / 8, kApplyRows, &s, &blocks))
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
