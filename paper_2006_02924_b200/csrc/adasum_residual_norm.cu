// The joint between two blocks of a residual network, and its gradients:
//
//     n = post(x)                                           norm after the block (or x itself)
//     h = residual_scale * residual + branch_scale * gate * dropout(n)
//     y = pre(h)                                            norm before the next block
//
// A norm is u = x rstd or (x - mean) rstd, times a weight, plus a bias; rstd = (mean(u'^2) + eps)^(-1/2) of the centred (or
// raw) values.  With v the gradient of u (that of the result times the weight), the gradient of its input is
//
//     rstd (v - u mean(u v) [- mean(v)])                    [layer norm only]
//
// All rows of x, residual, h and y are read or written once: HBM traffic bounds both directions.  A group of threads
// owns whole rows, eight neighbouring columns per thread, two rows at a time (one exchange of sums serves both), so a
// thread meets the same columns in every row and sums the vectors' gradients in registers.  A group is 4 to 32 lanes
// of a warp for up to 256 columns, up to 16 warps of a block for up to 4096, and a cluster of blocks, which exchange
// their sums through distributed shared memory, beyond that.
//
// Gradients of vectors are summed per block and then over the blocks by a second kernel, both in a fixed order: the
// results are the same from run to run.  With a gate for every so many rows, the rows of one gate row are cut into
// pieces that a group walks one after another, and each piece leaves its own sum.
#include "adasum_random.cuh"
#include "adasum_vectors.cuh"

namespace adasum {
namespace {

constexpr int kRows = 2;                   // rows that a group handles at a time
constexpr int kMaxThreads = 512;
constexpr int kMaxWarps = kMaxThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int64_t kMaxFeatures = (int64_t)kMaxCluster * kMaxThreads * 8;
constexpr int kMaxBlocks = 148 * 4;        // blocks that leave sums of the vectors' gradients
constexpr int kVectors = 5;                // gradients of vectors: post weight, post bias, pre weight, pre bias, gate

// A vector of parameters (p = nullptr: all `fill`).
struct Vector {
    const void* p;
    int dtype;
    bool aligned;
};

// How rows are dealt out.  Rows come in units of `unit_rows` (the last unit of a gate row may be shorter); unit k of a
// group is unit number group + k * groups.
struct Deal {
    int lanes;                 // lanes of a group inside a warp
    int warps;                 // warps of a group inside a block
    int groups_per_block;
    int cluster;               // blocks of a group
    int block_vectors;         // vectors of eight columns per block
    uint32_t groups;           // of the whole launch
    uint32_t units, steps, rounds;     // a unit takes `steps` times kRows rows; a group `rounds` units
    uint32_t pieces;           // units per gate row
    int64_t gate_rows_span;    // rows of a gate row (all rows, without a gate's gradient)
    int64_t unit_rows;
};

struct NormArgs {
    Deal deal;
    int64_t rows;
    int features, post, pre;
    float inv_features, eps, branch_scale, residual_scale;
    Vector post_weight, post_bias, pre_weight, pre_bias, gate;
    int64_t gate_stride;
    RowDivider rows_per_gate;
    Dropout drop;
    const void *x, *residual, *h, *grad_y, *grad_h;
    void *out_h, *out_y, *grad_x, *grad_residual;
    int64_t x_stride, residual_stride, h_stride, y_stride, grad_y_stride, grad_h_stride, grad_x_stride, grad_residual_stride;
    float* stats;              // [post mean, post rstd, pre mean, pre rstd][rows]
    // gradients of the vectors
    bool want[kVectors];
    float* parts;              // [block or cluster][kVectors][columns]
    int64_t columns;           // whole vectors
    float* gate_parts;         // [unit][columns], where a gate row's sum is cut; nullptr: written at once
    void* grad_gate;
    int grad_gate_dtype;
    float gate_scale;
    bool accumulate, gate_by_unit;
    bool branch;               // there is a branch whose gradient is wanted
};

__device__ __forceinline__ void load_vector_of(const Vector& v, int64_t at, int count, float fill, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = fill;
    if (v.p == nullptr || count <= 0)
        return;
    if (v.dtype == ADASUM_F32)
        load_up_to_eight(static_cast<const float*>(v.p) + at, v.aligned, count, x);
    else if (v.dtype == ADASUM_F16)
        load_up_to_eight(static_cast<const __half*>(v.p) + at, v.aligned, count, x);
    else
        load_up_to_eight(static_cast<const __nv_bfloat16*>(v.p) + at, v.aligned, count, x);
}

// 1 / sqrt(v), one Newton step on the approximation (its 2^-23 shows in fp32 results).
__device__ __forceinline__ float reciprocal_root(float v)
{
    const float y = rsqrtf(v);
    return v > 0.0f && v < __uint_as_float(0x7f800000u) ? fmaf(0.5f * y, fmaf(-v * y, y, 1.0f), y) : y;
}

// A thread's place in its group.
struct Member {
    const Deal& deal;
    uint32_t group;
    int vector;                // of the row
    int warp_in_group, slot;   // slot: the group's number inside the block
    uint32_t rank;             // of the block in its cluster
    uint32_t parity = 0;
    __device__ __forceinline__ explicit Member(const Deal& d) : deal(d)
    {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        rank = 0;
        uint32_t block = blockIdx.x;
        if (d.cluster > 1) {
            rank = blockIdx.x % d.cluster;
            block = blockIdx.x / d.cluster;
        }
        if (d.warps == 1) {
            slot = threadIdx.x / d.lanes;
            warp_in_group = 0;
            vector = lane & (d.lanes - 1);
        } else {
            slot = warp / d.warps;
            warp_in_group = warp - slot * d.warps;
            vector = warp_in_group * 32 + lane;
        }
        if (vector >= d.block_vectors)
            vector = 1 << 28;                        // beyond every row
        else
            vector += rank * d.block_vectors;
        group = block * d.groups_per_block + slot;
    }
    __device__ __forceinline__ bool leads() const
    {
        return (deal.warps == 1 ? (threadIdx.x & (deal.lanes - 1)) == 0 : warp_in_group == 0 && (threadIdx.x & 31) == 0) && rank == 0;
    }
};

// A cluster's blocks write into each other's shared memory: none may do so before the other runs.
__device__ __forceinline__ void blocks_present(const Deal& d)
{
    if (d.cluster > 1)
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct Exchange {
    float warp_sum[2][kMaxWarps][4];
    float block_sum[2][kMaxCluster][4];
};

// Sums over the group of N (<= 4) values per thread, in a fixed order; every thread gets them.  All threads of the
// block call it equally often.  Two buffers in turn: a thread that is two calls ahead has passed a barrier that
// the others reach only after reading.
template <int N>
__device__ __forceinline__ void group_sum(Member& m, Exchange& e, float (&v)[N])
{
    const Deal& d = m.deal;
    for (int step = (d.warps == 1 ? d.lanes : 32) >> 1; step > 0; step >>= 1) {
#pragma unroll
        for (int n = 0; n < N; ++n)
            v[n] += __shfl_xor_sync(0xffffffffu, v[n], step);
    }
    if (d.warps == 1)
        return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n)
            e.warp_sum[m.parity][warp][n] = v[n];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(m.slot + 1), "r"(32 * d.warps) : "memory");
    const int from = lane & (kMaxWarps - 1);
#pragma unroll
    for (int n = 0; n < N; ++n)
        v[n] = from < d.warps ? e.warp_sum[m.parity][m.slot * d.warps + from][n] : 0.0f;
#pragma unroll
    for (int step = kMaxWarps / 2; step > 0; step >>= 1) {
#pragma unroll
        for (int n = 0; n < N; ++n)
            v[n] += __shfl_xor_sync(0xffffffffu, v[n], step);
    }
    if (d.cluster > 1) {
        if (threadIdx.x < (unsigned)d.cluster) {
            const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(&e.block_sum[m.parity][m.rank][0]));
            uint32_t remote;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(mine), "r"(threadIdx.x));
#pragma unroll
            for (int n = 0; n < N; ++n)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote + 4 * n), "f"(v[n]) : "memory");
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float total = 0.0f;
            for (int c = 0; c < d.cluster; ++c)
                total += e.block_sum[m.parity][c][n];
            v[n] = total;
        }
    }
    m.parity ^= 1;
}

__device__ __forceinline__ bool in_range(float s) { return fabsf(s) < __uint_as_float(0x7f800000u); }
// Has a sum of the group (of the warp's groups) left fp32's range, or is not a number?  The same answer for all its threads.
__device__ __forceinline__ bool any_out_of_range(const Member& m, const float (&s)[kRows])
{
    bool out = false;
#pragma unroll
    for (int u = 0; u < kRows; ++u)
        out |= !in_range(s[u]);
    return m.deal.warps == 1 ? __any_sync(0xffffffffu, out) : out;
}

// Statistics of kRows rows; x becomes the normalised values.  Elements beyond the row are zeros and stay out.
__device__ __forceinline__ void normalise(Member& m, Exchange& e, const NormArgs& a, int kind, int count, float (&x)[kRows][8],
                                          float (&mean)[kRows], float (&rstd)[kRows])
{
    float s[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
        mean[u] = 0.0f;
    if (kind == ADASUM_NORM_LAYER) {
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            s[u] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[u] += x[u][i];
        }
        group_sum(m, e, s);
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            mean[u] = s[u] * a.inv_features;
        if (any_out_of_range(m, s)) {            // such rows are divided before they are added
            float t[kRows];
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                t[u] = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    t[u] = fmaf(x[u][i], a.inv_features, t[u]);
            }
            group_sum(m, e, t);
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                mean[u] = in_range(s[u]) ? mean[u] : t[u];
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[u][i] = i < count ? x[u][i] - mean[u] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        s[u] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s[u] = fmaf(x[u][i], x[u][i], s[u]);
    }
    group_sum(m, e, s);
#pragma unroll
    for (int u = 0; u < kRows; ++u)
        rstd[u] = reciprocal_root(fmaf(s[u], a.inv_features, a.eps));
    if (any_out_of_range(m, s)) {                // such rows: of the values times 2^-96
        const float down = __uint_as_float((127u - 96u) << 23);
        float t[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            t[u] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                t[u] = fmaf(x[u][i] * down, x[u][i] * down, t[u]);
        }
        group_sum(m, e, t);
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            rstd[u] = in_range(s[u]) ? rstd[u] : down * reciprocal_root(fmaf(t[u], a.inv_features, a.eps * down * down));
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[u][i] *= rstd[u];
}

__device__ __forceinline__ void affine(const Vector& weight, const Vector& bias, int64_t column, int count, float (&x)[kRows][8])
{
    float w[8], b[8];
    load_vector_of(weight, column, count, 1.0f, w);
    load_vector_of(bias, column, count, 0.0f, b);
#pragma unroll
    for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            x[u][i] = fmaf(x[u][i], w[i], b[i]);
}

__device__ __forceinline__ int64_t gate_row(const NormArgs& a, int64_t row)
{
    uint64_t q;
    uint32_t at;
    divide_row(a.rows_per_gate, (uint64_t)row, q, at);
    return (int64_t)q;
}

__device__ __forceinline__ void mask_words(const NormArgs& a, const int64_t (&row)[kRows], int vector, uint32_t (&word)[kRows][4])
{
    uint64_t number[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
        number[u] = (uint64_t)row[u] * (uint32_t)((a.features + 7) / 8) + (uint32_t)vector;
    random_words(a.drop, __ldg(reinterpret_cast<const unsigned long long*>(a.drop.seed)), number, word);
}

template <typename T, typename R, bool VEC>
__global__ void __launch_bounds__(kMaxThreads, 2)
residual_norm_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ Exchange exchange;
    Member m(a.deal);
    blocks_present(a.deal);
    const int64_t column = (int64_t)m.vector * 8;
    const int count = (int)max((int64_t)0, min((int64_t)8, a.features - column));
    for (uint32_t round = 0; round < a.deal.rounds; ++round) {
        int64_t row[kRows];
        int in[kRows];                           // elements of the vector, 0 beyond the last row
        float n[kRows][8], h[kRows][8], mean[kRows], rstd[kRows];
        Raw<T> rx[kRows];
        Raw<R> rr[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            row[u] = ((int64_t)round * a.deal.groups + m.group) * kRows + u;
            in[u] = row[u] < a.rows ? count : 0;
            rx[u] = load_vector<VEC>(static_cast<const T*>(a.x) + row[u] * a.x_stride + column, a.x ? in[u] : 0);
            rr[u] = load_vector<VEC>(static_cast<const R*>(a.residual) + row[u] * a.residual_stride + column,
                                     a.residual ? in[u] : 0);
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            values_of(decode(rx[u]), n[u]);
        if (a.post != ADASUM_NORM_NONE) {
            normalise(m, exchange, a, a.post, count, n, mean, rstd);
            if (a.stats && m.leads()) {
#pragma unroll
                for (int u = 0; u < kRows; ++u)
                    if (row[u] < a.rows) {
                        a.stats[row[u]] = mean[u];
                        a.stats[a.rows + row[u]] = rstd[u];
                    }
            }
            affine(a.post_weight, a.post_bias, column, count, n);
        }
        if (a.drop.seed && a.x) {
            uint32_t word[kRows][4];
            mask_words(a, row, m.vector, word);
#pragma unroll
            for (int u = 0; u < kRows; ++u)
                drop(a.drop, word[u], n[u]);
        }
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            float r[8];
            values_of(decode(rr[u]), r);
            if (a.gate.p) {
                float g[8];
                load_vector_of(a.gate, gate_row(a, row[u]) * a.gate_stride + column, in[u], 1.0f, g);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    n[u][i] *= g[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[u][i] = a.x ? a.branch_scale * n[u][i] : 0.0f;
                if (a.residual)
                    h[u][i] = fmaf(a.residual_scale, r[i], h[u][i]);
                if (i >= count)
                    h[u][i] = 0.0f;
            }
            if (a.out_h && in[u] > 0)
                store_values<VEC>(static_cast<R*>(a.out_h) + row[u] * a.h_stride + column, in[u], h[u]);
        }
        if (a.pre != ADASUM_NORM_NONE) {
            normalise(m, exchange, a, a.pre, count, h, mean, rstd);
            affine(a.pre_weight, a.pre_bias, column, count, h);
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                if (in[u] > 0)
                    store_values<VEC>(static_cast<T*>(a.out_y) + row[u] * a.y_stride + column, in[u], h[u]);
                if (a.stats && m.leads() && row[u] < a.rows) {
                    a.stats[2 * a.rows + row[u]] = mean[u];
                    a.stats[3 * a.rows + row[u]] = rstd[u];
                }
            }
        }
    }
}

// Normalised values of a row from its kept statistics; zeros beyond the row.
template <typename T>
__device__ __forceinline__ void kept_normalised(const Raw<T>& raw, float mean, float rstd, int count, float (&u)[8])
{
    values_of(decode(raw), u);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        u[i] = i < count ? (u[i] - mean) * rstd : 0.0f;
}

// v, the gradients of the normalised values u, to the gradients of the norm's input; zeros beyond the row.
__device__ __forceinline__ void norm_back(Member& m, Exchange& e, const NormArgs& a, int kind, int count, const float (&u)[kRows][8],
                                          const float (&rstd)[kRows], float (&v)[kRows][8])
{
    float s[2 * kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        s[r] = s[kRows + r] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[r] = fmaf(u[r][i], v[r][i], s[r]);
            s[kRows + r] += v[r][i];
        }
    }
    group_sum(m, e, s);
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const float slope = s[r] * a.inv_features, shift = kind == ADASUM_NORM_LAYER ? s[kRows + r] * a.inv_features : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[r][i] = i < count ? rstd[r] * (v[r][i] - shift - u[r][i] * slope) : 0.0f;
    }
}

__device__ __forceinline__ void write_sum(void* dst, int dtype, int64_t at, float sum, float scale, bool accumulate)
{
    float y = sum * scale;
    if (accumulate)
        y += load_as_float(dst, dtype, at);
    store_from_float(dst, dtype, at, y);
}

template <typename T, typename R, bool VEC>
__global__ void __launch_bounds__(kMaxThreads, 1)
residual_norm_grad_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ Exchange exchange;
    __shared__ float columns[kMaxThreads * 8];
    start_next_kernel();
    Member m(a.deal);
    blocks_present(a.deal);
    const int64_t column = (int64_t)m.vector * 8;
    const int count = (int)max((int64_t)0, min((int64_t)8, a.features - column));
    const bool post = a.post != ADASUM_NORM_NONE, pre = a.pre != ADASUM_NORM_NONE && a.grad_y;
    float sum[kVectors][8] = {};
    uint32_t step = 0, unit = m.group;
    int64_t first = 0, end = 0;
    for (uint32_t turn = 0; turn < a.deal.rounds * a.deal.steps; ++turn) {
        if (step == 0) {                         // a new unit
            const uint32_t of = unit / a.deal.pieces, piece = unit - of * a.deal.pieces;
            const int64_t span_end = min(a.rows, (int64_t)(of + 1) * a.deal.gate_rows_span);
            first = (int64_t)of * a.deal.gate_rows_span + (int64_t)piece * a.deal.unit_rows;
            end = unit < a.deal.units ? min(span_end, first + a.deal.unit_rows) : first;
        }
        int64_t row[kRows];
        int in[kRows];
        Raw<T> rx[kRows], ry[kRows];
        Raw<R> rh[kRows], rd[kRows];
        float u[kRows][8], d[kRows][8], rstd[kRows], post_mean[kRows], post_rstd[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            row[r] = first + (int64_t)step * kRows + r;
            in[r] = row[r] < end ? count : 0;
            ry[r] = load_vector<VEC>(static_cast<const T*>(a.grad_y) + row[r] * a.grad_y_stride + column, pre ? in[r] : 0);
            rh[r] = load_vector<VEC>(static_cast<const R*>(a.h) + row[r] * a.h_stride + column, pre ? in[r] : 0);
            rd[r] = load_vector<VEC>(static_cast<const R*>(a.grad_h) + row[r] * a.grad_h_stride + column, a.grad_h ? in[r] : 0);
            rx[r] = load_vector<VEC>(static_cast<const T*>(a.x) + row[r] * a.x_stride + column, a.x ? in[r] : 0);
        }
        if (pre) {
            float w[8];
            load_vector_of(a.pre_weight, column, count, 1.0f, w);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const bool valid = row[r] < end;
                const float mean = valid && a.pre == ADASUM_NORM_LAYER ? a.stats[2 * a.rows + row[r]] : 0.0f;
                rstd[r] = valid ? a.stats[3 * a.rows + row[r]] : 0.0f;
                kept_normalised(rh[r], mean, rstd[r], in[r], u[r]);
                float dy[8];
                values_of(decode(ry[r]), dy);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum[2][i] = fmaf(dy[i], u[r][i], sum[2][i]);
                    sum[3][i] += dy[i];
                    d[r][i] = dy[i] * w[i];
                }
            }
            norm_back(m, exchange, a, a.pre, count, u, rstd, d);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            float dh[8], back[8];
            values_of(decode(rd[r]), dh);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[r][i] = pre ? dh[i] + d[r][i] : dh[i];
                back[i] = a.residual_scale * d[r][i];
                d[r][i] *= a.branch_scale;
            }
            if (a.grad_residual && in[r] > 0)
                store_values<VEC>(static_cast<R*>(a.grad_residual) + row[r] * a.grad_residual_stride + column, in[r], back);
        }
        if (a.branch) {
            uint32_t word[kRows][4];
            if (a.drop.seed)
                mask_words(a, row, m.vector, word);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const bool valid = row[r] < end;
                post_mean[r] = valid && a.post == ADASUM_NORM_LAYER ? a.stats[row[r]] : 0.0f;
                post_rstd[r] = post && valid ? a.stats[a.rows + row[r]] : 1.0f;
                kept_normalised(rx[r], post_mean[r], post_rstd[r], in[r], u[r]);
            }
            if (a.gate.p) {                      // (without x its gradient is not wanted)
                float n[kRows][8];
#pragma unroll
                for (int r = 0; r < kRows; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        n[r][i] = u[r][i];
                if (post)
                    affine(a.post_weight, a.post_bias, column, count, n);
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    if (a.drop.seed)
                        drop(a.drop, word[r], n[r]);
                    float g[8];
                    load_vector_of(a.gate, gate_row(a, row[r]) * a.gate_stride + column, in[r], 1.0f, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (in[r] > 0)
                            sum[4][i] = fmaf(d[r][i], n[r][i], sum[4][i]);
                        d[r][i] *= g[i];
                    }
                }
            }
            if (a.drop.seed) {
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    drop(a.drop, word[r], d[r]);
            }
            if (post) {
                float w[8];
                load_vector_of(a.post_weight, column, count, 1.0f, w);
#pragma unroll
                for (int r = 0; r < kRows; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        sum[0][i] = fmaf(d[r][i], u[r][i], sum[0][i]);
                        sum[1][i] += d[r][i];
                        d[r][i] *= w[i];
                    }
                norm_back(m, exchange, a, a.post, count, u, post_rstd, d);
            }
            if (a.grad_x) {
#pragma unroll
                for (int r = 0; r < kRows; ++r)
                    if (in[r] > 0)
                        store_values<VEC>(static_cast<T*>(a.grad_x) + row[r] * a.grad_x_stride + column, in[r], d[r]);
            }
        }
        if (++step == a.deal.steps) {
            step = 0;
            if (a.gate_by_unit && unit < a.deal.units) {
                if (a.gate_parts) {
                    float* dst = a.gate_parts + (int64_t)unit * a.columns + column;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < count)
                            dst[i] = sum[4][i];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < count)
                            write_sum(a.grad_gate, a.grad_gate_dtype, (int64_t)unit * a.features + column + i, sum[4][i],
                                      a.gate_scale, a.accumulate);
                }
            }
            if (a.gate_by_unit) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    sum[4][i] = 0.0f;
            }
            unit += a.deal.groups;
        }
    }
    // the block's sums: its groups' in order
    const int members = a.deal.warps == 1 ? a.deal.lanes : 32 * a.deal.warps, at = threadIdx.x % members;
    const uint32_t part = a.deal.cluster > 1 ? blockIdx.x / a.deal.cluster : blockIdx.x;
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
        if (!a.want[v])
            continue;
        if (a.deal.groups_per_block > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i)
                columns[i * kMaxThreads + threadIdx.x] = sum[v][i];
            __syncthreads();
            if (threadIdx.x < members) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float total = 0.0f;
                    for (int g = 0; g < a.deal.groups_per_block; ++g)
                        total += columns[i * kMaxThreads + g * members + at];
                    sum[v][i] = total;
                }
            }
        }
        if (threadIdx.x < members && count > 0) {
            float4* dst = reinterpret_cast<float4*>(a.parts + ((int64_t)part * kVectors + v) * a.columns + column);
            dst[0] = make_float4(sum[v][0], sum[v][1], sum[v][2], sum[v][3]);
            dst[1] = make_float4(sum[v][4], sum[v][5], sum[v][6], sum[v][7]);
        }
    }
}

// The parts of every sum added in order: grid.y = the vectors that are wanted, then the gate's rows.  32 columns x 8
// shares of the parts per block.
struct JoinArgs {
    const float* parts;
    const float* gate_parts;
    int64_t columns;
    int features;
    uint32_t parts_count, pieces;
    int vectors;
    int which[kVectors];
    void* grad[kVectors];
    int dtype, gate_dtype;
    float scale, gate_scale;
    bool accumulate;
    void* grad_gate;
};
__global__ void __launch_bounds__(256) residual_norm_join_kernel(const __grid_constant__ JoinArgs a)
{
    __shared__ float share[8][32];
    wait_for_previous_kernel();
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t column = (int64_t)blockIdx.x * 32 + lane;
    const bool gate = (int)blockIdx.y >= a.vectors;
    const uint32_t gate_row = blockIdx.y - a.vectors;
    const int v = gate ? 0 : a.which[blockIdx.y];
    const uint32_t n = gate ? a.pieces : a.parts_count;
    const int64_t apart = gate ? a.columns : kVectors * a.columns;
    const float* p = gate ? a.gate_parts + (int64_t)gate_row * a.pieces * a.columns : a.parts + v * a.columns;
    float total = 0.0f;
    if (column < a.features) {
#pragma unroll 8
        for (uint32_t i = slice; i < n; i += 8)
            total += __ldcg(p + i * apart + column);
    }
    share[slice][lane] = total;
    __syncthreads();
    if (slice == 0 && column < a.features) {
        total = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            total += share[i][lane];
        if (gate)
            write_sum(a.grad_gate, a.gate_dtype, (int64_t)gate_row * a.features + column, total, a.gate_scale, a.accumulate);
        else
            write_sum(a.grad[v], v == 4 ? a.gate_dtype : a.dtype, column, total, v == 4 ? a.gate_scale : a.scale, a.accumulate);
    }
}

// ---- host --------------------------------------------------------------------------------------------

// How a launch deals its rows out; `blocks` at most, whole clusters.
void plan_groups(int64_t features, Deal* d)
{
    const int64_t vectors = (features + 7) / 8;
    d->cluster = (int)((vectors + kMaxThreads - 1) / kMaxThreads);
    d->block_vectors = (int)((vectors + d->cluster - 1) / d->cluster);
    d->lanes = 4;
    while (d->lanes < 32 && d->lanes < d->block_vectors)
        d->lanes *= 2;
    d->warps = (d->block_vectors + 31) / 32;
    if (d->warps == 1)
        d->groups_per_block = 256 / d->lanes;
    else
        d->groups_per_block = d->cluster > 1 || kMaxWarps / d->warps < 1 ? 1 : kMaxWarps / d->warps;
}
int threads_of(const Deal& d) { return d.groups_per_block * (d.warps == 1 ? d.lanes : 32 * d.warps); }

// Blocks that run at once where `full` blocks of kMaxThreads threads fit a multiprocessor.
int64_t resident_blocks(const Deal& d, int sms, int full)
{
    const int64_t n = (int64_t)sms * (full * kMaxThreads / threads_of(d));
    return n < kMaxBlocks ? n : kMaxBlocks;
}

// Rows in units of kRows, without a gate's gradient; else units inside gate rows, enough of them for `most` blocks.
void plan_units(int64_t rows, int64_t gate_span, bool by_unit, int64_t most_blocks, Deal* d, unsigned* blocks)
{
    const int64_t most_groups = (most_blocks / d->cluster > 0 ? most_blocks / d->cluster : 1) * d->groups_per_block;
    int64_t gates = 1, pieces;
    if (!by_unit) {
        d->gate_rows_span = rows;
        d->unit_rows = kRows;
        pieces = (rows + kRows - 1) / kRows;
    } else {
        gates = (rows + gate_span - 1) / gate_span;
        const int64_t span = gate_span < rows ? gate_span : rows;
        pieces = (most_groups + gates - 1) / gates;
        const int64_t most_pieces = (span + kRows - 1) / kRows;
        pieces = pieces < most_pieces ? pieces : most_pieces;
        d->gate_rows_span = gate_span;
        d->unit_rows = ((span + pieces - 1) / pieces + kRows - 1) / kRows * kRows;
        pieces = (span + d->unit_rows - 1) / d->unit_rows;
    }
    d->pieces = (uint32_t)pieces;
    d->units = (uint32_t)(gates * pieces);
    d->steps = (uint32_t)(d->unit_rows / kRows);
    int64_t n = ((int64_t)d->units + d->groups_per_block - 1) / d->groups_per_block * d->cluster;
    if (n > most_blocks / d->cluster * d->cluster)
        n = most_blocks / d->cluster * d->cluster;
    *blocks = (unsigned)n;
    d->groups = (uint32_t)(n / d->cluster * d->groups_per_block);
    d->rounds = (d->units + d->groups - 1) / d->groups;
}

template <typename Kernel>
cudaError_t launch_rows(Kernel* kernel, unsigned blocks, const NormArgs& a, cudaStream_t stream)
{
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(blocks);
    config.blockDim = dim3((unsigned)threads_of(a.deal));
    config.stream = stream;
    cudaLaunchAttribute attribute;
    attribute.id = cudaLaunchAttributeClusterDimension;
    attribute.val.clusterDim.x = (unsigned)a.deal.cluster;
    attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
    config.attrs = &attribute;
    config.numAttrs = a.deal.cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&config, kernel, a);
}

// Calls f(value of T, value of R) for the types of a call: R is T or fp32.
template <typename F>
void with_types(const adasum_residual_norm_t& b, F&& f)
{
    with_type(b.dtype, [&](auto t) {
        if (b.stream_dtype == b.dtype)
            f(t, t);
        else
            f(t, float{});
    });
}

Vector vector_of(const void* p, adasum_dtype_t dtype) { return Vector{p, (int)dtype, aligned_to(p, 16)}; }

adasum_status_t check_block(const adasum_residual_norm_t* b)
{
    if (!b)
        return fail(ADASUM_ERR_NULL, "the description is NULL");
    if (!extent_ok(b->rows) || b->features < 0 || b->features > kMaxFeatures)
        return fail(ADASUM_ERR_ARG, "rows = %lld, features = %lld out of range", (long long)b->rows, (long long)b->features);
    if (!operator_dtype(b->dtype) || !operator_dtype(b->stream_dtype) || !operator_dtype(b->param_dtype) || !operator_dtype(b->gate_dtype))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d, %d, %d: fp32, fp16 or bf16", (int)b->dtype, (int)b->stream_dtype,
                    (int)b->param_dtype, (int)b->gate_dtype);
    if (b->stream_dtype != b->dtype && b->stream_dtype != ADASUM_F32)
        return fail(ADASUM_ERR_DTYPE, "the residual stream is of the blocks' type or fp32");
    auto norm_ok = [](int n) { return n >= ADASUM_NORM_NONE && n <= ADASUM_NORM_LAYER; };
    if (!norm_ok(b->post_norm) || !norm_ok(b->pre_norm))
        return fail(ADASUM_ERR_ARG, "unknown norm %d or %d", (int)b->post_norm, (int)b->pre_norm);
    if (!(b->eps >= 0.0f))
        return fail(ADASUM_ERR_ARG, "eps is negative or NaN");
    const int64_t pb = operator_bytes(b->param_dtype);
    if (!aligned_to(b->post_weight, pb) || !aligned_to(b->post_bias, pb) || !aligned_to(b->pre_weight, pb) || !aligned_to(b->pre_bias, pb))
        return fail(ADASUM_ERR_ARG, "a norm's weight or bias is not aligned to its element size");
    if (b->gate) {
        if (!aligned_to(b->gate, operator_bytes(b->gate_dtype)))
            return fail(ADASUM_ERR_ARG, "gate is not aligned to its element size");
        if (b->rows_per_gate < 1)
            return fail(ADASUM_ERR_ARG, "rows_per_gate = %lld", (long long)b->rows_per_gate);
        if (b->rows_per_gate < b->rows && !stride_ok(b->gate_stride, b->features))
            return fail(ADASUM_ERR_ARG, "stride %lld of gate is shorter than a row or out of range", (long long)b->gate_stride);
    }
    return ADASUM_OK;
}

int64_t gate_rows_of(const adasum_residual_norm_t& b)
{
    return b.rows > 0 ? (b.rows + b.rows_per_gate - 1) / b.rows_per_gate : 0;
}

adasum_status_t describe(const adasum_residual_norm_t& b, bool has_x, NormArgs* a)
{
    *a = NormArgs{};
    a->rows = b.rows;
    a->features = (int)b.features;
    a->post = has_x ? b.post_norm : ADASUM_NORM_NONE;
    a->pre = b.pre_norm;
    a->inv_features = 1.0f / (float)b.features;
    a->eps = b.eps;
    a->branch_scale = b.branch_scale;
    a->residual_scale = b.residual_scale;
    a->post_weight = vector_of(b.post_weight, b.param_dtype);
    a->post_bias = vector_of(b.post_bias, b.param_dtype);
    a->pre_weight = vector_of(b.pre_weight, b.param_dtype);
    a->pre_bias = vector_of(b.pre_bias, b.param_dtype);
    a->gate = vector_of(has_x ? b.gate : nullptr, b.gate_dtype);
    if (b.gate) {
        const int64_t span = b.rows_per_gate < b.rows ? b.rows_per_gate : b.rows;
        a->gate_stride = span < b.rows ? b.gate_stride : 0;
        a->gate.aligned = aligned_to(b.gate, 16) && a->gate_stride * operator_bytes(b.gate_dtype) % 16 == 0;
        a->rows_per_gate = row_divider(span);
        if (span == b.rows)
            a->rows_per_gate = RowDivider{0, 2};     // every row's quotient is 0
    }
    a->columns = (b.features + 7) / 8 * 8;
    return plan_dropout(b.dropout, b.seed, b.site, &a->drop);
}

// A buffer that a call reads or writes.
struct Span {
    const void* p;
    size_t bytes;
    int64_t stride;
};
bool any_overlap(const Span* written, int writes, const Span* others, int count)
{
    for (int i = 0; i < writes; ++i) {
        for (int j = 0; j < count; ++j)
            if (spans_overlap(written[i].p, written[i].bytes, others[j].p, others[j].bytes))
                return true;
        for (int j = i + 1; j < writes; ++j)
            if (spans_overlap(written[i].p, written[i].bytes, written[j].p, written[j].bytes))
                return true;
    }
    return false;
}

// Bytes of the sums that a gradient call leaves for the joining kernel.
size_t norm_workspace(const adasum_residual_norm_t& b, bool by_unit)
{
    const int64_t columns = (b.features + 7) / 8 * 8;
    size_t total = (size_t)kMaxBlocks * kVectors * (size_t)columns * 4;
    if (by_unit) {
        // pieces of a gate row: fewer than groups / gates + 1, so fewer than twice the groups in all where cut
        Deal d{};
        plan_groups(b.features, &d);
        total += 2 * (size_t)kMaxBlocks * (size_t)d.groups_per_block * (size_t)columns * 4;
    }
    return (total + 255) / 256 * 256;
}

}  // namespace
}  // namespace adasum

extern "C" {

adasum_status_t adasum_residual_norm(const adasum_residual_norm_t* b, const void* x, int64_t x_stride,
                                     const void* residual, int64_t residual_stride, void* h, int64_t h_stride, void* y,
                                     int64_t y_stride, float* stats, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    adasum_status_t status = check_block(b);
    if (status != ADASUM_OK)
        return status;
    NormArgs a;
    if ((status = describe(*b, x != nullptr, &a)) != ADASUM_OK)
        return status;
    const int64_t rows = b->rows, features = b->features;
    if (rows == 0 || features == 0)
        return ADASUM_OK;
    if (!x && !residual)
        return fail(ADASUM_ERR_NULL, "x and residual are NULL");
    const bool pre = b->pre_norm != ADASUM_NORM_NONE;
    if (!h && !pre)
        return fail(ADASUM_ERR_NULL, "h is NULL, and there is no norm before the next block");
    if (x && (status = check_matrix("x", x, x_stride, features, b->dtype)) != ADASUM_OK)
        return status;
    if (residual && (status = check_matrix("residual", residual, residual_stride, features, b->stream_dtype)) != ADASUM_OK)
        return status;
    if (h && (status = check_matrix("h", h, h_stride, features, b->stream_dtype)) != ADASUM_OK)
        return status;
    if (pre && (status = check_matrix("y", y, y_stride, features, b->dtype)) != ADASUM_OK)
        return status;
    if (!aligned_to(stats, 4))
        return fail(ADASUM_ERR_ARG, "stats is not 4-byte aligned");
    const int64_t tb = operator_bytes(b->dtype), rb = operator_bytes(b->stream_dtype), pb = operator_bytes(b->param_dtype);
    const size_t vector_bytes = (size_t)(features * pb);
    const Span x_span{x, x ? matrix_span(rows, features, x_stride, tb) : 0, x_stride};
    const Span r_span{residual, residual ? matrix_span(rows, features, residual_stride, rb) : 0, residual_stride};
    const Span written[] = {{h, h ? matrix_span(rows, features, h_stride, rb) : 0, h_stride},
                            {pre ? y : nullptr, pre ? matrix_span(rows, features, y_stride, tb) : 0, y_stride},
                            {stats, stats ? (size_t)rows * 16 : 0, 0}};
    const Span vectors[] = {{b->post_weight, vector_bytes, 0}, {b->post_bias, vector_bytes, 0}, {b->pre_weight, vector_bytes, 0},
                            {b->pre_bias, vector_bytes, 0},
                            {b->gate, b->gate ? matrix_span(gate_rows_of(*b), features, a.gate_stride, operator_bytes(b->gate_dtype)) : 0, 0},
                            {a.drop.seed, 8, 0}};
    if (any_overlap(written, 3, vectors, 6))
        return fail(ADASUM_ERR_ARG, "h, y or stats overlap each other, the norms' vectors, the gate or the seed");
    // h may be the residual itself, y may be x itself: a row is read before it is written, by the same threads
    const bool h_in_place = h && h == residual && h_stride == residual_stride;
    const bool y_in_place = pre && y == x && y_stride == x_stride;
    for (int i = 0; i < 3; ++i) {
        if (spans_overlap(written[i].p, written[i].bytes, x_span.p, x_span.bytes) && !(i == 1 && y_in_place))
            return fail(ADASUM_ERR_ARG, "an output overlaps x (y may be x itself)");
        if (spans_overlap(written[i].p, written[i].bytes, r_span.p, r_span.bytes) && !(i == 0 && h_in_place))
            return fail(ADASUM_ERR_ARG, "an output overlaps residual (h may be the residual itself)");
    }
    a.x = x;
    a.x_stride = x_stride;
    a.residual = residual;
    a.residual_stride = residual_stride;
    a.out_h = h;
    a.h_stride = h_stride;
    a.out_y = y;
    a.y_stride = y_stride;
    a.stats = stats;
    const int sms = device_sms();
    if (sms == 0)
        return fail(ADASUM_ERR_CUDA, "no device");
    unsigned blocks;
    plan_groups(features, &a.deal);
    plan_units(rows, rows, false, resident_blocks(a.deal, sms, 2), &a.deal, &blocks);
    const bool vec = features % 8 == 0 && (!x || rows_aligned(x, x_stride, tb)) && (!residual || rows_aligned(residual, residual_stride, rb)) &&
                     (!h || rows_aligned(h, h_stride, rb)) && (!pre || rows_aligned(y, y_stride, tb));
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    cudaError_t err = cudaSuccess;
    with_types(*b, [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        err = launch_rows(vec ? residual_norm_kernel<T, R, true> : residual_norm_kernel<T, R, false>, blocks, a, stream);
    });
    ADASUM_CUDA_CHECK(err);
    profile_mark(stream, ADASUM_KERNEL_RESIDUAL_NORM, 0, 0, false);
    return ADASUM_OK;
}

size_t adasum_residual_norm_grad_workspace_bytes(const adasum_residual_norm_t* b)
{
    using namespace adasum;
    if (!b || !extent_ok(b->rows) || b->features < 0 || b->features > kMaxFeatures)
        return 0;
    return norm_workspace(*b, b->gate != nullptr);
}

adasum_status_t adasum_residual_norm_grad(const adasum_residual_norm_t* b, const adasum_residual_norm_grads_t* g,
                                          void* workspace, size_t workspace_bytes, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    adasum_status_t status = check_block(b);
    if (status != ADASUM_OK)
        return status;
    if (!g)
        return fail(ADASUM_ERR_NULL, "the gradients' description is NULL");
    if (!operator_dtype(g->grad_dtype) || !operator_dtype(g->gate_grad_dtype))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d: fp32, fp16 or bf16", (int)g->grad_dtype, (int)g->gate_grad_dtype);
    const bool branch = g->x != nullptr || g->grad_x != nullptr;
    NormArgs a;
    if ((status = describe(*b, branch, &a)) != ADASUM_OK)
        return status;
    const int64_t rows = b->rows, features = b->features;
    if (features == 0)
        return ADASUM_OK;
    const bool pre = b->pre_norm != ADASUM_NORM_NONE && g->grad_y != nullptr;
    const bool post = branch && b->post_norm != ADASUM_NORM_NONE;
    if ((g->grad_gate && !b->gate) || ((g->grad_post_weight || g->grad_post_bias) && b->post_norm == ADASUM_NORM_NONE) ||
        ((g->grad_pre_weight || g->grad_pre_bias) && b->pre_norm == ADASUM_NORM_NONE))
        return fail(ADASUM_ERR_ARG, "the gradient of a norm or gate that the block does not have");
    if ((g->grad_gate || g->grad_post_weight || g->grad_post_bias) && !branch && rows > 0)
        return fail(ADASUM_ERR_NULL, "x is NULL");
    const int64_t tb = operator_bytes(b->dtype), rb = operator_bytes(b->stream_dtype), pb = operator_bytes(b->param_dtype);
    const int64_t gb = operator_bytes(g->grad_dtype), gate_gb = operator_bytes(g->gate_grad_dtype);
    void* const vector_grads[kVectors] = {g->grad_post_weight, g->grad_post_bias, g->grad_pre_weight, g->grad_pre_bias, g->grad_gate};
    int wanted = 0;
    for (int v = 0; v < kVectors; ++v) {
        if (!aligned_to(vector_grads[v], v == 4 ? gate_gb : gb))
            return fail(ADASUM_ERR_ARG, "a vector's gradient is not aligned to its element size");
        wanted += vector_grads[v] != nullptr;
    }
    if (rows > 0) {
        if (!g->grad_y && !g->grad_h)
            return fail(ADASUM_ERR_NULL, "grad_y and grad_h are NULL");
        if (g->grad_y && b->pre_norm == ADASUM_NORM_NONE)
            return fail(ADASUM_ERR_ARG, "grad_y without a norm before the next block");
        if (branch && !g->x && (post || g->grad_gate))
            return fail(ADASUM_ERR_NULL, "x is NULL");
        if ((pre || post) && !g->stats)
            return fail(ADASUM_ERR_NULL, "stats is NULL");
        if (!aligned_to(g->stats, 4))
            return fail(ADASUM_ERR_ARG, "stats is not 4-byte aligned");
        const struct { const char* name; const void* p; int64_t stride; adasum_dtype_t dtype; bool needed; } matrices[] = {
            {"x", g->x, g->x_stride, b->dtype, post || g->grad_gate != nullptr}, {"h", g->h, g->h_stride, b->stream_dtype, pre},
            {"grad_y", g->grad_y, g->grad_y_stride, b->dtype, pre}, {"grad_h", g->grad_h, g->grad_h_stride, b->stream_dtype, false},
            {"grad_x", g->grad_x, g->grad_x_stride, b->dtype, false},
            {"grad_residual", g->grad_residual, g->grad_residual_stride, b->stream_dtype, false}};
        for (const auto& m : matrices)
            if ((m.p || m.needed) && (status = check_matrix(m.name, m.p, m.stride, features, m.dtype)) != ADASUM_OK)
                return status;
    }
    const int64_t gates = g->grad_gate ? gate_rows_of(*b) : 0;
    const bool by_unit = gates > 1;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    if (rows == 0) {                       // empty sums
        if (!g->accumulate)
            for (int v = 0; v < 4; ++v)
                if (vector_grads[v])
                    ADASUM_CUDA_CHECK(cudaMemsetAsync(vector_grads[v], 0, (size_t)(features * gb), stream));
        return ADASUM_OK;
    }
    const size_t need = norm_workspace(*b, b->gate != nullptr);
    if (wanted > 0) {
        if (!workspace || workspace_bytes < need)
            return fail(ADASUM_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace ? workspace_bytes : (size_t)0, need);
        if (!aligned_to(workspace, 256))
            return fail(ADASUM_ERR_ARG, "workspace is not 256-byte aligned");
    }
    auto span = [&](const void* p, int64_t stride, int64_t bytes) {
        return Span{p, p ? matrix_span(rows, features, stride, bytes) : 0, stride};
    };
    const Span written[] = {span(g->grad_x, g->grad_x_stride, tb), span(g->grad_residual, g->grad_residual_stride, rb),
                            {wanted > 0 ? workspace : nullptr, need, 0},
                            {vector_grads[0], (size_t)(features * gb), 0}, {vector_grads[1], (size_t)(features * gb), 0},
                            {vector_grads[2], (size_t)(features * gb), 0}, {vector_grads[3], (size_t)(features * gb), 0},
                            {vector_grads[4], (size_t)(gates * features * gate_gb), 0}};
    const Span read[] = {span(g->x, g->x_stride, tb), span(g->h, g->h_stride, rb), {g->stats, (size_t)rows * 16, 0},
                         {b->post_weight, (size_t)(features * pb), 0}, {b->post_bias, (size_t)(features * pb), 0},
                         {b->pre_weight, (size_t)(features * pb), 0}, {b->pre_bias, (size_t)(features * pb), 0},
                         {b->gate, b->gate ? matrix_span(gate_rows_of(*b), features, a.gate_stride, operator_bytes(b->gate_dtype)) : 0, 0},
                         {a.drop.seed, 8, 0}};
    if (any_overlap(written, 8, read, 9))
        return fail(ADASUM_ERR_ARG, "the outputs and the workspace overlap each other or an input");
    // grad_x may be grad_y itself, grad_residual may be grad_h itself
    const Span gy = span(g->grad_y, g->grad_y_stride, tb), gh = span(g->grad_h, g->grad_h_stride, rb);
    for (int i = 0; i < 8; ++i) {
        if (spans_overlap(written[i].p, written[i].bytes, gy.p, gy.bytes) &&
            !(i == 0 && g->grad_x == g->grad_y && g->grad_x_stride == g->grad_y_stride))
            return fail(ADASUM_ERR_ARG, "an output overlaps grad_y (grad_x may be grad_y itself)");
        if (spans_overlap(written[i].p, written[i].bytes, gh.p, gh.bytes) &&
            !(i == 1 && g->grad_residual == g->grad_h && g->grad_residual_stride == g->grad_h_stride))
            return fail(ADASUM_ERR_ARG, "an output overlaps grad_h (grad_residual may be grad_h itself)");
    }
    if (!pre)
        a.pre = ADASUM_NORM_NONE;
    a.x = g->x;
    a.x_stride = g->x_stride;
    a.h = g->h;
    a.h_stride = g->h_stride;
    a.grad_y = pre ? g->grad_y : nullptr;
    a.grad_y_stride = g->grad_y_stride;
    a.grad_h = g->grad_h;
    a.grad_h_stride = g->grad_h_stride;
    a.grad_x = g->grad_x;
    a.grad_x_stride = g->grad_x_stride;
    a.grad_residual = g->grad_residual;
    a.grad_residual_stride = g->grad_residual_stride;
    a.stats = const_cast<float*>(g->stats);
    a.branch = branch;
    a.accumulate = g->accumulate != 0;
    a.grad_gate = g->grad_gate;
    a.grad_gate_dtype = (int)g->gate_grad_dtype;
    a.gate_scale = g->gate_scale;
    a.gate_by_unit = by_unit;
    const int sms = device_sms();
    if (sms == 0)
        return fail(ADASUM_ERR_CUDA, "no device");
    unsigned blocks;
    plan_groups(features, &a.deal);
    plan_units(rows, b->gate ? b->rows_per_gate : rows, by_unit, resident_blocks(a.deal, sms, 1), &a.deal, &blocks);
    a.parts = static_cast<float*>(workspace);
    a.gate_parts = by_unit && a.deal.pieces > 1 ? a.parts + (size_t)kMaxBlocks * kVectors * (size_t)a.columns : nullptr;
    JoinArgs j{};
    for (int v = 0; v < kVectors; ++v) {
        // without grad_y the norm before the next block has no part in the gradients: its vectors' are zero
        a.want[v] = vector_grads[v] != nullptr && !(v == 4 && by_unit);
        j.grad[v] = vector_grads[v];
        if (a.want[v])
            j.which[j.vectors++] = v;
    }
    const bool vec = features % 8 == 0 && (!g->x || rows_aligned(g->x, g->x_stride, tb)) && (!pre || rows_aligned(g->h, g->h_stride, rb)) &&
                     (!pre || rows_aligned(g->grad_y, g->grad_y_stride, tb)) && (!g->grad_h || rows_aligned(g->grad_h, g->grad_h_stride, rb)) &&
                     (!g->grad_x || rows_aligned(g->grad_x, g->grad_x_stride, tb)) &&
                     (!g->grad_residual || rows_aligned(g->grad_residual, g->grad_residual_stride, rb));
    profile_mark(stream, -1, 0, 0, true);
    cudaError_t err = cudaSuccess;
    with_types(*b, [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        err = launch_rows(vec ? residual_norm_grad_kernel<T, R, true> : residual_norm_grad_kernel<T, R, false>, blocks, a, stream);
    });
    ADASUM_CUDA_CHECK(err);
    profile_mark(stream, ADASUM_KERNEL_RESIDUAL_NORM_GRAD, 0, 0, false);
    const int64_t joined = j.vectors + (a.gate_parts ? gates : 0);
    if (joined > 0) {
        j.parts = a.parts;
        j.gate_parts = a.gate_parts;
        j.columns = a.columns;
        j.features = a.features;
        j.parts_count = blocks / a.deal.cluster;
        j.pieces = a.deal.pieces;
        j.dtype = (int)g->grad_dtype;
        j.gate_dtype = (int)g->gate_grad_dtype;
        j.scale = g->scale;
        j.gate_scale = g->gate_scale;
        j.accumulate = a.accumulate;
        j.grad_gate = g->grad_gate;
        ADASUM_CUDA_CHECK(launch_after(residual_norm_join_kernel, dim3((unsigned)((features + 31) / 32), (unsigned)joined), 256, 0,
                                       stream, j));
        profile_mark(stream, ADASUM_KERNEL_RESIDUAL_NORM_GRAD, 1, 0, false);
    }
    return ADASUM_OK;
}

}  // extern "C"
