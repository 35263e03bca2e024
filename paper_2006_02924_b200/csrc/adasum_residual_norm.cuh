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
// All rows of x, residual, h and y are read or written once: HBM traffic bounds both directions.  Rows are brought to
// shared memory by asynchronous copies one or two turns ahead of their use, so that loads are on their way while sums are
// exchanged; every thread copies what it reads itself, which takes no barrier.  A group of threads
// owns whole rows, one to four vectors of eight columns per thread (one, and two rows at a time, where rows are short or
// not aligned), so a thread meets the same columns in every row and sums the vectors' gradients in registers.  A group is
// 4 to 32 lanes of a warp, several warps of a block, or a cluster of blocks, which exchange their sums through distributed
// shared memory.
//
// Gradients of vectors are summed per block and then over the blocks by a second kernel, both in a fixed order: the
// results are the same from run to run.  With a gate for every so many rows, the rows of one gate row are cut into
// pieces that a group walks one after another, and each piece leaves its own sum.
#pragma once

#include <atomic>

#include "adasum_random.cuh"
#include "adasum_vectors.cuh"

namespace adasum {
namespace {

constexpr int kMaxWarps = 16;
constexpr int kMaxCluster = 8;
constexpr int64_t kMaxFeatures = ADASUM_NORM_MAX_FEATURES;
constexpr int kMaxProcessors = 148;        // multiprocessors that a gradient call uses
constexpr int kGradThreads = 512;          // of a multiprocessor, at least, in gradient calls
constexpr int kMaxParts = 2 * kMaxProcessors;     // blocks that leave sums of the vectors' gradients
constexpr int kVectors = 5;                // gradients of vectors: post weight, post bias, pre weight, pre bias, gate

// A vector of parameters, or the gate (p = nullptr: there is none).
struct Vector {
    const void* p;
    int dtype;
    bool aligned;              // every row starts on 16 bytes
};

// How rows are dealt out.  Rows come in units of `unit_rows` (the last unit of a gate row may be shorter); unit k of a
// group is unit number group + k * groups.
struct Deal {
    int per_thread;            // vectors of a thread
    int rows_at_once;
    int lanes;                 // lanes of a group inside a warp
    int warps;                 // warps of a group inside a block
    int groups_per_block;
    int cluster;               // blocks of a group
    int block_vectors;         // vectors of eight columns per block
    uint32_t groups;           // of the whole launch
    uint32_t units, steps, rounds;     // a unit takes `steps` times rows_at_once rows; a group `rounds` units
    uint32_t pieces;           // units per gate row
    int stages;                // turns whose rows are in shared memory or on their way
    int64_t gate_rows_span;    // rows of a gate row (all rows, without a gate's gradient)
    int64_t unit_rows;
};

struct NormArgs {
    Deal deal;
    int64_t rows;
    int features, post, pre;
    float inv_features, eps, branch_scale, residual_scale;
    float least_squares;       // a row whose sum of squares is smaller is scaled up first; 0: eps makes that needless
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
    uint32_t turn_pieces;      // of 16 bytes that a thread brings per turn
    uint32_t rows_at;          // of shared memory, in bytes: the rows follow the vectors
    bool branch;               // there is a branch whose gradient is wanted
    bool want_gate;
};

// The loops below handle packed pairs of fp32 values (two per instruction): with one instruction per value both kernels
// were bound by instruction issue (forward 42 to 66, backward 75 instructions an element).

// Weights, biases and the gate's rows, of any type and alignment, are brought to shared memory as fp32 once: reading
// them where they are used made the code larger than the instruction caches (one row of 1024: 7.2 us).
__device__ __forceinline__ Eight shared_eight(const float* p)
{
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    Eight x;
    x.p[0] = pair_of(a.x, a.y);
    x.p[1] = pair_of(a.z, a.w);
    x.p[2] = pair_of(b.x, b.y);
    x.p[3] = pair_of(b.z, b.w);
    return x;
}
__device__ __forceinline__ float sum_of(const Eight& x)
{
    const float2 f = values_of((x.p[0] + x.p[1]) + (x.p[2] + x.p[3]));
    return f.x + f.y;
}
__device__ __forceinline__ float dot_of(const Eight& x, const Eight& y)
{
    const float2 f = values_of(fma2(x.p[0], y.p[0], x.p[1] * y.p[1]) + fma2(x.p[2], y.p[2], x.p[3] * y.p[3]));
    return f.x + f.y;
}
__device__ __forceinline__ void scale(Eight& x, float by)
{
    const Pair b = both(by);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x.p[i] = x.p[i] * b;
}
// Zeros beyond the row.  WHOLE: vectors are whole or nothing, and those that are nothing stay out of the sums instead.
template <bool WHOLE>
__device__ __forceinline__ void cut_off(Eight& x, int count)
{
    if constexpr (!WHOLE) {
        float y[8];
        values_of(x, y);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            y[i] = i < count ? y[i] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            x.p[i] = pair_of(y[2 * i], y[2 * i + 1]);
    }
}
__device__ __forceinline__ void drop(const Dropout& d, const uint32_t (&word)[4], Eight& x)
{
    float y[8];
    values_of(x, y);
    drop(d, word, y);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x.p[i] = pair_of(y[2 * i], y[2 * i + 1]);
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
    int vector, members;       // the thread's first vector of the row; the next ones are `members` further
    int end;                   // vectors of the row up to the block's last
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
        members = d.warps == 1 ? d.lanes : 32 * d.warps;
        end = (rank + 1) * d.block_vectors;
        vector += rank * d.block_vectors;
        group = block * d.groups_per_block + slot;
    }
    __device__ __forceinline__ int vector_number(int v) const { return vector + v * members; }
    __device__ __forceinline__ int64_t column(int v) const { return (int64_t)vector_number(v) * 8; }
    // Place among the block's columns; that of the last vector for threads that have none.
    __device__ __forceinline__ int local_column(int v) const
    {
        return min(vector_number(v) - (int)rank * deal.block_vectors, deal.block_vectors - 1) * 8;
    }
    // Elements of the thread's v-th vector.
    __device__ __forceinline__ int count(int v, int features) const
    {
        return vector_number(v) < end ? max(0, min(8, features - 8 * vector_number(v))) : 0;
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
    float warp_sum[2][kMaxWarps / 2][4][kMaxWarps];      // [turn][group][value][warp]
    float block_sum[2][kMaxCluster][4];
};

// Sums over the group of N (1, 2 or 4) values per thread, in a fixed order; every thread gets them.  All threads of the
// block call it equally often.  Two buffers in turn: a thread that is two calls ahead has passed a barrier that
// the others reach only after reading.
//
// Inside a warp of several the values part ways: halves of the lanes exchange what the other half goes on with, so that N
// values take 6 shuffles for N = 2 or 4 instead of 5 N.
template <int N>
__device__ __forceinline__ void group_sum(Member& m, Exchange& e, float (&v)[N])
{
    const Deal& d = m.deal;
    if (d.warps == 1) {
#pragma unroll
        for (int step = 16; step > 0; step >>= 1) {
            if (step < d.lanes) {
#pragma unroll
                for (int n = 0; n < N; ++n)
                    v[n] += __shfl_xor_sync(0xffffffffu, v[n], step);
            }
        }
        return;
    }
    constexpr int kLanes = 32 / N;               // that end up with the same value
    const int lane = threadIdx.x & 31;
    float mine;
    if constexpr (N == 4) {
        const bool upper = lane & 16, odd = lane & 8;
        float a = upper ? v[2] : v[0], b = upper ? v[3] : v[1];
        a += __shfl_xor_sync(0xffffffffu, upper ? v[0] : v[2], 16);
        b += __shfl_xor_sync(0xffffffffu, upper ? v[1] : v[3], 16);
        mine = odd ? b : a;
        mine += __shfl_xor_sync(0xffffffffu, odd ? a : b, 8);
    } else if constexpr (N == 2) {
        const bool upper = lane & 16;
        mine = upper ? v[1] : v[0];
        mine += __shfl_xor_sync(0xffffffffu, upper ? v[0] : v[1], 16);
    } else {
        mine = v[0];
    }
#pragma unroll
    for (int step = kLanes / 2; step > 0; step >>= 1)
        mine += __shfl_xor_sync(0xffffffffu, mine, step);
    if (lane % kLanes == 0)
        e.warp_sum[m.parity][m.slot][lane / kLanes][m.warp_in_group] = mine;
    asm volatile("bar.sync %0, %1;" ::"r"(m.slot + 1), "r"(32 * d.warps) : "memory");
    const int from = lane % kLanes;
    const float* row = e.warp_sum[m.parity][m.slot][lane / kLanes];
    mine = from < d.warps ? row[from] : 0.0f;
    if (kLanes < kMaxWarps && from + kLanes < d.warps)
        mine += row[from + kLanes];
#pragma unroll
    for (int step = kLanes / 2; step > 0; step >>= 1)
        mine += __shfl_xor_sync(0xffffffffu, mine, step);
#pragma unroll
    for (int n = 0; n < N; ++n)
        v[n] = N == 1 ? mine : __shfl_sync(0xffffffffu, mine, n * kLanes);
    if (d.cluster > 1) {
        if (threadIdx.x < (unsigned)d.cluster) {
            const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(&e.block_sum[m.parity][m.rank][0]));
            uint32_t remote;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(mine), "r"(threadIdx.x));
#pragma unroll
            for (int n = 0; n < N; ++n)
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote + 4 * n), "f"(v[n]) : "memory");
        }
        __syncwarp();
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

// ---- rows on their way -------------------------------------------------------------------------------
//
// Shared memory holds [stage][vector of the turn][thread] pieces of 16 bytes.

// A row's vectors to this thread's pieces, `apart` bytes between pieces; zeros without an access where there is nothing.
template <typename T, int V>
__device__ __forceinline__ void fetch_row(uint32_t& slot, uint32_t apart, const void* base, int64_t at, int members, bool valid,
                                          const int (&count)[V])
{
    const char* p = reinterpret_cast<const char*>(static_cast<const T*>(base) + at);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int bytes = valid && count[v] > 0 ? 16 : 0;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slot), "l"(p + 16 * i), "r"(bytes) : "memory");
            slot += apart;
        }
        p += members * (int)(8 * sizeof(T));
    }
}
template <typename T>
__device__ __forceinline__ Raw<T> fetched(uint32_t slot, uint32_t apart)
{
    Raw<T> raw;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i)
        raw.w[i] = load_shared_16B(slot + i * apart);
    return raw;
}
__device__ __forceinline__ void close_turn() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until the oldest of the turns that are on their way has arrived.
__device__ __forceinline__ void wait_for_turn(int stages)
{
    if (stages >= 3)
        asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (stages == 2)
        asm volatile("cp.async.wait_group 1;" ::: "memory");
    else
        asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// ---- norms ---------------------------------------------------------------------------------------------

__device__ __forceinline__ bool in_range(float s) { return fabsf(s) < __uint_as_float(0x7f800000u); }
// Does something hold for a thread of the group (of the warp's groups)?  `some` is the same for all threads of a group; so is the answer.
__device__ __forceinline__ bool any_of(const Member& m, bool some) { return m.deal.warps == 1 ? __any_sync(0xffffffffu, some) : some; }

// Powers of two that bring a row's squares back into fp32's range, and the least sum of squares that is taken as it is: of
// 2^-100, squares below fp32's normal values (2^-150 off each, 2^15 at most) take 2^-35 away.  Smaller sums make no difference
// beside an eps of 2^-66 or more.
constexpr float kRowDown = 0x1p-96f, kRowUp = 0x1p96f, kLeastSquares = 0x1p-100f, kEpsAbove = 0x1p-66f;

// Statistics of ROWS rows; x becomes the normalised values.  count: the elements of the thread's vectors.
template <bool WHOLE, int ROWS, int V>
__device__ __forceinline__ void normalise(Member& m, Exchange& e, const NormArgs& a, int kind, const int (&count)[V],
                                          Eight (&x)[ROWS][V], float (&mean)[ROWS], float (&rstd)[ROWS])
{
    float s[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u)
        mean[u] = 0.0f;
    if (kind == ADASUM_NORM_LAYER) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            s[u] = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v)
                s[u] += sum_of(x[u][v]);
        }
        group_sum(m, e, s);
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            mean[u] = s[u] * a.inv_features;
        bool outside = false;
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            outside |= !in_range(s[u]);
        if (any_of(m, outside)) {                // such rows are divided before they are added
            float t[ROWS];
#pragma unroll
            for (int u = 0; u < ROWS; ++u) {
                t[u] = 0.0f;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    Eight y = x[u][v];
                    scale(y, a.inv_features);
                    t[u] += sum_of(y);
                }
            }
            group_sum(m, e, t);
#pragma unroll
            for (int u = 0; u < ROWS; ++u)
                mean[u] = in_range(s[u]) ? mean[u] : t[u];
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const Pair off = both(-mean[u]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[u][v].p[i] = x[u][v].p[i] + off;
                cut_off<WHOLE>(x[u][v], count[v]);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        s[u] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
            s[u] += count[v] > 0 ? dot_of(x[u][v], x[u][v]) : 0.0f;
    }
    group_sum(m, e, s);
    float factor[ROWS];                          // of the values
    bool outside = false;
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        factor[u] = rstd[u] = reciprocal_root(fmaf(s[u], a.inv_features, a.eps));
        outside |= !(s[u] >= a.least_squares && in_range(s[u]));
    }
    if (any_of(m, outside)) {                    // such rows: of the values times 2^-96 or 2^96
        float t[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const float by = s[u] < a.least_squares ? kRowUp : kRowDown;
            t[u] = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Eight y = x[u][v];
                scale(y, by);
                t[u] += count[v] > 0 ? dot_of(y, y) : 0.0f;
            }
        }
        group_sum(m, e, t);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            if (s[u] < a.least_squares) {        // rstd may leave fp32's range, the normalised values do not
                factor[u] = reciprocal_root(fmaf(t[u], a.inv_features, a.eps * kRowUp * kRowUp));
                rstd[u] = kRowUp * factor[u];
#pragma unroll
                for (int v = 0; v < V; ++v)
                    scale(x[u][v], kRowUp);
            } else if (!in_range(s[u])) {
                factor[u] = rstd[u] = kRowDown * reciprocal_root(fmaf(t[u], a.inv_features, a.eps * kRowDown * kRowDown));
            }
        }
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u)
#pragma unroll
        for (int v = 0; v < V; ++v)
            scale(x[u][v], factor[u]);
}

// The norms' vectors of the block's columns, and every thread's columns of the gate's rows, in shared memory.
struct Staged {
    const float *post_weight, *post_bias, *pre_weight, *pre_bias;      // nullptr: there is none
    float* gate;                       // the thread's own
    int64_t gate_loaded[2];            // the gate's rows that it holds
};
template <typename T>
__device__ __forceinline__ Eight eight_of(const void* p, int64_t at, bool aligned, int count)
{
    const T* q = static_cast<const T*>(p) + at;
    return decode(aligned && count == 8 ? load_vector<true>(q, count) : load_vector<false>(q, count));
}
__device__ __forceinline__ void keep_eight(float* dst, const Eight& x)
{
    const float2 a = values_of(x.p[0]), b = values_of(x.p[1]), c = values_of(x.p[2]), d = values_of(x.p[3]);
    reinterpret_cast<float4*>(dst)[0] = make_float4(a.x, a.y, b.x, b.y);
    reinterpret_cast<float4*>(dst)[1] = make_float4(c.x, c.y, d.x, d.y);
}
// All four are on their way before the first is kept.
template <typename T>
__device__ __forceinline__ void stage_of(const NormArgs& a, int64_t first, float* const (&to)[4])
{
    const Vector* const from[4] = {&a.post_weight, &a.post_bias, &a.pre_weight, &a.pre_bias};
    for (int at = 8 * threadIdx.x; at < a.deal.block_vectors * 8; at += 8 * blockDim.x) {
        const int count = (int)max((int64_t)0, min((int64_t)8, a.features - first - at));
        Eight x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (to[k])
                x[k] = eight_of<T>(from[k]->p, first + at, from[k]->aligned, count);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (to[k])
                keep_eight(to[k] + at, x[k]);
    }
}
__device__ __forceinline__ Staged stage_vectors(const NormArgs& a, const Member& m, unsigned char* shared, int rows, int per_thread)
{
    float* next = reinterpret_cast<float*>(shared);
    const int columns = a.deal.block_vectors * 8;
    auto place = [&](const Vector& v) -> float* {
        float* const dst = v.p ? next : nullptr;
        next += v.p ? columns : 0;
        return dst;
    };
    float* const to[4] = {place(a.post_weight), place(a.post_bias), place(a.pre_weight), place(a.pre_bias)};
    const int64_t first = (int64_t)m.rank * columns;
    const int dtype = a.post_weight.p ? a.post_weight.dtype : a.post_bias.p ? a.post_bias.dtype : a.pre_weight.p ? a.pre_weight.dtype : a.pre_bias.dtype;
    if (dtype == ADASUM_F32)
        stage_of<float>(a, first, to);
    else if (dtype == ADASUM_F16)
        stage_of<__half>(a, first, to);
    else
        stage_of<__nv_bfloat16>(a, first, to);
    __syncthreads();
    Staged s{to[0], to[1], to[2], to[3], next + (int64_t)threadIdx.x * rows * per_thread * 8, {-1, -1}};
    return s;
}
// vectors staged by the host's reckoning: bytes
inline size_t staged_bytes(const NormArgs& a, bool whole, int threads)
{
    const int vectors = (a.post_weight.p != nullptr) + (a.post_bias.p != nullptr) + (a.pre_weight.p != nullptr) + (a.pre_bias.p != nullptr);
    const size_t gate = a.gate.p && !whole ? (size_t)threads * a.deal.rows_at_once * a.deal.per_thread * 32 : 0;
    return (size_t)vectors * a.deal.block_vectors * 32 + gate;
}

template <int ROWS, int V>
__device__ __forceinline__ void affine(const float* weight, const float* bias, const Member& m, Eight (&x)[ROWS][V])
{
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = m.local_column(v);
        if (weight) {
            const Eight w = shared_eight(weight + at);
#pragma unroll
            for (int u = 0; u < ROWS; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[u][v].p[i] = x[u][v].p[i] * w.p[i];
        }
        if (bias) {
            const Eight b = shared_eight(bias + at);
#pragma unroll
            for (int u = 0; u < ROWS; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[u][v].p[i] = x[u][v].p[i] + b.p[i];
        }
    }
}

__device__ __forceinline__ int64_t gate_row(const NormArgs& a, int64_t row)
{
    uint64_t q;
    uint32_t at;
    divide_row(a.rows_per_gate, (uint64_t)row, q, at);
    return (int64_t)q;
}

// The gate's rows of the rows at hand, if the thread does not hold them yet.
template <typename T, int V>
__device__ __noinline__ void stage_gate(const NormArgs& a, int64_t row, int vector, int members, int end, float* dst)
{
    Eight x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int number = vector + v * members;
        const int count = number < end ? max(0, min(8, a.features - 8 * number)) : 0;
        x[v] = eight_of<T>(a.gate.p, row * a.gate_stride + (int64_t)number * 8, a.gate.aligned, count);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
        keep_eight(dst + 8 * v, x[v]);
}
// Whole vectors of the gate come straight from its rows, of the blocks' type or fp32.
template <typename T>
__device__ __forceinline__ Eight gate_eight(const NormArgs& a, int64_t row, int64_t column)
{
    const int64_t at = gate_row(a, row) * a.gate_stride + column;
    if (a.gate.dtype == TypeCode<T>::value)
        return decode(load_vector<true>(static_cast<const T*>(a.gate.p) + at, 8));
    return decode(load_vector<true>(static_cast<const float*>(a.gate.p) + at, 8));
}
template <int ROWS, int V>
__device__ __forceinline__ void hold_gate(const NormArgs& a, const Member& m, const int64_t (&row)[ROWS], const bool (&valid)[ROWS], Staged& s)
{
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const int64_t q = gate_row(a, row[u]);
        if (valid[u] && q != s.gate_loaded[u]) {
            float* const dst = s.gate + u * V * 8;
            if (a.gate.dtype == ADASUM_F32)
                stage_gate<float, V>(a, q, m.vector, m.members, m.end, dst);
            else if (a.gate.dtype == ADASUM_F16)
                stage_gate<__half, V>(a, q, m.vector, m.members, m.end, dst);
            else
                stage_gate<__nv_bfloat16, V>(a, q, m.vector, m.members, m.end, dst);
            s.gate_loaded[u] = q;
        }
    }
}

// The masks of two vectors at a time, which share the generator's round keys.
template <int ROWS, int V>
__device__ __forceinline__ void drop_vectors(const NormArgs& a, const Member& m, uint64_t seed, const int64_t (&row)[ROWS], Eight (&x)[ROWS][V])
{
#pragma unroll
    for (int j = 0; j < ROWS * V; j += 2) {
        constexpr int kPair = ROWS * V > 1 ? 2 : 1;
        uint64_t number[kPair];
        uint32_t word[kPair][4];
#pragma unroll
        for (int i = 0; i < kPair; ++i)
            number[i] = (uint64_t)row[(j + i) / V] * (uint32_t)(a.columns / 8) + (uint32_t)m.vector_number((j + i) % V);
        random_words(a.drop, seed, number, word);
#pragma unroll
        for (int i = 0; i < kPair; ++i)
            drop(a.drop, word[i], x[(j + i) / V][(j + i) % V]);
    }
}

// ---- host --------------------------------------------------------------------------------------------

// How a launch deals its rows out: `per_thread` vectors per thread, blocks of at most `most_threads`.
inline void plan_groups(int64_t features, int per_thread, int rows_at_once, int most_threads, Deal* d)
{
    const int64_t vectors = (features + 7) / 8;
    d->per_thread = per_thread;
    d->rows_at_once = rows_at_once;
    d->cluster = (int)((vectors + (int64_t)per_thread * most_threads - 1) / ((int64_t)per_thread * most_threads));
    d->block_vectors = (int)((vectors + d->cluster - 1) / d->cluster);
    const int threads = (d->block_vectors + per_thread - 1) / per_thread;
    d->lanes = 4;
    while (d->lanes < 32 && d->lanes < threads)
        d->lanes *= 2;
    d->warps = (threads + 31) / 32;
    if (d->warps == 1 && d->cluster > 1)
        d->warps = 2;                          // a cluster's blocks exchange sums as several warps do
    if (d->warps == 1)
        d->groups_per_block = 256 / d->lanes;
    else
        d->groups_per_block = d->cluster > 1 || most_threads / 32 / d->warps < 1 ? 1 : most_threads / 32 / d->warps;
}
inline int threads_of(const Deal& d) { return d.groups_per_block * (d.warps == 1 ? d.lanes : 32 * d.warps); }

constexpr size_t kSharedPerProcessor = 228 * 1024, kSharedPerBlock = 227 * 1024;
constexpr size_t kSharedBeside = sizeof(Exchange) + 1024;        // of a block, beside what the launch asks for

// Blocks of `threads` at most, turns on their way (two or three) and blocks per multiprocessor, of two sizes of blocks the one
// with which more warps are resident: large blocks share the vectors, small ones fill a multiprocessor better.
// `threads_resident`: as many as their registers allow.  Returns blocks per multiprocessor.
inline int plan_blocks(NormArgs* a, bool whole, int per_thread, int rows_at_once, int pieces_per_vector, int threads_resident, const int (&threads)[2])
{
    Deal best{};
    int best_threads = 0, best_blocks = 0;
    for (int most_threads : threads) {
        Deal d{};
        plan_groups(a->features, per_thread, rows_at_once, most_threads, &d);
        if (d.cluster > kMaxCluster)
            continue;
        a->deal = d;
        a->turn_pieces = (uint32_t)(d.rows_at_once * per_thread * pieces_per_vector);
        const size_t fixed = staged_bytes(*a, whole, threads_of(d));
        const size_t turn = whole ? (size_t)a->turn_pieces * threads_of(d) * 16 : 0;
        if (fixed + turn > kSharedPerBlock - sizeof(Exchange))
            continue;
        int blocks = threads_resident / threads_of(d) > 0 ? threads_resident / threads_of(d) : 1;
        while (blocks > 1 && (fixed + 2 * turn + kSharedBeside) * blocks > kSharedPerProcessor)
            --blocks;
        size_t room = kSharedPerProcessor / blocks - kSharedBeside;
        room = room < kSharedPerBlock - sizeof(Exchange) ? room : kSharedPerBlock - sizeof(Exchange);
        const size_t stages = turn > 0 ? (room - fixed) / turn : 1;
        d.stages = stages < 1 ? 1 : stages > 3 ? 3 : (int)stages;
        // without a second turn on its way a block is worth half
        const int worth = blocks * threads_of(d) * (turn > 0 && d.stages == 1 ? 1 : 2);
        if (worth > best_threads || (worth == best_threads && d.stages > best.stages)) {
            best_threads = worth;
            best_blocks = blocks;
            best = d;
        }
    }
    a->deal = best;
    a->turn_pieces = (uint32_t)(best.rows_at_once * per_thread * pieces_per_vector);
    a->rows_at = best_blocks > 0 ? (uint32_t)staged_bytes(*a, whole, threads_of(best)) : 0;
    return best_blocks;
}

// Rows in units of what a group takes at once, without a gate's gradient; else units inside gate rows, cut so that the groups' turns end together.
inline void plan_units(int64_t rows, int64_t gate_span, bool by_unit, int64_t most_blocks, Deal* d, unsigned* blocks)
{
    const int64_t kRows = d->rows_at_once;
    const int64_t most_groups = (most_blocks / d->cluster > 0 ? most_blocks / d->cluster : 1) * d->groups_per_block;
    int64_t gates = 1, pieces;
    if (!by_unit) {
        d->gate_rows_span = rows;
        d->unit_rows = kRows;
        pieces = (rows + kRows - 1) / kRows;
    } else {
        gates = (rows + gate_span - 1) / gate_span;
        const int64_t span = gate_span < rows ? gate_span : rows;
        int64_t best = INT64_MAX;
        pieces = 1;
        // turns of the longest group, and one more per unit for leaving its sum; at most twice as many units as groups
        auto consider = [&](int64_t p) {
            if (p < 1 || (p > 1 && p * gates > 2 * most_groups))
                return;
            const int64_t unit_rows = ((span + p - 1) / p + kRows - 1) / kRows * kRows;
            const int64_t real = (span + unit_rows - 1) / unit_rows;
            const int64_t cost = (gates * real + most_groups - 1) / most_groups * (unit_rows / kRows + 1);
            if (cost < best) {
                best = cost;
                pieces = real;
                d->unit_rows = unit_rows;
            }
        };
        for (int64_t p = 1; p <= 8; ++p)
            consider(p);
        consider(most_groups / gates);
        consider(2 * most_groups / gates);
        d->gate_rows_span = gate_span;
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

// `prepared`: the kernel's own, a bit per device whose limit of shared memory has been raised.
template <typename Kernel>
cudaError_t launch_rows(Kernel* kernel, std::atomic<uint64_t>& prepared, unsigned blocks, const NormArgs& a, size_t shared_bytes,
                        cudaStream_t stream)
{
    if (shared_bytes > 40 * 1024) {
        int device = 0;
        cudaError_t err = cudaGetDevice(&device);
        if (err != cudaSuccess)
            return err;
        const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
        if (!(prepared.load(std::memory_order_relaxed) & bit) || bit == 0) {
            err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kSharedPerBlock - sizeof(Exchange)));
            if (err != cudaSuccess)
                return err;
            prepared.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    cudaLaunchConfig_t config = {};
    config.dynamicSmemBytes = shared_bytes;
    config.gridDim = dim3(blocks);
    config.blockDim = dim3((unsigned)threads_of(a.deal));
    config.stream = stream;
    cudaLaunchAttribute attributes[2];
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // as launch_after does
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = (unsigned)a.deal.cluster;
    attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    config.attrs = attributes;
    config.numAttrs = a.deal.cluster > 1 ? 2 : 1;
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

inline Vector vector_of(const void* p, adasum_dtype_t dtype) { return Vector{p, (int)dtype, aligned_to(p, 16)}; }

inline adasum_status_t check_block(const adasum_residual_norm_t* b)
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

// rows_per_gate may be anything up to the type's end.
inline int64_t gate_rows_of(const adasum_residual_norm_t& b) { return b.rows > 0 ? (b.rows - 1) / b.rows_per_gate + 1 : 0; }

inline adasum_status_t describe(const adasum_residual_norm_t& b, bool has_x, NormArgs* a)
{
    *a = NormArgs{};
    a->rows = b.rows;
    a->features = (int)b.features;
    a->post = has_x ? b.post_norm : ADASUM_NORM_NONE;
    a->pre = b.pre_norm;
    a->inv_features = 1.0f / (float)b.features;
    a->eps = b.eps;
    a->least_squares = b.eps < kEpsAbove ? kLeastSquares : 0.0f;
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
inline bool any_overlap(const Span* written, int writes, const Span* others, int count)
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

}  // namespace
}  // namespace adasum
