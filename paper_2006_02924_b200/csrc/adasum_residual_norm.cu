// The joint between two residual blocks: its forward pass.
#include "adasum_residual_norm.cuh"

namespace adasum {
namespace {

// WHOLE: 16-byte aligned rows of whole vectors.  FULL: a norm after the block or a gate.
//
// 16384 x 1024 bf16: RMS norm 25 us (5.3 TB/s), layer norm 28 us, with dropout 36 us (the generator 8; 55 % of the issue slots at
// 16 warps per multiprocessor: latency); 4096 x 4096 bf16 with an fp32 stream, two RMS norms and a gate 62 us (3.2 TB/s: a row's
// way through two sums, at half the warps); one row 4.0 us.
template <typename T, typename R, bool WHOLE, bool FULL, int V>
__global__ void __maxnreg__(V == 1 ? 64 : 80)
residual_norm_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int ROWS = WHOLE ? 1 : 2;
    extern __shared__ __align__(16) unsigned char rows_shared[];
    __shared__ Exchange exchange;
    start_next_kernel();
    Member m(a.deal);
    blocks_present(a.deal);
    wait_for_previous_kernel();
    int count[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        count[v] = m.count(v, a.features);
    Staged staged = stage_vectors(a, m, rows_shared, ROWS, V);
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(rows_shared)) + a.rows_at + threadIdx.x * 16;
    const uint32_t apart = blockDim.x * 16, stage_bytes = a.turn_pieces * apart;
    auto first_row = [&](uint32_t round) { return ((int64_t)round * a.deal.groups + m.group) * ROWS; };
    auto bring = [&](uint32_t round, uint32_t stage) {
        if (round < a.deal.rounds) {
            uint32_t slot = mine + stage * stage_bytes;
#pragma unroll
            for (int u = 0; u < ROWS; ++u) {
                const int64_t row = first_row(round) + u;
                const bool valid = row < a.rows;
                if (a.x)
                    fetch_row<T>(slot, apart, a.x, row * a.x_stride + m.column(0), m.members, valid, count);
                if (a.residual)
                    fetch_row<R>(slot, apart, a.residual, row * a.residual_stride + m.column(0), m.members, valid, count);
            }
        }
        close_turn();
    };
    if constexpr (WHOLE) {
        for (int t = 0; t < a.deal.stages; ++t)
            bring(t, t);
    }
    uint64_t seed = 0;
    if (a.drop.seed)
        seed = *a.drop.seed;
    const uint32_t r_piece = a.x ? V * (uint32_t)(sizeof(T) / 2) * apart : 0;      // place of the residual among the thread's pieces of a row
    uint32_t stage = 0;
    for (uint32_t round = 0; round < a.deal.rounds; ++round) {
        int64_t row[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            row[u] = first_row(round) + u;
        Eight h[ROWS][V];                        // the branch, then the residual stream
        float mean[ROWS], rstd[ROWS];
        // rows stay in shared memory until they are used: as registers they would be more than a thread has
        const uint32_t slot = mine + stage * stage_bytes;
        auto row_of = [&](auto t, const void* base, int64_t stride, uint32_t piece, int u, int v) {
            using E = decltype(t);
            if constexpr (WHOLE) {
                return decode(fetched<E>(slot + piece + v * (uint32_t)(sizeof(E) / 2) * apart + u * (stage_bytes / ROWS), apart));
            } else {
                return decode(load_vector<false>(static_cast<const E*>(base) + row[u] * stride + m.column(v), row[u] < a.rows ? count[v] : 0));
            }
        };
        if constexpr (WHOLE)
            wait_for_turn(a.deal.stages);
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v)
                h[u][v] = a.x ? row_of(T{}, a.x, a.x_stride, 0, u, v) : Eight{};
        if constexpr (FULL) {
            if (a.post != ADASUM_NORM_NONE) {
                normalise<WHOLE>(m, exchange, a, a.post, count, h, mean, rstd);
                if (a.stats && m.leads()) {
#pragma unroll
                    for (int u = 0; u < ROWS; ++u)
                        if (row[u] < a.rows) {
                            a.stats[row[u]] = mean[u];
                            a.stats[a.rows + row[u]] = rstd[u];
                        }
                }
                affine(staged.post_weight, staged.post_bias, m, h);
            }
        }
        if constexpr (FULL && !WHOLE) {
            if (a.gate.p) {
                bool valid[ROWS];
#pragma unroll
                for (int u = 0; u < ROWS; ++u)
                    valid[u] = row[u] < a.rows;
                hold_gate<ROWS, V>(a, m, row, valid, staged);
            }
        }
        if (a.drop.seed && a.x)
            drop_vectors(a, m, seed, row, h);
        const Pair branch = both(a.branch_scale), stream = both(a.residual_scale);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const bool valid = row[u] < a.rows;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (a.x) {
                    if constexpr (FULL) {
                        if (a.gate.p && valid && count[v] > 0) {
                            Eight g;
                            if constexpr (WHOLE)
                                g = gate_eight<T>(a, row[u], m.column(v));
                            else
                                g = shared_eight(staged.gate + (u * V + v) * 8);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                h[u][v].p[i] = h[u][v].p[i] * g.p[i];
                        }
                    }
                    if (a.residual) {
                        const Eight r = row_of(R{}, a.residual, a.residual_stride, r_piece, u, v);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            h[u][v].p[i] = fma2(stream, r.p[i], h[u][v].p[i] * branch);
                    } else {
                        scale(h[u][v], a.branch_scale);
                    }
                } else {
                    h[u][v] = row_of(R{}, a.residual, a.residual_stride, 0, u, v);
                    scale(h[u][v], a.residual_scale);
                }
                if (FULL && count[v] <= 0)
                    h[u][v] = Eight{};
                cut_off<WHOLE>(h[u][v], count[v]);
                if (a.out_h && valid && count[v] > 0)
                    store_vector<WHOLE>(static_cast<R*>(a.out_h) + row[u] * a.h_stride + m.column(v), count[v], h[u][v]);
            }
        }
        if constexpr (WHOLE) {
            bring(round + a.deal.stages, stage);
            stage = stage + 1 == (uint32_t)a.deal.stages ? 0 : stage + 1;
        }
        if (a.pre != ADASUM_NORM_NONE) {
            normalise<WHOLE>(m, exchange, a, a.pre, count, h, mean, rstd);
            affine(staged.pre_weight, staged.pre_bias, m, h);
#pragma unroll
            for (int u = 0; u < ROWS; ++u) {
                const bool valid = row[u] < a.rows;
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (valid && count[v] > 0)
                        store_vector<WHOLE>(static_cast<T*>(a.out_y) + row[u] * a.y_stride + m.column(v), count[v], h[u][v]);
                if (a.stats && m.leads() && valid) {
                    a.stats[2 * a.rows + row[u]] = mean[u];
                    a.stats[3 * a.rows + row[u]] = rstd[u];
                }
            }
        }
    }
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
    const bool gate_whole = !a.gate.p || (a.gate.aligned && (b->gate_dtype == b->dtype || b->gate_dtype == ADASUM_F32));
    const bool vec = features % 8 == 0 && gate_whole && (!x || rows_aligned(x, x_stride, tb)) && (!residual || rows_aligned(residual, residual_stride, rb)) &&
                     (!h || rows_aligned(h, h_stride, rb)) && (!pre || rows_aligned(y, y_stride, tb));
    const bool full = a.post != ADASUM_NORM_NONE || a.gate.p;
    if (a.post == ADASUM_NORM_NONE)
        a.post_weight = a.post_bias = Vector{};
    if (!pre)
        a.pre_weight = a.pre_bias = Vector{};
    // several vectors per thread, where that leaves a row four threads or more: what is spent per thread and row falls.  bf16, RMS,
    // with 1, 2, 4: 16384 x 1024 and dropout 45, 40, 36 us; 1024 x 16384 66, 56, 28 us.  Beside a norm after the block
    // two, so that wide rows leave room for a turn ahead: 8192 x 2048 40, 35 us; 4096 x 4096 with a gate 60, 63, 79 us
    const bool four = vec && features > 128;
    unsigned blocks;
    const int per_processor = four ? plan_blocks(&a, vec, full ? 2 : 4, 1, (int)((x ? tb / 2 : 0) + (residual ? rb / 2 : 0)), 768, {512, 256})
                                   : plan_blocks(&a, vec, 1, vec ? 1 : 2, (int)((x ? tb / 2 : 0) + (residual ? rb / 2 : 0)), 1024, {512, 256});
    if (per_processor == 0)
        return fail(ADASUM_ERR_ARG, "%lld features are too many", (long long)features);
    plan_units(rows, rows, false, (int64_t)per_processor * sms, &a.deal, &blocks);
    const size_t shared = a.rows_at + (vec ? (size_t)a.deal.stages * a.turn_pieces * threads_of(a.deal) * 16 : 0);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    cudaError_t err = cudaSuccess;
    with_types(*b, [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        auto* kernel = !vec   ? residual_norm_kernel<T, R, false, true, 1>
                       : four ? full ? residual_norm_kernel<T, R, true, true, 2> : residual_norm_kernel<T, R, true, false, 4>
                              : residual_norm_kernel<T, R, true, true, 1>;
        static std::atomic<uint64_t> prepared[4] = {};         // of these types' kernels
        err = launch_rows(kernel, prepared[!vec ? 0 : !four ? 1 : full ? 2 : 3], blocks, a, shared, stream);
    });
    ADASUM_CUDA_CHECK(err);
    profile_mark(stream, ADASUM_KERNEL_RESIDUAL_NORM, 0, 0, false);
    return ADASUM_OK;
}

}  // extern "C"
