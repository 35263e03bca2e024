// The joint between two residual blocks: its gradients.
#include "adasum_residual_norm.cuh"

namespace adasum {
namespace {

// Normalised values of a row from its kept statistics.  Vectors beyond the row meet gradients of zero only.
template <bool WHOLE>
__device__ __forceinline__ Eight kept_normalised(const Eight& x, float mean, float rstd, int count)
{
    Eight u;
    const Pair off = both(-mean), by = both(rstd);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        u.p[i] = (x.p[i] + off) * by;
    cut_off<WHOLE>(u, count);
    return u;
}

// v, the gradients of the normalised values u, to the gradients of the norm's input; zeros beyond the row.  u(r, i)
// gives the normalised values, twice, so that they need not be kept.  CLEAR: zeros beyond the row, for sums to come.
template <bool WHOLE, bool CLEAR, int ROWS, int V, typename U>
__device__ __forceinline__ void norm_back(Member& m, Exchange& e, const NormArgs& a, int kind, const int (&count)[V], U&& u,
                                          const float (&rstd)[ROWS], Eight (&v)[ROWS][V])
{
    float slope[ROWS], shift[ROWS];
    if (kind == ADASUM_NORM_LAYER) {
        float s[2 * ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            s[r] = s[ROWS + r] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[r] += dot_of(u(r, i), v[r][i]);
                s[ROWS + r] += sum_of(v[r][i]);
            }
        }
        group_sum(m, e, s);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            slope[r] = s[r] * a.inv_features;
            shift[r] = s[ROWS + r] * a.inv_features;
        }
    } else {
        float s[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            s[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i)
                s[r] += dot_of(u(r, i), v[r][i]);
        }
        group_sum(m, e, s);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            slope[r] = s[r] * a.inv_features;
            shift[r] = 0.0f;
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const Pair off = both(-shift[r]), down = both(-slope[r]), by = both(rstd[r]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const Eight n = u(r, j);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[r][j].p[i] = fma2(n.p[i], down, v[r][j].p[i] + off) * by;
            if (CLEAR && count[j] <= 0)
                v[r][j] = Eight{};
            cut_off<WHOLE>(v[r][j], count[j]);
        }
    }
}

__device__ __forceinline__ void write_sum(void* dst, int dtype, int64_t at, float sum, float scale, bool accumulate)
{
    float y = sum * scale;
    if (accumulate)
        y += load_as_float(dst, dtype, at);
    store_from_float(dst, dtype, at, y);
}

// Where a group stands in its units.
struct Turn {
    uint32_t step, unit;
    int64_t row, end;          // first row of the turn, end of the unit
    __device__ __forceinline__ Turn(const Deal& d, uint32_t group, int64_t rows) : step(0), unit(group) { enter(d, rows); }
    __device__ __forceinline__ void enter(const Deal& d, int64_t rows)
    {
        if (d.units <= d.pieces) {               // one gate row: nothing to divide
            row = (int64_t)unit * d.unit_rows;
            end = unit < d.units ? min(rows, row + d.unit_rows) : row;
            return;
        }
        const uint32_t of = unit / d.pieces, piece = unit - of * d.pieces;
        const int64_t span_end = min(rows, (int64_t)(of + 1) * d.gate_rows_span);
        row = (int64_t)of * d.gate_rows_span + (int64_t)piece * d.unit_rows;
        end = unit < d.units ? min(span_end, row + d.unit_rows) : row;
    }
    __device__ __forceinline__ void advance(const Deal& d, int64_t rows)
    {
        row += d.rows_at_once;
        if (++step == d.steps) {
            step = 0;
            unit += d.groups;
            enter(d, rows);
        }
    }
};

// WHOLE: 16-byte aligned rows of whole vectors.  FULL: a norm after the block or a gate.
//
// With the join, 16384 x 1024 bf16 and an RMS norm 41 us (4.1 TB/s), a layer norm with dropout 50 us: latency at 16 warps per
// multiprocessor, 65 % of the issue slots.
// 4096 x 4096 bf16 with an fp32 stream, two norms and a gate 115 us (2.6 TB/s): a row's way through two sums and three reads of its
// values from shared memory, at 16 warps (128 registers).  999 x 203 fp32 14.5 us, one row 7.9 us: two launches.
// Registers: 16384 x 1024 with a layer norm 64: 53 us, 80: 48, 96: 43.
template <typename T, typename R, bool WHOLE, bool FULL, int V>
__global__ void __maxnreg__(FULL ? 128 : 96)
residual_norm_grad_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int ROWS = WHOLE ? 1 : 2;
    extern __shared__ __align__(16) unsigned char rows_shared[];
    __shared__ Exchange exchange;
    float* columns = reinterpret_cast<float*>(rows_shared + a.rows_at);      // after the rows
    start_next_kernel();
    Member m(a.deal);
    blocks_present(a.deal);
    wait_for_previous_kernel();
    int count[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        count[v] = m.count(v, a.features);
    const bool post = FULL && a.post != ADASUM_NORM_NONE, pre = a.pre != ADASUM_NORM_NONE && a.grad_y;
    const bool with_x = FULL && a.x;
    Staged staged = stage_vectors(a, m, rows_shared, ROWS, V);
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(rows_shared)) + a.rows_at + threadIdx.x * 16;
    const uint32_t apart = blockDim.x * 16, stage_bytes = a.turn_pieces * apart;
    const uint32_t turns = a.deal.rounds * a.deal.steps;
    // places of a row's vectors among the thread's pieces
    const uint32_t t_bytes = V * (uint32_t)(sizeof(T) / 2) * apart, r_bytes = V * (uint32_t)(sizeof(R) / 2) * apart;
    const uint32_t h_piece = t_bytes, d_piece = pre ? t_bytes + r_bytes : 0, x_piece = d_piece + (a.grad_h ? r_bytes : 0);
    Turn now(a.deal, m.group, a.rows), ahead(a.deal, m.group, a.rows);
    auto bring = [&](uint32_t turn, uint32_t stage) {
        if (turn < turns) {
            uint32_t slot = mine + stage * stage_bytes;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int64_t row = ahead.row + r;
                const bool valid = row < ahead.end;
                if (pre) {
                    fetch_row<T>(slot, apart, a.grad_y, row * a.grad_y_stride + m.column(0), m.members, valid, count);
                    fetch_row<R>(slot, apart, a.h, row * a.h_stride + m.column(0), m.members, valid, count);
                }
                if (a.grad_h)
                    fetch_row<R>(slot, apart, a.grad_h, row * a.grad_h_stride + m.column(0), m.members, valid, count);
                if (with_x)
                    fetch_row<T>(slot, apart, a.x, row * a.x_stride + m.column(0), m.members, valid, count);
            }
            ahead.advance(a.deal, a.rows);
        }
        close_turn();
    };
    // statistics of the next turn, loaded a turn ahead
    float next_stats[ROWS][4];
    auto load_stats = [&](const Turn& t) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool valid = t.row + r < t.end;
            const float* p = a.stats + t.row + r;
            if constexpr (FULL) {
                next_stats[r][0] = valid && a.post == ADASUM_NORM_LAYER ? *p : 0.0f;
                next_stats[r][1] = post ? valid ? p[a.rows] : 0.0f : 1.0f;
            }
            next_stats[r][2] = valid && pre && a.pre == ADASUM_NORM_LAYER ? p[2 * a.rows] : 0.0f;
            next_stats[r][3] = valid && pre ? p[3 * a.rows] : 0.0f;
        }
    };
    // sums of the vectors' gradients: pre weight, pre bias, then post weight, post bias, gate
    Eight sum[FULL ? kVectors : 2][V] = {};
    if constexpr (WHOLE) {
        for (int t = 0; t < a.deal.stages; ++t)
            bring(t, t);
    }
    uint64_t seed = 0;
    if (a.drop.seed)
        seed = *a.drop.seed;
    load_stats(now);
    uint32_t stage = 0;
    for (uint32_t turn = 0; turn < turns; ++turn) {
        int64_t row[ROWS];
        bool valid[ROWS];
        Eight d[ROWS][V];
        float rstd[ROWS], post_rstd[ROWS], post_mean[ROWS], mean[ROWS];
        if constexpr (WHOLE)
            wait_for_turn(a.deal.stages);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            row[r] = now.row + r;
            valid[r] = row[r] < now.end;
            if constexpr (FULL) {
                post_mean[r] = next_stats[r][0];
                post_rstd[r] = next_stats[r][1];
            }
            mean[r] = next_stats[r][2];
            rstd[r] = next_stats[r][3];
        }
        // rows stay in shared memory until they are used: as registers they would be more than a thread has
        const uint32_t slot = mine + stage * stage_bytes;
        auto row_of = [&](auto t, const void* base, int64_t stride, uint32_t piece, int r, int v) {
            using E = decltype(t);
            if constexpr (WHOLE) {
                return decode(fetched<E>(slot + piece + v * (uint32_t)(sizeof(E) / 2) * apart + r * (stage_bytes / ROWS), apart));
            } else {
                return decode(load_vector<false>(static_cast<const E*>(base) + row[r] * stride + m.column(v), valid[r] ? count[v] : 0));
            }
        };
        const uint32_t unit = now.unit;
        const bool last_of_unit = now.step + 1 == a.deal.steps;
        now.advance(a.deal, a.rows);
        load_stats(now);
        if (pre) {
            auto u = [&](int r, int v) {
                return kept_normalised<WHOLE>(row_of(R{}, a.h, a.h_stride, h_piece, r, v), mean[r], rstd[r], valid[r] ? count[v] : 0);
            };
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    d[r][v] = row_of(T{}, a.grad_y, a.grad_y_stride, 0, r, v);
                    const Eight n = u(r, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sum[0][v].p[i] = fma2(d[r][v].p[i], n.p[i], sum[0][v].p[i]);
                        sum[1][v].p[i] = sum[1][v].p[i] + d[r][v].p[i];
                    }
                }
            affine(staged.pre_weight, nullptr, m, d);
            norm_back<WHOLE, FULL>(m, exchange, a, a.pre, count, u, rstd, d);
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!pre)
                    d[r][v] = Eight{};
                if (a.grad_h) {
                    const Eight dh = row_of(R{}, a.grad_h, a.grad_h_stride, d_piece, r, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        d[r][v].p[i] = dh.p[i] + d[r][v].p[i];
                }
                if (a.grad_residual && valid[r] && count[v] > 0) {
                    Eight back = d[r][v];
                    if (a.residual_scale != 1.0f)
                        scale(back, a.residual_scale);
                    store_vector<WHOLE>(static_cast<R*>(a.grad_residual) + row[r] * a.grad_residual_stride + m.column(v), count[v], back);
                }
            }
        if (a.branch) {
            if (a.branch_scale != 1.0f) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        scale(d[r][v], a.branch_scale);
            }
            if constexpr (FULL) {
                auto u = [&](int r, int v) {
                    return kept_normalised<WHOLE>(row_of(T{}, a.x, a.x_stride, x_piece, r, v), post_mean[r], post_rstd[r],
                                                  valid[r] ? count[v] : 0);
                };
                if (a.gate.p) {
                    if constexpr (!WHOLE)
                        hold_gate<ROWS, V>(a, m, row, valid, staged);
                    if (a.want_gate) {
                        Eight n[ROWS][V];
#pragma unroll
                        for (int r = 0; r < ROWS; ++r)
#pragma unroll
                            for (int v = 0; v < V; ++v)
                                n[r][v] = u(r, v);
                        if (post)
                            affine(staged.post_weight, staged.post_bias, m, n);
                        if (a.drop.seed)
                            drop_vectors(a, m, seed, row, n);
#pragma unroll
                        for (int r = 0; r < ROWS; ++r)
#pragma unroll
                            for (int v = 0; v < V; ++v)
                                if (valid[r]) {
#pragma unroll
                                    for (int i = 0; i < 4; ++i)
                                        sum[4][v].p[i] = fma2(d[r][v].p[i], n[r][v].p[i], sum[4][v].p[i]);
                                }
                    }
#pragma unroll
                    for (int r = 0; r < ROWS; ++r)
#pragma unroll
                        for (int v = 0; v < V; ++v)
                            if (valid[r] && count[v] > 0) {
                                Eight g;
                                if constexpr (WHOLE)
                                    g = gate_eight<T>(a, row[r], m.column(v));
                                else
                                    g = shared_eight(staged.gate + (r * V + v) * 8);
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    d[r][v].p[i] = d[r][v].p[i] * g.p[i];
                            }
                }
                if (a.drop.seed)
                    drop_vectors(a, m, seed, row, d);
                if (post) {
#pragma unroll
                    for (int r = 0; r < ROWS; ++r)
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            const Eight n = u(r, v);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                sum[2][v].p[i] = fma2(d[r][v].p[i], n.p[i], sum[2][v].p[i]);
                                sum[3][v].p[i] = sum[3][v].p[i] + d[r][v].p[i];
                            }
                        }
                    affine(staged.post_weight, nullptr, m, d);
                    norm_back<WHOLE, false>(m, exchange, a, a.post, count, u, post_rstd, d);
                }
            } else {
                if (a.drop.seed)
                    drop_vectors(a, m, seed, row, d);
            }
            if (a.grad_x) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (valid[r] && count[v] > 0)
                            store_vector<WHOLE>(static_cast<T*>(a.grad_x) + row[r] * a.grad_x_stride + m.column(v), count[v], d[r][v]);
            }
        }
        if constexpr (WHOLE) {
            bring(turn + a.deal.stages, stage);
            stage = stage + 1 == (uint32_t)a.deal.stages ? 0 : stage + 1;
        }
        if constexpr (FULL) {
            if (last_of_unit && a.gate_by_unit) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float total[8];
                    values_of(sum[4][v], total);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (unit < a.deal.units && i < count[v]) {
                            if (a.gate_parts)
                                a.gate_parts[(int64_t)unit * a.columns + m.column(v) + i] = total[i];
                            else
                                write_sum(a.grad_gate, a.grad_gate_dtype, (int64_t)unit * a.features + m.column(v) + i, total[i],
                                          a.gate_scale, a.accumulate);
                        }
                    sum[4][v] = Eight{};
                }
            }
        }
    }
    // The block's sums: its groups' in order, a thread per column.
    const uint32_t part = a.deal.cluster > 1 ? blockIdx.x / a.deal.cluster : blockIdx.x;
    const int wide = V * m.members * 8, first = (int)m.rank * a.deal.block_vectors * 8;
    const int mine_at = (m.slot * V * m.members + (m.vector - (int)m.rank * a.deal.block_vectors)) * 8;
    const int end = min(a.deal.block_vectors * 8, (int)a.columns - first);
#pragma unroll
    for (int k = 0; k < (FULL ? kVectors : 2); ++k) {
        const int want = k < 2 ? k + 2 : k < 4 ? k - 2 : 4;      // as the arguments count them
        if (!a.want[want])
            continue;
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v)
            keep_eight(columns + mine_at + v * m.members * 8, sum[k][v]);
        __syncthreads();
        float* dst = a.parts + ((int64_t)part * kVectors + want) * a.columns + first;
        for (int c = threadIdx.x; c < end; c += blockDim.x) {
            float total = 0.0f;
#pragma unroll 4
            for (int g = 0; g < a.deal.groups_per_block; ++g)
                total += columns[g * wide + c];
            dst[c] = total;
        }
    }
}

// The parts of every sum added in order: grid.y = the vectors that are wanted, then the gate's rows.  128 columns x 32
// shares of the parts per block, four columns per thread: loads in flight are what it needs (4096 x 4096 with 8 gates: 4.4 us less
// than with a column per thread).
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
constexpr int kShares = 32, kJoinColumns = 128;
__global__ void __launch_bounds__(32 * kShares) residual_norm_join_kernel(const __grid_constant__ JoinArgs a)
{
    __shared__ float4 share[kShares][32];
    wait_for_previous_kernel();
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t column = (int64_t)blockIdx.x * kJoinColumns + 4 * lane;
    const bool gate = (int)blockIdx.y >= a.vectors;
    const uint32_t gate_row = blockIdx.y - a.vectors;
    const int v = gate ? 0 : a.which[blockIdx.y];
    const uint32_t n = gate ? a.pieces : a.parts_count;
    const int64_t apart = gate ? a.columns : kVectors * a.columns;
    const float* p = gate ? a.gate_parts + (int64_t)gate_row * a.pieces * a.columns : a.parts + v * a.columns;
    float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (column < a.columns) {
#pragma unroll 8
        for (uint32_t i = slice; i < n; i += kShares) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(p + i * apart + column));
            sum.x += x.x;
            sum.y += x.y;
            sum.z += x.z;
            sum.w += x.w;
        }
    }
    share[slice][lane] = sum;
    __syncthreads();
    const int64_t at = (int64_t)blockIdx.x * kJoinColumns + threadIdx.x;
    if (threadIdx.x < kJoinColumns && at < a.features) {
        const float* part = reinterpret_cast<const float*>(share) + threadIdx.x;
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < kShares; ++i)
            total += part[i * kJoinColumns];
        if (gate)
            write_sum(a.grad_gate, a.gate_dtype, (int64_t)gate_row * a.features + at, total, a.gate_scale, a.accumulate);
        else
            write_sum(a.grad[v], v == 4 ? a.gate_dtype : a.dtype, at, total, v == 4 ? a.gate_scale : a.scale, a.accumulate);
    }
}

// ---- host --------------------------------------------------------------------------------------------

// Bytes of the sums that a gradient call leaves for the joining kernel.
size_t norm_workspace(const adasum_residual_norm_t& b, bool by_unit)
{
    const int64_t columns = (b.features + 7) / 8 * 8;
    size_t total = (size_t)kMaxParts * kVectors * (size_t)columns * 4;
    if (by_unit) {
        // fewer than twice as many units as groups, which have one vector per thread beside a gate
        Deal d{};
        plan_groups(b.features, 1, 1, kGradThreads, &d);
        const size_t groups = (size_t)(kGradThreads / (d.warps == 1 ? d.lanes : 32 * d.warps));
        total += 2 * (size_t)kMaxProcessors * groups * (size_t)columns * 4;
    }
    return (total + 255) / 256 * 256;
}

}  // namespace
}  // namespace adasum

extern "C" {

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
    a.want_gate = g->grad_gate != nullptr;
    const int sms = device_sms() < kMaxProcessors ? device_sms() : kMaxProcessors;
    if (sms == 0)
        return fail(ADASUM_ERR_CUDA, "no device");
    const bool gate_whole = !a.gate.p || (a.gate.aligned && (b->gate_dtype == b->dtype || b->gate_dtype == ADASUM_F32));
    const bool vec = features % 8 == 0 && gate_whole && (!g->x || rows_aligned(g->x, g->x_stride, tb)) && (!pre || rows_aligned(g->h, g->h_stride, rb)) &&
                     (!pre || rows_aligned(g->grad_y, g->grad_y_stride, tb)) && (!g->grad_h || rows_aligned(g->grad_h, g->grad_h_stride, rb)) &&
                     (!g->grad_x || rows_aligned(g->grad_x, g->grad_x_stride, tb)) &&
                     (!g->grad_residual || rows_aligned(g->grad_residual, g->grad_residual_stride, rb));
    // two vectors per thread, where their sums leave registers for it and a row then has eight threads or more (bf16, RMS, with
    // 1, 2: 16384 x 1024 57, 42 us; 1024 x 16384 151, 59 us; beside a norm after the block, 4096 x 4096, 120, 130 us)
    const bool full = post || (branch && b->gate);
    const int per_thread = !vec || features <= 128 || full ? 1 : 2;
    if (!full)
        a.x = nullptr;                     // without a norm or a gate its values make no difference
    if (!post)
        a.post_weight = a.post_bias = Vector{};
    if (!pre)
        a.pre_weight = Vector{};
    a.pre_bias = Vector{};                 // gradients do not depend on it
    unsigned blocks;
    const int per_processor = plan_blocks(&a, vec, per_thread, vec ? 1 : 2, (int)((pre ? (tb + rb) / 2 : 0) + (g->grad_h ? rb / 2 : 0) + (a.x ? tb / 2 : 0)),
                                          full || per_thread == 1 ? kGradThreads : 640, {512, 256});
    if (per_processor == 0)
        return fail(ADASUM_ERR_ARG, "%lld features are too many", (long long)features);
    plan_units(rows, b->gate ? b->rows_per_gate : rows, by_unit, per_processor * sms < kMaxParts ? per_processor * sms : kMaxParts, &a.deal, &blocks);
    a.parts = static_cast<float*>(workspace);
    a.gate_parts = by_unit && a.deal.pieces > 1 ? a.parts + (size_t)kMaxParts * kVectors * (size_t)a.columns : nullptr;
    JoinArgs j{};
    for (int v = 0; v < kVectors; ++v) {
        // without grad_y the norm before the next block has no part in the gradients: its vectors' are zero
        a.want[v] = vector_grads[v] != nullptr && !(v == 4 && by_unit);
        j.grad[v] = vector_grads[v];
        if (a.want[v])
            j.which[j.vectors++] = v;
    }
    profile_mark(stream, -1, 0, 0, true);
    cudaError_t err = cudaSuccess;
    with_types(*b, [&](auto t, auto r) {
        using T = decltype(t);
        using R = decltype(r);
        const size_t threads = (size_t)threads_of(a.deal), sums = wanted > 0 ? threads * per_thread * 32 : 0;
        const size_t rows_bytes = vec ? (size_t)a.deal.stages * a.turn_pieces * threads * 16 : 0;
        auto* kernel = !vec               ? residual_norm_grad_kernel<T, R, false, true, 1>
                       : per_thread == 2 ? residual_norm_grad_kernel<T, R, true, false, 2>
                                         : residual_norm_grad_kernel<T, R, true, true, 1>;
        static std::atomic<uint64_t> prepared[3] = {};         // of these types' kernels
        err = launch_rows(kernel, prepared[!vec ? 0 : per_thread], blocks, a, a.rows_at + (rows_bytes > sums ? rows_bytes : sums), stream);
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
        ADASUM_CUDA_CHECK(launch_after(residual_norm_join_kernel, dim3((unsigned)((features + kJoinColumns - 1) / kJoinColumns), (unsigned)joined), 32 * kShares, 0,
                                       stream, j));
        profile_mark(stream, ADASUM_KERNEL_RESIDUAL_NORM_GRAD, 1, 0, false);
    }
    return ADASUM_OK;
}

}  // extern "C"
