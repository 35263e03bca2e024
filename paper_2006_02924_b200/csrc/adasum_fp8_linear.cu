// Products of packed 8-bit matrices: a linear layer, and the gradient of its input.
//
//     y[r][n]  = sum_k x[r][k] w[n][k] + bias[n]
//     dx[r][k] = sum_n dy[r][n] w[n][k]
//
// D[m][t] = sum over s of W[m][s] T[t][s] on the fifth-generation tensor cores, with the weights' outputs (features, for the
// gradient) as rows m and the tokens as columns t, so that the lanes of a warp hold neighbouring elements of a row of the
// result.  2 R N K operations on R K + N K bytes read and R N elements written: bound by the tensor cores from a few
// hundred tokens on, by the weights' bytes (and the launch) below.
//
// The instruction multiplies e4m3 codes and applies a power of two per row and 32 products of either operand itself
// (block scaling).  Steps cover 128 products here, so one step byte serves the four instructions of a step of depth 128.  The gradient
// reads the same packed weights with the summed index as the slow one ("MN-major"): a step per 128 x 128 block is
// the same for either direction, and nothing is transposed.
//
// A pair of blocks (a cluster of two) owns a tile of 256 rows m x TOKENS tokens.  Each block brings 128 rows of W and
// half the tokens per step, and its tensor core multiplies its 128 rows with all tokens: with the operands halved per
// block, shared memory and the L2 deliver half of what two separate blocks would need.
//
//   copies   one thread per block: bulk tensor copies of 128 x 128 codes of W and TOKENS / 2 x 128 of T, 128-byte swizzle,
//            zeros beyond the matrices, and of the step bytes of its rows and of all tokens
//   D        one thread of the pair's first block copies the step bytes to tensor memory and issues the multiplications;
//            sixteen warps per block add the sums from tensor memory into fp32 registers and store the result
//
// Sums are formed in tensor memory over kChain steps (1024 products) at most: the tensor core truncates where it adds, and over
// thousands of products that adds up.  Tensor memory (512 columns) holds two such sums, so that the next is formed while
// the previous one is read, and two sets of step bytes; that is why a tile has 192 tokens and not 256.  (240 would
// fit, but such tiles begin inside a block of step bytes, and the stores and the fence that it takes to move them to their places cost
// every step 1200 cycles on its way: with four warps in turn 71 to 83 us for 16384 tokens, 1024 to 4096, and 243 to 280 for 4096 to
// 4096, against 73 and 254.)  Small products take tiles of 128 or 64 tokens, so that more pairs have one (plan_tiles).
//
// What bounds it: with all pairs at work, in part shared memory (each tensor core reads its rows and all tokens of a step, 448
// cycles for 384 of multiplications) and the power limit; tiles of 192 tokens also spill 72 to 80 bytes a thread: 16384 tokens in bf16, 1024 to 4096 67 us (2.05 PFLOP/s), its gradient 66 us (2.07),
// 4096 to 4096 250 us (2.2); a product of 8192 x 8192 x 8192 470 to 530 us (2.1 to 2.3).  The tensor cores' counter stands at 51
// to 58 %.  Small products are bound by start and latency: 1024 to 4096, 1 to 64 tokens 5.7 us, 512 tokens 7.2, 2048 tokens 13.8.
//
// Tiles are dealt to the pairs whole, unless that leaves too many pairs idle; then the steps of all tiles are cut into
// equal runs, and a tile whose steps fall to several pairs is joined, in their order, by fp8_join_kernel.  The
// association of every sum is fixed by the sizes and the number of pairs that fit the device.
//
// Where a tile has five to eight steps and a pair several tiles of the same rows, the weights' codes stay in shared memory
// and only tokens move: less than half the bytes from the L2 (16384 tokens, 1024 to 4096: 73 -> 67 us).
//
// Every wait has a limit.  A thread whose wait runs out records it and goes on without waiting, but hands over and issues
// nothing more, so the waits that depend on it run out in turn and the launch ends; the block leaves NaN for all its
// shares of tiles, and adasum_fp8_linear_status reports it.  Before a block ends its copies have landed, and the
// pair's multiplications and their arrivals are done.
#include <atomic>

#include "adasum_fp8.cuh"
#include "adasum_tensor.cuh"

namespace adasum {
namespace {

constexpr int kHalf = 128;                       // rows of W that a block of the pair brings
constexpr int kTileRows = 2 * kHalf;
constexpr int kDepth = kFp8Block;                // products per step
constexpr int kChain = 8;                        // steps that are summed in tensor memory
constexpr int kStaySteps = 8;                     // of a tile whose weights may stay
constexpr int kShortChain = 4;                   // at least, where few tiles are cut: shorter runs save less than their parts cost to join
constexpr int kWeightBytes = kHalf * kDepth;     // of a step and block
constexpr int kParts = 4;                        // of a tile's tokens: four warps sum and store each
constexpr int kSumWarps = 4 * kParts, kCopyWarp = kSumWarps, kMultiplyWarp = kCopyWarp + 1, kMemoryWarp = kCopyWarp + 2;
constexpr int kBlockThreads = 32 * (kSumWarps + 4);
constexpr uint32_t kBand = 8;                     // tiles of rows that are dealt out next to each other
constexpr int kMaxPairs = 74;                    // 148 multiprocessors
constexpr size_t kStatusBytes = 1024;
constexpr int kStatusCount = 255;                // word that holds the number of blocks
constexpr long long kWaitCycles = 2000000000;    // about a second (a real wait is microseconds): the clock counts pauses too
constexpr long long kSelftestCycles = 2000000;   // about a millisecond
constexpr int kLastWait = 4;                     // limits, for the last commit: other warps' waits may have to run out first

// Shared memory: the stages' codes, then the stages' step bytes.  A step's weights are part of its stage, or (STAY) have places
// of their own in front of the stages' codes and step bytes, one per step of a tile.
template <int TOKENS, bool STAY>
struct Shape {
    static constexpr int kHalfTokens = TOKENS / 2, kPartTokens = TOKENS / kParts;
    static constexpr int kTokenBytes = kHalfTokens * kDepth;             // whole groups of 8 rows: 1024-byte aligned
    static constexpr int kStageBytes = (STAY ? 0 : kWeightBytes) + kTokenBytes;
    // blocks of 128 rows that a tile's tokens lie in; a tile starts at the beginning of one or 64 rows into it
    static constexpr int kRowBlocks = TOKENS > 128 ? 2 : 1;
    static constexpr int kScaleBytes = ((STAY ? 0 : 1) + kRowBlocks) * kFp8StepBytes;     // step bytes of the block's rows and of the tokens
    static constexpr int kStages = TOKENS > 128 ? 7 : 8;
    static constexpr int kStayBytes = STAY ? kStaySteps * kWeightBytes : 0, kStayScaleBytes = STAY ? kStaySteps * kFp8StepBytes : 0;
    static constexpr size_t kSharedBytes =
        (size_t)kStages * (kStageBytes + kScaleBytes) + kStayBytes + kStayScaleBytes + 1024;      // + room to align to 1024
    // columns of tensor memory: a sum, step bytes (4 for the rows, 4 or 8 for the tokens), the other sum, step bytes
    static constexpr int kSumColumns = 256, kScaleAt = 192;
    static_assert(TOKENS == 192 || TOKENS == 128 || TOKENS == 64, "");
    static_assert(kSharedBytes <= 227 * 1024 - 512, "");
};

struct LinearArgs {
    int64_t rows, wide;                // of the result
    const void* bias;
    int bias_dtype;
    void* out;
    int64_t out_stride;
    int out_dtype;
    bool pairs_aligned;                // two neighbouring elements may be stored at once
    // units of chain_steps steps, tile after tile (tiles of the same tokens next to each other)
    uint32_t tiles_k, tiles, iterations, chain_steps, chains, units;
    bool whole;                        // no tile is cut: runs are whole tiles
    int* status;                       // one word per block, and their number
    long long wait_cycles;             // limit of a wait
    int withheld;                      // hand-over that never completes (self-test), or ADASUM_HAND_OVER_NONE
    float* slots;                      // [pair][first or last tile of its run][block][token][row of the block]
};

// Where a role stands in its pair's work.  Whole tiles are dealt out one by one, pair after pair, so that the pairs walk
// the summed index in step and read the same rows at the same time; cut ones as runs (4608 tokens, 4096 to 4096: whole tiles 73 us,
// runs and the join 86); tiles whose weights stay as runs too, tokens fastest.
template <bool STAY>
struct Walk : Cursor {
    uint32_t pairs, until;
    __device__ __forceinline__ Walk(const LinearArgs& a, uint32_t pairs_, uint32_t pair)
        : Cursor(a, a.whole ? 0 : first_unit(a.units, pairs_, pair), a.whole ? 0 : first_unit(a.units, pairs_, pair + 1)), pairs(pairs_)
    {
        if (a.whole) {
            part = 0;
            if constexpr (STAY) {
                unit = first_unit(a.tiles, pairs, pair) * a.chains;
                until = first_unit(a.tiles, pairs, pair + 1) * a.chains;
            } else {
                unit = pair * a.chains;
                until = a.units;
            }
            enter_tile(a);
        }
    }
    __device__ __forceinline__ void enter_tile(const LinearArgs& a)
    {
        if (unit >= until) {
            part = 3;
            return;
        }
        chain = 0;
        stop = unit + a.chains;
        const uint32_t tile = unit / a.chains, tiles_n = a.tiles / a.tiles_k;
        if constexpr (STAY) {
            tile_k = tile / tiles_n;
            tile_n = tile - tile_k * tiles_n;
            return;
        }
        // in bands of kBand tiles of rows, so that the tiles at hand share both operands (16384 tokens, 4096 to 4096: row after
        // row 266 us, in bands 254)
        const uint32_t band = tile / (kBand * tiles_n), first = band * kBand, width = min(kBand, a.tiles_k - first);
        const uint32_t rest = tile - first * tiles_n;
        tile_n = rest / width;
        tile_k = first + rest - tile_n * width;
    }
    __device__ __forceinline__ void advance(const LinearArgs& a)
    {
        if (!a.whole) {
            Cursor::advance(a);
            return;
        }
        ++chain;
        if (++unit == stop) {
            if (!STAY)
                unit += (pairs - 1) * a.chains;
            enter_tile(a);
        }
    }
};

// ---- instructions ------------------------------------------------------------------------------------

// An address in the shared memory of the pair's first block.
__device__ __forceinline__ uint32_t address_in_first(uint32_t address)
{
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(remote) : "r"(address));
    return remote;
}
// Copies to this block's shared memory whose bytes count on a barrier of either block of the pair.
__device__ __forceinline__ void copy_to_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
                 "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void copy_to_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
                 "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}

// Codes with the summed index fast: rows of 128 bytes, eight rows 1024 bytes, 128-byte swizzle.  The same words describe
// codes with the summed index slow: 128 rows m side by side, eight products 1024 bytes further.
__device__ __forceinline__ uint64_t codes_descriptor(uint32_t address)
{
    return (uint64_t)((address & 0x3ffffu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// Step bytes: 32 rows of 16 bytes, eight rows 128 bytes, no swizzle.
__device__ __forceinline__ uint64_t steps_descriptor(uint32_t address)
{
    return (uint64_t)((address & 0x3ffffu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
__device__ __forceinline__ void copy_steps(uint32_t tensor_address, uint64_t descriptor)
{
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tensor_address), "l"(descriptor) : "memory");
}
__device__ __forceinline__ void multiply(uint32_t sum, uint64_t w, uint64_t t, uint32_t instruction, uint32_t w_steps,
                                         uint32_t t_steps, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(sum),
                 "l"(w), "l"(t), "r"(instruction), "r"(w_steps), "r"(t_steps), "r"(accumulate)
                 : "memory");
}
// N consecutive columns of tensor memory, 8 or 4 at a time; the caller waits for them.
template <int N>
__device__ __forceinline__ void load_sums(uint32_t address, float* r)
{
    if constexpr (N >= 8) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
                     : "r"(address)
                     : "memory");
        load_sums<N - 8>(address + 8, r + 8);
    } else if constexpr (N == 4) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3])
                     : "r"(address)
                     : "memory");
    }
}
// What was loaded may be used only after the wait.
template <int N>
__device__ __forceinline__ void wait_for_sums(float* r)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i)
        asm volatile("" : "+f"(r[i]));
}

// A thread's column of the result: one row m, consecutive tokens.
template <typename TO, int COUNT>
__device__ __forceinline__ void write_column(const LinearArgs& a, int64_t t, int64_t m, float bias, const float (&sum)[COUNT])
{
    TO* p = static_cast<TO*>(a.out) + t * a.out_stride + m;
    const int count = m < a.wide ? (int)min((int64_t)COUNT, a.rows - t) : 0;
#pragma unroll
    for (int i = 0; i < COUNT; ++i, p += a.out_stride)
        if (i < count)
            store_from_float(p, TypeCode<TO>::value, 0, sum[i] + bias);
}
// The same with two elements per store: of two tokens, lanes of even rows take the first and those of odd rows the second,
// both with their neighbour's element.  Every row and the result start on two elements.
template <typename TO, int COUNT>
__device__ __forceinline__ void write_pairs(const LinearArgs& a, int64_t t, int64_t m, float bias, const float (&sum)[COUNT])
{
    const int odd = threadIdx.x & 1;
    const int count = m < a.wide ? (int)min((int64_t)COUNT, a.rows - t) - odd : 0;
    TO* p = static_cast<TO*>(a.out) + (t + odd) * a.out_stride + (m - odd);
    const int64_t step = 2 * a.out_stride;
#pragma unroll
    for (int i = 0; i < COUNT; i += 2, p += step) {
        const float x = sum[i] + bias, y = sum[i + 1] + bias;
        const float other = __shfl_xor_sync(0xffffffffu, odd ? x : y, 1);
        const float low = odd ? other : x, high = odd ? y : other;
        if (i < count) {
            // the result does not stay in the L2 in place of the operands (16384 tokens, 1024 to 4096: 75.7 -> 73.2 us)
            if constexpr (__is_same(TO, float))
                __stcs(reinterpret_cast<float2*>(p), make_float2(low, high));
            else if constexpr (__is_same(TO, __half))
                __stcs(reinterpret_cast<__half2*>(p), __floats2half2_rn(low, high));
            else
                __stcs(reinterpret_cast<__nv_bfloat162*>(p), __floats2bfloat162_rn(low, high));
        }
    }
}
template <typename TO, int COUNT>
__device__ __forceinline__ void write(const LinearArgs& a, int64_t t, int64_t m, const float (&sum)[COUNT])
{
    const float bias = a.bias && m < a.wide ? load_as_float(a.bias, a.bias_dtype, m) : 0.0f;
    if (a.pairs_aligned)
        write_pairs<TO>(a, t, m, bias, sum);
    else
        write_column<TO>(a, t, m, bias, sum);
}

// What a thread of the warps that sum leaves for its row and tokens where a wait of its block ran out: NaN, over whatever
// it has left for any tile of the pair's run.
template <int TOKENS, bool STAY>
__device__ __noinline__ void leave_nan(const LinearArgs& a, uint32_t pairs, uint32_t pair, uint32_t rank, uint32_t thread)
{
    constexpr int kPartTokens = Shape<TOKENS, false>::kPartTokens;
    const float nan = __uint_as_float(0x7fc00000u);
    const int row = 32 * ((thread >> 5) & 3) + (thread & 31), part = thread >> 7;
    uint32_t chain_begin = 0;
    bool fresh = true;
    for (Walk<STAY> c(a, pairs, pair); !c.done(); c.advance(a)) {
        if (fresh)
            chain_begin = c.chain;
        fresh = c.last_of_share(a);
        if (!fresh)
            continue;
        const int64_t m = (int64_t)c.tile_k * kTileRows + rank * kHalf + row;
        const int64_t t = (int64_t)c.tile_n * TOKENS + part * kPartTokens;
        if (chain_begin == 0 && c.chain + 1 == a.chains) {
            for (int i = 0; i < kPartTokens && m < a.wide && t + i < a.rows; ++i)
                store_from_float(a.out, a.out_dtype, (t + i) * a.out_stride + m, nan);
        } else {
            float* dst = a.slots + ((int64_t)(2 * pair + (c.part == 0 ? 1 : 0)) * 2 + rank) * TOKENS * kHalf + part * kPartTokens * kHalf + row;
            for (int i = 0; i < kPartTokens; ++i)
                dst[i * kHalf] = nan;
        }
    }
}

// ---- kernel ------------------------------------------------------------------------------------------
//
// GRAD: the weights' summed index is their row.  STAY: the weights of a tile stay for the pair's next tile of the same rows.
template <int TOKENS, bool GRAD, bool STAY>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kBlockThreads, 1)
fp8_linear_kernel(const __grid_constant__ LinearArgs a, const __grid_constant__ CUtensorMap token_map,
                  const __grid_constant__ CUtensorMap weight_map, const __grid_constant__ CUtensorMap token_step_map,
                  const __grid_constant__ CUtensorMap weight_step_map)
{
    using S = Shape<TOKENS, STAY>;
    constexpr int kStages = S::kStages, kHalfTokens = S::kHalfTokens, kPartTokens = S::kPartTokens;
    extern __shared__ __align__(1024) unsigned char dynamic_shared[];
    // landed (first block): both blocks' codes and step bytes of a step are there; multiplied: the tensor cores are done with
    // the step.  formed: a sum in tensor memory is complete; taken (first block): it has been read by both blocks.
    // finished: so are all multiplications that were ever issued.  nowhere: what threads that gave up arrive on.
    __shared__ __align__(8) unsigned long long landed[kStages], multiplied[kStages], formed[2], taken[2], finished, nowhere[2];
    __shared__ uint32_t tensor_memory_slot;
    __shared__ volatile uint32_t gave_up;        // some wait of this block ran out

    start_next_kernel();             // the join; it waits for this kernel's end by itself
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t stay0 = (shared_address(dynamic_shared) + 1023u) & ~1023u, stage0 = stay0 + S::kStayBytes;
    const uint32_t stay_scales0 = stage0 + kStages * S::kStageBytes, scales0 = stay_scales0 + S::kStayScaleBytes;
    const uint32_t landed0 = shared_address(landed), multiplied0 = shared_address(multiplied);
    const uint32_t formed0 = shared_address(formed), taken0 = shared_address(taken);
    const uint32_t finished0 = shared_address(&finished), nowhere0 = shared_address(nowhere);

    if (threadIdx.x == 0) {
        gave_up = 0;
        // a barrier that expects one arrival too many never completes a phase
        auto init = [&](uint32_t bar, uint32_t count, int hand_over) { barrier_init(bar, count + (a.withheld == hand_over)); };
        for (int s = 0; s < kStages; ++s) {
            init(landed0 + 8 * s, 1, ADASUM_HAND_OVER_LANDED);
            init(multiplied0 + 8 * s, 1, ADASUM_HAND_OVER_MULTIPLIED);
        }
        for (int s = 0; s < 2; ++s) {
            init(formed0 + 8 * s, 1, ADASUM_HAND_OVER_FORMED);
            init(taken0 + 8 * s, 2 * kSumWarps, ADASUM_HAND_OVER_TAKEN);
            barrier_init(nowhere0 + 8 * s, 1);
        }
        barrier_init(finished0, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMemoryWarp) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
            shared_address(&tensor_memory_slot)));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (warp == kCopyWarp && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&token_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&weight_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&token_step_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&weight_step_map) : "memory");
    }
    __syncthreads();
    cluster_barrier();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tensor_memory = tensor_memory_slot;
    wait_for_previous_kernel();      // the one that packed the tokens; nothing above reads or writes global memory
    if (threadIdx.x == 0) {
        a.status[blockIdx.x] = 0;
        if (blockIdx.x == 0)
            a.status[kStatusCount] = (int)gridDim.x;
    }

    // After a wait of this thread ran out it neither waits nor acts for its warp any more (arrives, multiplies, commits).
    bool waiting = true;
    uint32_t taken_at = taken0;
    auto wait_up_to = [&](uint32_t bar, uint32_t parity, long long cycles) {
        if (waiting && !wait_phase(bar, parity, cycles)) {
            waiting = false;
            taken_at = nowhere0;
            gave_up = 1;
            atomicExch(a.status + blockIdx.x, (int)ADASUM_DEVICE_TIMEOUT);
        }
    };
    auto wait = [&](uint32_t bar, uint32_t parity) { wait_up_to(bar, parity, a.wait_cycles); };

    if (warp < kSumWarps) {
        // ---- sums: warp w reads tensor-memory lanes 32 (w % 4) .. + 31 (rows m) of a quarter of the tokens
        const int quarter = warp & 3, part = warp >> 2;
        float sum[kPartTokens];
        uint32_t count = 0, chain_begin = 0;
        bool fresh = true;                       // the next unit is the first of its tile's share
        for (Walk<STAY> c(a, pairs, pair); !c.done(); c.advance(a), ++count) {
            if (fresh)
                chain_begin = c.chain;
            wait(formed0 + 8 * (count & 1), (count >> 1) & 1);
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t source = tensor_memory + (count & 1) * S::kSumColumns + part * kPartTokens + ((uint32_t)(32 * quarter) << 16);
            if (fresh) {
                load_sums<kPartTokens>(source, sum);
                wait_for_sums<kPartTokens>(sum);
            } else {
                constexpr int kBatch = 16;
#pragma unroll
                for (int g = 0; g < kPartTokens; g += kBatch) {
                    float r[kBatch];
                    load_sums<kBatch>(source + g, r);
                    wait_for_sums<kBatch>(r);
#pragma unroll
                    for (int i = 0; i < kBatch; ++i)
                        sum[g + i] += r[i];
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0)
                arrive_at_first(taken_at + 8 * (count & 1));

            fresh = c.last_of_share(a);
            if (!fresh)
                continue;
            // ---- the pair's last unit of this tile: the result, or this pair's part of it
            const int row = 32 * quarter + lane;
            if (chain_begin == 0 && c.chain + 1 == a.chains) {
                const int64_t m = (int64_t)c.tile_k * kTileRows + rank * kHalf + row;
                const int64_t t = (int64_t)c.tile_n * TOKENS + part * kPartTokens;
                if (a.out_dtype == ADASUM_F32)
                    write<float>(a, t, m, sum);
                else if (a.out_dtype == ADASUM_F16)
                    write<__half>(a, t, m, sum);
                else
                    write<__nv_bfloat16>(a, t, m, sum);
            } else {
                float* dst = a.slots + ((int64_t)(2 * pair + (c.part == 0 ? 1 : 0)) * 2 + rank) * TOKENS * kHalf + part * kPartTokens * kHalf + row;
#pragma unroll
                for (int i = 0; i < kPartTokens; ++i)
                    dst[i * kHalf] = sum[i];
            }
        }
        if (gave_up != 0)
            leave_nan<TOKENS, STAY>(a, pairs, pair, rank, threadIdx.x);
        // The last commit arrives in both blocks, and each waits for its own: in this warp, which has just seen the last sum.
        if (warp == 0) {
            waiting = true;
            wait_up_to(finished0, 0, kLastWait * a.wait_cycles);
        }
    } else if (warp == kCopyWarp) {
        // ---- copies of this block's rows of the weights and of its half of the tokens, and of the step bytes of both.
        // Both blocks' copies count on the first block's barrier, which expects their bytes.
        Ring<kStages> ring;
        uint32_t issued = 0;
        constexpr uint32_t kBytes = 2 * (S::kStageBytes + S::kScaleBytes), kStayingBytes = 2 * (kWeightBytes + kFp8StepBytes);
        uint32_t held = ~0u;                     // STAY: rows whose weights are there
        const uint32_t first_landed0 = address_in_first(landed0);
        for (Walk<STAY> c(a, pairs, pair); !c.done() && waiting; c.advance(a)) {
            const int m = (int)(c.tile_k * kTileRows + rank * kHalf), t = (int)(c.tile_n * TOKENS + rank * kHalfTokens);
            const int m_block = (int)(c.tile_k * 2 + rank), t_block = (int)((int64_t)c.tile_n * TOKENS / kFp8Block);
            const uint32_t end = c.first_step(a) + c.steps(a);
            const bool bring = !STAY || c.tile_k != held;
            held = c.tile_k;
            for (uint32_t step = c.first_step(a); step < end; ++step) {
                wait(multiplied0 + 8 * ring.stage, ring.phase ^ 1);
                // the last tile's step of the same place, which the stage's turn does not cover where tiles are short
                if (STAY && bring && a.iterations < (uint32_t)kStages && issued >= a.iterations) {
                    const uint32_t last = issued - a.iterations;
                    wait(multiplied0 + 8 * (last % kStages), (last / kStages) & 1);
                }
                waiting = __all_sync(0xffffffffu, waiting);
                if (!waiting)
                    break;
                const uint32_t dst = stage0 + ring.stage * S::kStageBytes, steps = scales0 + ring.stage * S::kScaleBytes;
                const uint32_t w_dst = STAY ? stay0 + step * kWeightBytes : dst, w_steps = STAY ? stay_scales0 + step * kFp8StepBytes : steps;
                const uint32_t t_dst = STAY ? dst : dst + kWeightBytes, t_steps = STAY ? steps : steps + kFp8StepBytes;
                const uint32_t bar = first_landed0 + 8 * ring.stage;
                const int s = (int)step;
                if (elected()) {
                    if (rank == 0)
                        expect_bytes(landed0 + 8 * ring.stage, STAY && bring ? kBytes + kStayingBytes : kBytes);
                    if (bring) {
                        copy_to_pair(w_dst, &weight_map, GRAD ? m : s * kDepth, GRAD ? s * kDepth : m, bar);
                        // the words of all rows of a block of the weights are the same: they serve either direction
                        copy_to_pair(w_steps, &weight_step_map, 0, GRAD ? m_block : s, GRAD ? s : m_block, bar);
                    }
                    copy_to_pair(t_dst, &token_map, s * kDepth, t, bar);
#pragma unroll
                    for (int i = 0; i < S::kRowBlocks; ++i)
                        copy_to_pair(t_steps + i * kFp8StepBytes, &token_step_map, 0, s, t_block + i, bar);
                }
                __syncwarp();
                ++issued;
                ring.advance();
            }
        }
        // Nothing may still be on its way into shared memory when the blocks end.  The first block's barrier counts both
        // blocks' copies; where the blocks issued different numbers, some wait has run out since, a thousand times the
        // copies' time ago.
        waiting = true;
        for (uint32_t back = rank == 0 ? min(issued, (uint32_t)kStages) : 0; back > 0; --back) {
            const uint32_t step = issued - back;
            wait(landed0 + 8 * (step % kStages), (step / kStages) & 1);
        }
    } else if (warp == kMultiplyWarp && rank == 0) {
        // ---- multiplications: e4m3 codes, steps as powers of two, fp32 sums, 256 x TOKENS
        constexpr uint32_t kInstruction = ((GRAD ? 1u : 0u) << 15) | ((uint32_t)(TOKENS >> 3) << 17) | (1u << 23) |
                                          ((uint32_t)(kTileRows >> 4) << 24);
        // One thread does all of it: what it spends per step must stay below the multiplications' 384 cycles.
        if (elected()) {
            Ring<kStages> ring;
            uint32_t count = 0, turn = 0;
            const uint64_t codes0 = codes_descriptor(stage0), steps0 = steps_descriptor(scales0);
            const uint64_t stay_codes0 = codes_descriptor(stay0), stay_steps0 = steps_descriptor(stay_scales0);
            for (Walk<STAY> c(a, pairs, pair); !c.done(); c.advance(a), ++count) {
                const uint32_t target = tensor_memory + (count & 1) * S::kSumColumns;
                const uint32_t offset = (c.tile_n * TOKENS % kFp8Block) / 32;        // columns of 32 tokens each
                wait(taken0 + 8 * (count & 1), ((count >> 1) & 1) ^ 1);
                uint32_t accumulate = 0, place = 0;
                for (uint32_t steps = c.steps(a); steps > 0; --steps) {
                    wait(landed0 + 8 * ring.stage, ring.phase);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (waiting) {
                        const uint64_t stage = codes0 + ring.stage * (S::kStageBytes >> 4), stage_steps = steps0 + ring.stage * (S::kScaleBytes >> 4);
                        const uint64_t w = STAY ? stay_codes0 + place * (kWeightBytes >> 4) : stage;
                        const uint64_t t = STAY ? stage : stage + (kWeightBytes >> 4);
                        const uint64_t b = STAY ? stage_steps : stage_steps + (kFp8StepBytes >> 4);
                        const uint32_t w_steps = tensor_memory + S::kScaleAt + (turn & 1) * S::kSumColumns, t_steps = w_steps + 4;
                        copy_steps(w_steps, STAY ? stay_steps0 + place * (kFp8StepBytes >> 4) : stage_steps);
                        copy_steps(t_steps, b);
                        if (S::kRowBlocks > 1)
                            copy_steps(t_steps + 4, b + (kFp8StepBytes >> 4));
#pragma unroll
                        for (int s = 0; s < kDepth / 32; ++s)
                            // 32 products are 32 bytes further on, or 32 rows of 128 bytes (in units of 16)
                            multiply(target, w + (GRAD ? 256 : 2) * s, t + 2 * s, kInstruction, w_steps, t_steps + offset,
                                     s > 0 ? 1u : accumulate);
                        commit_to_both(multiplied0 + 8 * ring.stage);
                        if (steps == 1)
                            commit_to_both(formed0 + 8 * (count & 1));
                    }
                    accumulate = 1;
                    ++place;
                    ++turn;
                    ring.advance();
                }
            }
            commit_to_both(finished0);
        }
        __syncwarp();
    }
    __syncwarp();
    // Neither block may end, nor free its tensor memory, while the other still multiplies or arrives here: both have
    // waited for the last commit, the first block's copies of it included.
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    cluster_barrier();
    if (warp == kMemoryWarp)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tensor_memory) : "memory");
}

// Tiles whose units fell to several pairs: the pairs' parts added in order.  grid.x = tiles, grid.y = parts of a tile's
// 2 x `tokens` rows of 128; one warp per row, four elements per lane.  Latency: 3 to 4 us (64 tokens, 4096 to 1024: 32 parts, 8.8 us
// with the product) to 9 (512 tokens, 8192 to 1024: 12 MB of parts from the L2).
constexpr int kJoinThreads = 256;

__global__ void __launch_bounds__(kJoinThreads)
fp8_join_kernel(const __grid_constant__ LinearArgs a, uint32_t pairs, int tokens, bool vec)
{
    wait_for_previous_kernel();
    const uint32_t tile = blockIdx.x;
    const uint32_t first = pair_of_unit(a.units, pairs, tile * a.chains);
    const uint32_t last = pair_of_unit(a.units, pairs, tile * a.chains + a.chains - 1);
    if (first == last)
        return;                      // written by the product itself
    const int at = blockIdx.y * (kJoinThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (at >= 2 * tokens)
        return;
    const uint32_t tile_k = tile % a.tiles_k, tile_n = tile / a.tiles_k;
    // only the first pair's run can have started in an earlier tile
    const uint32_t first_slot = 2 * first + (tile == first_unit(a.units, pairs, first) / a.chains ? 0 : 1);
    const int64_t slot_floats = (int64_t)2 * tokens * kHalf;
    const float* source = a.slots + (int64_t)at * kHalf + 4 * lane;
    float sum[4] = {};
#pragma unroll 8
    for (uint32_t pair = first; pair <= last; ++pair) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(source + (pair == first ? first_slot : 2 * pair) * slot_floats));
        sum[0] += v.x;
        sum[1] += v.y;
        sum[2] += v.z;
        sum[3] += v.w;
    }
    const int64_t t = (int64_t)tile_n * tokens + at % tokens;
    const int64_t m = (int64_t)tile_k * kTileRows + at / tokens * kHalf + 4 * lane;
    if (t >= a.rows || m >= a.wide)
        return;
    const int64_t e = t * a.out_stride + m;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (a.bias && m + i < a.wide)
            sum[i] += load_as_float(a.bias, a.bias_dtype, m + i);
    if (vec) {
        store_vector_from_float<4>(a.out, a.out_dtype, e, sum);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (m + i < a.wide)
                store_from_float(a.out, a.out_dtype, e + i, sum[i]);
    }
}

// Nothing to sum: the bias, or zeros.
__global__ void __launch_bounds__(256) fp8_bias_kernel(const __grid_constant__ LinearArgs a, RowDivider divider, uint64_t elements)
{
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n == 0)
        a.status[kStatusCount] = 0;
    if (n >= elements)
        return;
    uint64_t row;
    uint32_t column;
    divide_row(divider, n, row, column);
    store_from_float(a.out, a.out_dtype, (int64_t)row * a.out_stride + column,
                     a.bias ? load_as_float(a.bias, a.bias_dtype, column) : 0.0f);
}

// ---- host --------------------------------------------------------------------------------------------

struct Work {
    int tokens;                // of a tile
    uint32_t tiles_k, tiles, iterations, chain_steps, chains, units, pairs;
    bool fits, whole, stay;
    int64_t cost;              // cycles, about
};

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to; }

// Tiles of `tokens` tokens.  `most`: pairs that run at once.  A step costs shared memory (of 64 tokens: the loads from the
// L2) about 448, 360 and 320 cycles for 192, 128 and 64 tokens.  Tiles are dealt out whole, or cut into equal runs of steps whose
// parts a second kernel joins, whichever comes to less.  The join costs a launch, the parts' way through the L2 and, where
// the product leaves it no idle multiprocessors to be brought in early, another microsecond.  Measured on 60 products of 1 to
// 4608 tokens, the choice is the best of the six in 53 and 4 % off at worst (8192 to 1024, 512 tokens: 64 whole 19.4 us, cut
// 18.3, 128 whole 20.1, cut 16.8, 192 whole 23.3, cut 19.4; 2048 tokens: 35.8, 39.1, 21.1, 27.8, 24.7, 28.6).
Work plan_tiles(int tokens, int64_t rows, int64_t wide, int64_t depth, int64_t most)
{
    Work w{};
    w.tokens = tokens;
    const int64_t tiles_k = up(wide, kTileRows), tiles = tiles_k * up(rows, tokens), iterations = up(depth, kDepth);
    const int64_t limit = int64_t(1) << 31;
    w.fits = tiles < limit && tiles < limit / iterations;
    if (!w.fits)
        return w;
    int64_t cut_steps = kChain;
    if (tiles * up(iterations, kChain) < 2 * most) {
        cut_steps = tiles * iterations / (2 * most);
        cut_steps = cut_steps < kShortChain ? kShortChain : cut_steps;
    }
    const int64_t cut_units = tiles * up(iterations, cut_steps), cut_pairs = cut_units < most ? cut_units : most;
    const int64_t run = up(cut_units, cut_pairs) * cut_steps, share = up(tiles * iterations, cut_pairs);
    const int64_t parts = cut_pairs + (tiles < cut_pairs ? tiles : cut_pairs);
    const int64_t step = tokens == 192 ? 448 : tokens == 128 ? 360 : 320;
    const int64_t whole = up(tiles, most) * iterations * step;
    const int64_t cut = (run < share ? run : share) * step + 4200 + parts * tokens * 2 / 3 + (2 * cut_pairs > most ? 2500 : 0);
    w.whole = whole <= cut;
    w.cost = w.whole ? whole : cut;
    w.tiles_k = (uint32_t)tiles_k;
    w.tiles = (uint32_t)tiles;
    w.iterations = (uint32_t)iterations;
    w.chain_steps = (uint32_t)(w.whole ? kChain : cut_steps);
    w.chains = (uint32_t)up(iterations, w.chain_steps);
    w.units = w.tiles * w.chains;
    w.pairs = (uint32_t)(!w.whole ? cut_pairs : tiles < most ? tiles : most);
    // Weights of five to eight steps stay in shared memory while a pair walks the tokens, where it has tiles enough of the same
    // rows (1024 to 4096, brought anew for each tile or kept: 2048 tokens 14.0, 14.5 us, 4608 23.5, 22.9, 8192 39.1, 36.3, 16384 74.3, 68.6;
    // with four steps, 512 to 2048, 16384 tokens: 35.7, 38.0: what it takes to store the result).
    w.stay = tokens == 192 && w.whole && iterations > kStaySteps / 2 && iterations <= kStaySteps && tiles >= 4 * most;
    return w;
}

// Tokens of a tile, or 0 if there are too many tiles.  More than the rows fill never cost less.
int tile_tokens(int64_t rows, int64_t wide, int64_t depth)
{
    Work best{};
    for (int tokens : {64, 128, 192}) {
        const Work w = plan_tiles(tokens, rows, wide, depth, kMaxPairs);
        if (w.fits && (!best.fits || w.cost < best.cost))
            best = w;
    }
    return best.tokens;
}

// An upper bound for any number of pairs, never falling as rows rise: partial sums of the largest tile that so few
// rows take, for as many pairs as there are steps of the smallest.
size_t linear_workspace(int64_t rows, int64_t wide, int64_t depth)
{
    if (rows == 0 || wide == 0 || depth == 0)
        return kStatusBytes;
    const int64_t tokens = rows <= 64 ? 64 : rows <= 128 ? 128 : 192;
    const int64_t tiles = up(rows, 64) * up(wide, kTileRows);
    const int64_t pairs = tiles >= kMaxPairs || tiles * up(depth, kDepth) >= kMaxPairs ? kMaxPairs : tiles * up(depth, kDepth);
    return kStatusBytes + (size_t)(pairs * 2 * kTileRows * tokens) * sizeof(float);
}

template <int TOKENS, bool GRAD, bool STAY>
cudaError_t prepare_kernel(uint32_t* pairs)
{
    static std::atomic<uint32_t> cached[64] = {};
    int device = 0;
    cudaError_t err = cudaGetDevice(&device);
    if (err != cudaSuccess)
        return err;
    if (device < 0 || device >= 64)
        return cudaErrorInvalidDevice;
    *pairs = cached[device].load(std::memory_order_relaxed);
    if (*pairs == 0) {
        auto* kernel = fp8_linear_kernel<TOKENS, GRAD, STAY>;
        const size_t shared = Shape<TOKENS, STAY>::kSharedBytes;
        if ((err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared)) != cudaSuccess)
            return err;
        cudaLaunchConfig_t config = {};
        config.gridDim = dim3(2 * kMaxPairs);
        config.blockDim = dim3(kBlockThreads);
        config.dynamicSmemBytes = shared;
        cudaLaunchAttribute attribute;
        attribute.id = cudaLaunchAttributeClusterDimension;
        attribute.val.clusterDim.x = 2;
        attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
        config.attrs = &attribute;
        config.numAttrs = 1;
        int clusters = 0;
        if ((err = cudaOccupancyMaxActiveClusters(&clusters, kernel, &config)) != cudaSuccess)
            return err;
        if (clusters < 1)
            return cudaErrorLaunchOutOfResources;
        *pairs = clusters < kMaxPairs ? (uint32_t)clusters : kMaxPairs;
        cached[device].store(*pairs, std::memory_order_relaxed);
    }
    return cudaSuccess;
}

// Calls f(constant of the tile's tokens, constant of the direction, constant: the weights stay).
template <int N>
struct Number { static constexpr int value = N; };
template <typename F>
void with_shape(const Work& w, bool grad, F&& f)
{
    auto with_tokens = [&](auto g) {
        if (w.tokens == 64)
            f(Number<64>{}, g, Number<0>{});
        else if (w.tokens == 128)
            f(Number<128>{}, g, Number<0>{});
        else if (w.stay)
            f(Number<192>{}, g, Number<1>{});
        else
            f(Number<192>{}, g, Number<0>{});
    };
    if (grad)
        with_tokens(Number<1>{});
    else
        with_tokens(Number<0>{});
}

adasum_status_t describe_codes(CUtensorMap* map, const void* codes, int64_t width, int64_t rows, int box_rows)
{
    EncodeTiled encode = encode_tiled();
    if (!encode)
        return fail(ADASUM_ERR_CUDA, "the driver has no tensor map encoder");
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)width};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, unit[2] = {1, 1};
    const CUresult err = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, unit,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return err == CUDA_SUCCESS ? ADASUM_OK : fail(ADASUM_ERR_CUDA, "tensor map of packed codes: error %d", (int)err);
}

// Step bytes: [row block][column block][512 bytes].
adasum_status_t describe_steps(CUtensorMap* map, const void* steps, int64_t columns, int64_t rows)
{
    EncodeTiled encode = encode_tiled();
    if (!encode)
        return fail(ADASUM_ERR_CUDA, "the driver has no tensor map encoder");
    const cuuint64_t blocks = (cuuint64_t)fp8_blocks(columns);
    const cuuint64_t dims[3] = {kFp8StepBytes / 4, blocks, (cuuint64_t)fp8_blocks(rows)};
    const cuuint64_t strides[2] = {kFp8StepBytes, blocks * kFp8StepBytes};
    const cuuint32_t box[3] = {kFp8StepBytes / 4, 1, 1}, unit[3] = {1, 1, 1};
    const CUresult err = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(steps), dims, strides, box, unit,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return err == CUDA_SUCCESS ? ADASUM_OK : fail(ADASUM_ERR_CUDA, "tensor map of step bytes: error %d", (int)err);
}

adasum_status_t linear(const void* x, const void* w, int64_t rows, int64_t features, int64_t outputs, const void* bias,
                       adasum_dtype_t bias_dtype, void* out, int64_t out_stride, adasum_dtype_t out_dtype, void* workspace,
                       size_t workspace_bytes, bool grad, void* stream_ptr, int hand_over)
{
    clear_error();
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs))
        return fail(ADASUM_ERR_ARG, "rows = %lld, features = %lld, outputs = %lld out of range", (long long)rows,
                    (long long)features, (long long)outputs);
    if (!operator_dtype(out_dtype) || (bias && !operator_dtype(bias_dtype)))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d: fp32, fp16 or bf16", (int)out_dtype, (int)bias_dtype);
    const int64_t depth = grad ? outputs : features, wide = grad ? features : outputs;
    if (rows == 0 || wide == 0)
        return ADASUM_OK;
    if (depth > 0 && (!x || !w))
        return fail(ADASUM_ERR_NULL, "a packed matrix is NULL");
    if (!aligned_to(x, 16) || !aligned_to(w, 16))
        return fail(ADASUM_ERR_ARG, "a packed matrix is not 16-byte aligned");
    adasum_status_t status = check_matrix(grad ? "dx" : "y", out, out_stride, wide, out_dtype);
    if (status != ADASUM_OK)
        return status;
    if (bias && !aligned_to(bias, operator_bytes(bias_dtype)))
        return fail(ADASUM_ERR_ARG, "bias is not aligned to its element size");
    const int tokens = depth > 0 ? tile_tokens(rows, wide, depth) : 64;
    if (tokens == 0)
        return fail(ADASUM_ERR_ARG, "%lld x %lld x %lld is too large", (long long)rows, (long long)features, (long long)outputs);
    const size_t need = linear_workspace(rows, wide, depth);
    if (!workspace || workspace_bytes < need)
        return fail(ADASUM_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace ? workspace_bytes : (size_t)0, need);
    if (!aligned_to(workspace, 256))
        return fail(ADASUM_ERR_ARG, "workspace is not 256-byte aligned");
    const size_t out_bytes = matrix_span(rows, wide, out_stride, operator_bytes(out_dtype));
    const size_t x_bytes = fp8_bytes(rows, depth), w_bytes = fp8_bytes(outputs, features);
    const size_t bias_bytes = bias ? (size_t)(outputs * operator_bytes(bias_dtype)) : 0;
    if (spans_overlap(out, out_bytes, x, x_bytes) || spans_overlap(out, out_bytes, w, w_bytes) ||
        spans_overlap(out, out_bytes, bias, bias_bytes) || spans_overlap(out, out_bytes, workspace, need) ||
        spans_overlap(workspace, need, x, x_bytes) || spans_overlap(workspace, need, w, w_bytes) ||
        spans_overlap(workspace, need, bias, bias_bytes))
        return fail(ADASUM_ERR_ARG, "the output or the workspace overlaps an input or each other");

    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    LinearArgs a{};
    a.rows = rows;
    a.wide = wide;
    a.bias = bias;
    a.bias_dtype = (int)bias_dtype;
    a.out = out;
    a.out_stride = out_stride;
    a.out_dtype = (int)out_dtype;
    a.status = static_cast<int*>(workspace);
    a.pairs_aligned = wide % 2 == 0 && out_stride % 2 == 0 && aligned_to(out, 2 * operator_bytes(out_dtype));
    if (depth == 0) {
        const uint64_t elements = (uint64_t)rows * (uint64_t)wide, blocks = (elements + 255) / 256;
        if (blocks > 0x7fffffffu)
            return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)rows, (long long)wide);
        fp8_bias_kernel<<<(unsigned)blocks, 256, 0, stream>>>(a, row_divider(wide), elements);
        ADASUM_CUDA_CHECK(cudaGetLastError());
        return ADASUM_OK;
    }
    uint32_t most = 0;
    cudaError_t err = cudaSuccess;
    Work l = plan_tiles(tokens, rows, wide, depth, kMaxPairs);
    auto prepare = [&](auto t, auto g, auto s) {
        err = prepare_kernel<decltype(t)::value, decltype(g)::value != 0, decltype(s)::value != 0>(&most);
    };
    with_shape(l, grad, prepare);
    ADASUM_CUDA_CHECK(err);
    if (most != kMaxPairs) {
        l = plan_tiles(tokens, rows, wide, depth, most);
        with_shape(l, grad, prepare);
        ADASUM_CUDA_CHECK(err);
    }
    const uint8_t* token_codes = static_cast<const uint8_t*>(x);
    const uint8_t* weight_codes = static_cast<const uint8_t*>(w);
    CUtensorMap token_map, weight_map, token_step_map, weight_step_map;
    status = describe_codes(&token_map, token_codes, fp8_width(depth), rows, tokens / 2);
    if (status == ADASUM_OK)
        status = describe_codes(&weight_map, weight_codes, fp8_width(features), outputs, kHalf);
    if (status == ADASUM_OK)
        status = describe_steps(&token_step_map, token_codes + rows * fp8_width(depth), depth, rows);
    if (status == ADASUM_OK)
        status = describe_steps(&weight_step_map, weight_codes + outputs * fp8_width(features), features, outputs);
    if (status != ADASUM_OK)
        return status;
    a.tiles_k = l.tiles_k;
    a.tiles = l.tiles;
    a.iterations = l.iterations;
    a.chain_steps = l.chain_steps;
    a.chains = l.chains;
    a.units = l.units;
    a.whole = l.whole;
    a.wait_cycles = hand_over == ADASUM_HAND_OVER_NONE ? kWaitCycles : kSelftestCycles;
    a.withheld = hand_over;
    a.slots = reinterpret_cast<float*>(static_cast<char*>(workspace) + kStatusBytes);
    profile_mark(stream, -1, 0, 0, true);
    with_shape(l, grad, [&](auto t, auto g, auto s) {
        constexpr int TOKENS = decltype(t)::value;
        constexpr bool STAY = decltype(s)::value != 0;
        err = launch_after(fp8_linear_kernel<TOKENS, decltype(g)::value != 0, STAY>, dim3(2 * l.pairs), kBlockThreads,
                           Shape<TOKENS, STAY>::kSharedBytes, stream, a, token_map, weight_map, token_step_map, weight_step_map);
    });
    ADASUM_CUDA_CHECK(err);
    profile_mark(stream, ADASUM_KERNEL_FP8_LINEAR, 0, 0, false);
    if (!l.whole) {
        const bool vec = aligned_to(out, 16) && out_stride % 4 == 0 && wide % 4 == 0;
        ADASUM_CUDA_CHECK(launch_after(fp8_join_kernel, dim3(l.tiles, (unsigned)up(2 * tokens, kJoinThreads / 32)), kJoinThreads, 0,
                                       stream, a, l.pairs, tokens, vec));
        profile_mark(stream, ADASUM_KERNEL_FP8_LINEAR, 1, 0, false);
    }
    return ADASUM_OK;
}

}  // namespace
}  // namespace adasum

extern "C" {

size_t adasum_fp8_linear_workspace_bytes(int64_t rows, int64_t features, int64_t outputs)
{
    using namespace adasum;
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs))
        return 0;
    const size_t forward = linear_workspace(rows, outputs, features), grad = linear_workspace(rows, features, outputs);
    return forward > grad ? forward : grad;
}

adasum_status_t adasum_fp8_linear(const void* x, const void* w, int64_t rows, int64_t features, int64_t outputs,
                                  const void* bias, adasum_dtype_t bias_dtype, void* y, int64_t y_stride,
                                  adasum_dtype_t out_dtype, void* workspace, size_t workspace_bytes, void* stream_ptr)
{
    return adasum::linear(x, w, rows, features, outputs, bias, bias_dtype, y, y_stride, out_dtype, workspace, workspace_bytes,
                          false, stream_ptr, ADASUM_HAND_OVER_NONE);
}

adasum_status_t adasum_fp8_linear_grad(const void* dy, const void* w, int64_t rows, int64_t features, int64_t outputs,
                                       void* dx, int64_t dx_stride, adasum_dtype_t out_dtype, void* workspace,
                                       size_t workspace_bytes, void* stream_ptr)
{
    return adasum::linear(dy, w, rows, features, outputs, nullptr, out_dtype, dx, dx_stride, out_dtype, workspace, workspace_bytes,
                          true, stream_ptr, ADASUM_HAND_OVER_NONE);
}

adasum_status_t adasum_fp8_linear_selftest(const void* x, const void* w, int64_t rows, int64_t features, int64_t outputs,
                                           void* y, int64_t y_stride, adasum_dtype_t out_dtype, void* workspace,
                                           size_t workspace_bytes, void* stream_ptr, int32_t hand_over)
{
    using namespace adasum;
    clear_error();
    if (hand_over < ADASUM_HAND_OVER_LANDED || hand_over > ADASUM_HAND_OVER_TAKEN || hand_over == ADASUM_HAND_OVER_ADDED ||
        hand_over == ADASUM_HAND_OVER_READY)
        return fail(ADASUM_ERR_ARG, "unknown hand-over %d", (int)hand_over);
    return linear(x, w, rows, features, outputs, nullptr, out_dtype, y, y_stride, out_dtype, workspace, workspace_bytes, false,
                  stream_ptr, hand_over);
}

adasum_status_t adasum_fp8_linear_status(const void* workspace, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    if (!workspace)
        return fail(ADASUM_ERR_NULL, "workspace is NULL");
    int words[kStatusBytes / sizeof(int)] = {};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    ADASUM_CUDA_CHECK(cudaMemcpyAsync(words, workspace, kStatusBytes, cudaMemcpyDeviceToHost, stream));
    ADASUM_CUDA_CHECK(cudaStreamSynchronize(stream));
    for (int i = 0; i < words[kStatusCount] && i < 2 * kMaxPairs; ++i)
        if (words[i] == ADASUM_DEVICE_TIMEOUT)
            return fail(ADASUM_ERR_TIMEOUT, "a bounded wait of block %d ran out", i);
    return ADASUM_OK;
}

}  // extern "C"
