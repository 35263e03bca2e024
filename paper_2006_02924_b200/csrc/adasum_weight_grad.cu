// Gradients of a linear layer from the kept values of its input:
//
//     grad_weight[n][k] = scale * sum_t grad_out[t][n] * (kept x)[t][k]
//     grad_bias[n]      = scale * sum_t grad_out[t][n]
//
// A product D[k][n] = X^T G on the fifth-generation tensor cores, summed over the tokens t: 2 T N K
// operations on T (2 N + K) bytes, bound by the tensor cores from a few thousand tokens on.
//
// A pair of blocks (a cluster of two, on two neighbouring multiprocessors) owns a tile of 256 features x
// 256 outputs.  Each block brings 128 features of X and 128 outputs of G per step of 64 tokens, and its
// tensor core adds 128 features x 256 outputs: with both operands halved per block, shared memory and the
// L2 deliver half of what two separate blocks would need.  Both operands arrive with the summed index t
// as the slow one ("MN-major"), as they lie in memory; nothing is transposed.
//
//   G    one thread per block: bulk tensor copies of 64 outputs x 64 tokens, 128-byte swizzle, zeros
//        beyond the matrix; the codes of X (128 features x 64 tokens) come the same way, their step bytes,
//        whose rows have no alignment, by ordinary loads of one warp
//   X    two groups of four warps per block in turn: 16 codes at a time from shared memory to the 16-bit type
//        (exact: at most 7 significant bits times a power of two) and back to shared memory in the swizzled
//        form the tensor core reads.  (Codes loaded by these warps themselves, ahead of their use: 462 against 349 us then,
//        the fence that makes their stores visible to the tensor core waits for every load on its way.)
//   D    one thread of the pair's first block issues the multiplications; eight warps per block add the sums of
//        every 512 tokens from tensor memory into fp32 registers
//
// The last point is for precision: the tensor core truncates where it adds, and over thousands of tokens that
// adds up; 32 additions of 16 products each between roundings to nearest stay below the error of an fp32
// sum.  (256, 512 or 1024 tokens: 134, 128, 126 us for 16384 tokens of 1024 x 4096.)
// Tensor memory holds two such sums, so the next is formed while the previous one is read.
//
// The steps of all tiles, tile after tile, are cut into equal runs, one per pair, so every pair works to
// the end whatever the sizes are; a tile whose steps fall to several pairs is joined, in their order, by
// weight_grad_join_kernel.  The association of every sum is fixed by the sizes and
// the number of pairs that fit the device: results are deterministic.
//
// Every wait has a limit.  A thread whose wait runs out records it and goes on without waiting, but hands over and
// issues nothing more, so the waits that depend on it run out in turn and the launch ends, a few limits later;
// adasum_checkpoint_weight_grad_status reports it, and the block leaves NaN for all its shares of tiles, so that no caller
// takes a part of a sum for a gradient.  Before a block ends its copies have landed, and the pair's
// multiplications and their arrivals are done: a last commit says so, whatever happened before.  (Those two waits have
// limits as well; copies and multiplications need microseconds, so one that ran out means that the device itself is stuck.)
#include <cuda.h>

#include "adasum_operators.cuh"

namespace adasum {
namespace {

constexpr int kGroup = 32;                       // features that share a step byte
constexpr int kHalf = 128;                       // features and outputs that a block of the pair brings
constexpr int kTileSide = 256;                   // features and outputs of a pair's tile
constexpr int kDepth = 64;                       // tokens per step
// Steps that are summed in tensor memory; fp32 gradients take three steps for the same tokens, each of which truncates.
constexpr int kChain = 8, kChainPlanes = 4;
constexpr int kStages = 7;                       // steps of gradients, codes and step bytes that are on their way
constexpr int kDecoded = 3;                      // steps of decoded values
constexpr int kPanelBytes = kDepth * 128;        // 64 features or outputs x 64 tokens, two bytes each
constexpr int kOperandBytes = 2 * kPanelBytes;
constexpr int kCodeBytes = kDepth * kHalf;
constexpr int kStageBytes = kOperandBytes + kCodeBytes;          // gradients, then codes
constexpr int kSumWarps = 8;
constexpr int kCodeWarps = 4, kCodeGroups = 2;   // warps that decode a step; groups of them that take turns
constexpr int kFirstCodeWarp = kSumWarps, kCopyWarp = kFirstCodeWarp + kCodeWarps * kCodeGroups;
constexpr int kMultiplyWarp = kCopyWarp + 1, kMemoryWarp = kCopyWarp + 2, kStepWarp = kCopyWarp + 3;
constexpr int kBlockThreads = 32 * (kCopyWarp + 4);
constexpr size_t kSharedBytes = (size_t)kStages * kStageBytes + (size_t)kDecoded * kOperandBytes + 1024;   // + room to align to 1024
constexpr int kMaxPairs = 74;                    // 148 multiprocessors
constexpr int64_t kSlotFloats = (int64_t)kTileSide * kTileSide;
constexpr long long kWaitCycles = 2000000000;    // about a second (a real wait is microseconds): the clock counts pauses too
constexpr long long kSelftestCycles = 2000000;   // about a millisecond
constexpr int kLastWait = 4;                     // limits, for the last commit: other warps' waits may have to run out first

struct WeightGradArgs {
    const int8_t* codes;
    const uint8_t* steps;
    int64_t rows, features, width, outputs;
    float scale;
    void* weight;
    void* bias;
    int out_dtype;
    bool accumulate;
    bool cut;                // some tile falls to several pairs: the join runs
    // units of chain_steps steps, tile after tile (tiles of a column of outputs next to each other)
    uint32_t tiles_k, tiles, iterations, chain_steps, chains, units;
    int* status;             // one word per block
    long long wait_cycles;   // limit of a wait
    int withheld;            // hand-over that never completes (self-test), or ADASUM_HAND_OVER_NONE
    float* slots;            // [pair][first or last tile of its run][block][output][feature of the block]
    float* bias_slots;       // [pair + tile][256 outputs]: the pairs' shares of the tiles' parts of the bias gradient
};

__host__ __device__ inline uint32_t first_unit(uint32_t units, uint32_t pairs, uint32_t pair)
{
    return (uint32_t)((uint64_t)pair * units / pairs);
}
// The pair whose run holds a unit: the largest p with floor(p units / pairs) <= unit.
__host__ __device__ inline uint32_t pair_of_unit(uint32_t units, uint32_t pairs, uint32_t unit)
{
    return (uint32_t)((((uint64_t)unit + 1) * pairs - 1) / units);
}

__device__ __forceinline__ void write_gradient(const WeightGradArgs& a, void* dst, int64_t e, float sum)
{
    float y = sum * a.scale;
    if (a.accumulate)
        y += load_as_float(dst, a.out_dtype, e);
    store_from_float(dst, a.out_dtype, e, y);
}

// A thread's column of a tile: one feature, 128 consecutive outputs.  Typed loops: the sums live in registers,
// so every loop over them is unrolled, and a choice of type inside would be unrolled with it.
template <typename TO>
__device__ __forceinline__ void write_column(const WeightGradArgs& a, int64_t n, int64_t k, float (&sum)[128])
{
    TO* p = static_cast<TO*>(a.weight) + n * a.features + k;
    const int count = (int)min((int64_t)128, a.outputs - n);
    if (a.accumulate) {
        const TO* q = p;
#pragma unroll
        for (int i = 0; i < 128; ++i, q += a.features)
            sum[i] = fmaf(sum[i], a.scale, i < count ? load_one(q) : 0.0f);
    } else {
#pragma unroll
        for (int i = 0; i < 128; ++i)
            sum[i] *= a.scale;
    }
#pragma unroll
    for (int i = 0; i < 128; ++i, p += a.features)
        if (i < count)
            store_from_float(p, TypeCode<TO>::value, 0, sum[i]);
}

// ---- instructions --------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t shared_address(const void* p)
{
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
// Returns false if the barrier does not complete the phase within `cycles`.
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, long long cycles)
{
    long long began = 0;
    for (uint32_t spin = 0;; ++spin) {
        if (mbarrier_try_wait_parity(bar, parity))
            return true;
        if ((spin & 15) == 0) {                  // an attempt may itself pause for a while
            const long long now = clock64();
            if (spin == 0)
                began = now;
            else if (now - began > cycles)
                return false;
        }
    }
}
// Arrives on the same barrier of the pair's first block.  Block scope is enough: what is handed over lies in the
// arriving block's own shared (or tensor) memory, already visible to its tensor core by the proxy fence (or the
// tensor-memory fence) before; cluster scope costs a memory barrier per arrival (349 against 259 us).
__device__ __forceinline__ void arrive_at_first(uint32_t bar)
{
    asm volatile("{\n\t.reg .b32 remote;\n\tmapa.shared::cluster.u32 remote, %0, 0;\n\t"
                 "mbarrier.arrive.shared::cluster.b64 _, [remote];\n\t}" ::"r"(bar)
                 : "memory");
}
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Arrives on the barrier at this offset in both blocks once all multiplications issued so far are done.
__device__ __forceinline__ void commit_to_both(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}
// One lane of a converged warp.  (With a lane number instead, the compiler cannot see that one thread issues.)
__device__ __forceinline__ bool elected()
{
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
template <int REGS>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }

// Operand in shared memory with the summed index slow, 128-byte swizzle: rows of 64 features (outputs), one
// row per token; eight rows 1024 bytes, the next 64 features one panel further.
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t address)
{
    return (uint64_t)((address & 0x3ffffu) >> 4) | (uint64_t)(kPanelBytes >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

__device__ __forceinline__ void load_sums(uint32_t address, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(address)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// ---- the codes of a step --------------------------------------------------------------------------------

// Two pairs of codes to two words of the 16-bit type, in that type (the packed instructions handle two values
// and need no conversion at the end).
//
// bf16: a code's low seven bits l go into the last place of 128 + l, its sign bit b selects 128 + 128 b, and
// the difference is the code; both are exact, and so is the product with a power of two between 2^-126 and
// 2^121.
//
// fp16: code + 128 in the last place of 1024, 1152 taken off.  The step may be outside fp16's range while the
// product is inside, so it is multiplied in two factors, each at most 2^15 and the first at least 2^-14: the
// first product is exact or overflows only if the whole does; the second is the one rounding.
template <typename T>
struct Decoder;
template <>
struct Decoder<__nv_bfloat16> {
    __nv_bfloat162 step;
    __device__ __forceinline__ explicit Decoder(uint32_t byte)
    {
        const uint32_t w = byte * 0x00800080u;           // the exponent field of either half
        step = *reinterpret_cast<const __nv_bfloat162*>(&w);
    }
    __device__ __forceinline__ uint32_t pair(uint32_t packed, uint32_t selector) const
    {
        const uint32_t w = __byte_perm(packed, 0x43434343u, selector);
        const uint32_t low = w & 0xff7fff7fu, sign = w & 0xff80ff80u;
        const __nv_bfloat162 x = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&low),
                                                 *reinterpret_cast<const __nv_bfloat162*>(&sign)),
                                         step);
        return *reinterpret_cast<const uint32_t*>(&x);
    }
    __device__ __forceinline__ uint2 four(uint32_t packed) const
    {
        return make_uint2(pair(packed, 0x4140), pair(packed, 0x4342));
    }
};
template <>
struct Decoder<__half> {
    __half2 first, second;
    __device__ __forceinline__ explicit Decoder(uint32_t byte)
    {
        // 2^(byte - 127) = first * second; 255 (NaN) must stay NaN, 0 (beyond the matrix) be zero
        const int e = (int)byte - 127, a = max(-14, min(15, e)), b = max(-25, min(15, e - a));
        const float f = byte == 255u ? __uint_as_float(0x7fc00000u) : byte == 0u ? 0.0f : __uint_as_float((uint32_t)(a + 127) << 23);
        first = __float2half2_rn(f);
        second = __float2half2_rn(__uint_as_float((uint32_t)(b + 127) << 23));
    }
    __device__ __forceinline__ uint32_t pair(uint32_t biased, uint32_t selector) const
    {
        const uint32_t w = __byte_perm(biased, 0x64646464u, selector);
        const uint32_t offset = 0x64806480u;             // 1024 + 128
        const __half2 q = __hsub2(*reinterpret_cast<const __half2*>(&w), *reinterpret_cast<const __half2*>(&offset));
        const __half2 x = __hmul2(__hmul2(q, first), second);
        return *reinterpret_cast<const uint32_t*>(&x);
    }
    __device__ __forceinline__ uint2 four(uint32_t packed) const
    {
        const uint32_t biased = packed ^ 0x80808080u;
        return make_uint2(pair(biased, 0x4140), pair(biased, 0x4342));
    }
};

// Where a role stands in its pair's run of units [begin, end).
//
// A run is the end of one tile, some whole tiles and the beginning of another.  They are walked in the order
// beginning, end, whole tiles: all runs are equally long, so at any time the pairs stand at one of two tokens
// (the beginnings at s, all others at the same distance from it, modulo the tokens), read the same rows of both
// matrices at the same time and find them in the L2's nearer half.
struct Cursor {
    uint32_t unit, stop, chain, tile_k, tile_n, part;
    uint32_t begin, end;
    __device__ __forceinline__ Cursor(const WeightGradArgs& a, uint32_t b, uint32_t e) : part(0), begin(b), end(e)
    {
        unit = max(b, e / a.chains * a.chains);          // the beginning of the last tile, if it is cut off
        stop = e;
        if (e / a.chains == b / a.chains)
            unit = stop;                                 // a run inside one tile is an "end" throughout
        enter(a);
    }
    __device__ __forceinline__ void enter(const WeightGradArgs& a)
    {
        while (unit == stop && part < 3) {
            ++part;
            const uint32_t first_whole =
                end / a.chains == begin / a.chains ? end : (begin + a.chains - 1) / a.chains * a.chains;
            if (part == 1) {
                unit = begin;
                stop = min(end, first_whole);
            } else if (part == 2) {
                unit = min(end, first_whole);
                stop = max(unit, end / a.chains * a.chains);
            }
        }
        const uint32_t tile = unit / a.chains;
        chain = unit - tile * a.chains;
        tile_n = tile / a.tiles_k;
        tile_k = tile - tile_n * a.tiles_k;
    }
    __device__ __forceinline__ bool done() const { return part == 3; }
    // Is this the last unit of the pair's share of the tile?
    __device__ __forceinline__ bool last_of_share(const WeightGradArgs& a) const
    {
        return unit + 1 == stop || chain + 1 == a.chains;
    }
    __device__ __forceinline__ uint32_t first_step(const WeightGradArgs& a) const { return chain * a.chain_steps; }
    __device__ __forceinline__ uint32_t steps(const WeightGradArgs& a) const
    {
        return min(a.chain_steps, a.iterations - chain * a.chain_steps);
    }
    __device__ __forceinline__ void advance(const WeightGradArgs& a)
    {
        ++unit;
        if (unit == stop) {
            enter(a);
        } else if (++chain == a.chains) {
            chain = 0;
            if (++tile_k == a.tiles_k) {
                tile_k = 0;
                ++tile_n;
            }
        }
    }
};

// What a thread of the warps that sum leaves for its feature and outputs where a wait of its block ran out: NaN, over
// whatever it has left for any tile of the pair's run.  (Inlined, it costs the whole kernel 10 %.)
__device__ __noinline__ void leave_nan(const WeightGradArgs& a, uint32_t begin, uint32_t end, uint32_t pair, uint32_t rank,
                                       uint32_t thread)
{
    const float nan = __uint_as_float(0x7fc00000u);
    const int feature = 32 * ((thread >> 5) & 3) + (thread & 31), side = thread >> 7;
    uint32_t chain_begin = 0;
    bool fresh = true;
    for (Cursor c(a, begin, end); !c.done(); c.advance(a)) {
        if (fresh)
            chain_begin = c.chain;
        fresh = c.last_of_share(a);
        if (!fresh)
            continue;
        const int64_t k = (int64_t)c.tile_k * kTileSide + rank * kHalf + feature;
        const int64_t n = (int64_t)c.tile_n * kTileSide + side * kHalf;
        if (chain_begin == 0 && c.chain + 1 == a.chains) {
            for (int i = 0; i < kHalf && k < a.features && n + i < a.outputs; ++i)
                store_from_float(a.weight, a.out_dtype, (n + i) * a.features + k, nan);
        } else {
            float* dst = a.slots + (2 * pair + (c.part == 0 ? 1 : 0)) * kSlotFloats + (rank * kTileSide + side * kHalf) * kHalf + feature;
            for (int i = 0; i < kHalf; ++i)
                dst[i * kHalf] = nan;
        }
        if (a.bias && thread < kHalf) {
            const int output = rank * kHalf + thread;
            const int64_t m = (int64_t)c.tile_n * kTileSide + output;
            if (a.cut)
                a.bias_slots[(int64_t)(pair + c.tile_n * a.tiles_k + c.tile_k) * kTileSide + output] = nan;
            else if (c.tile_k == 0 && m < a.outputs)
                store_from_float(a.bias, a.out_dtype, m, nan);
        }
    }
}

// A position in a ring of N stages and the parity of its current round.
template <int N>
struct Ring {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void advance()
    {
        if (++stage == N) {
            stage = 0;
            phase ^= 1;
        }
    }
};

// Step bytes of one row (token) for the block's 128 features, zeros beyond the matrix.
__device__ __forceinline__ uint32_t load_steps(const uint8_t* steps, int64_t groups, int64_t rows, int64_t row, int64_t group)
{
    if (row >= rows || group >= groups)
        return 0;
    const uint8_t* p = steps + row * groups + group;
    if ((groups & 3) == 0)               // every row starts on a word: the table itself does too
        return __ldg(reinterpret_cast<const uint32_t*>(p));
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (group + i < groups)
            w |= (uint32_t)__ldg(p + i) << (8 * i);
    return w;
}

// ---- kernel ---------------------------------------------------------------------------------------------
//
// 16384 tokens, 1024 features, 4096 outputs, bf16 to fp32: 115 us, and the join 10 us (1.07 PFLOP/s together; with the bias
// 138 us).  Bound by shared memory: a step of 64 tokens moves 80 KB through it, 640 cycles, for 512 cycles of
// multiplications.  fp32 gradients: 350 us for the three products after 100 us (6.7 TB/s) that lay them out.
//
// T: 16-bit type of both operands.  PLANES: 1, or 3 for fp32 gradients, which arrive as three bf16 matrices
// that add up to them; a step then is one plane of one block of tokens, planes fastest, the smallest first: what is added
// while a sum is small is truncated at its size (64 tokens 3.9e-7 -> 0.6e-7 of the norm, 333 tokens 3.3e-7 -> 2.5e-7).
// Warps 0 .. 7 sum, 8 .. 15 decode, 16 copies, 17 multiplies (first block only), 18 owns the tensor memory,
// 19 loads step bytes.
// Registers: 256 x 152 + 256 x 64 + 128 x 48 = 640 x 96.
template <typename T, int PLANES, bool BIAS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kBlockThreads, 1)
weight_grad_kernel(const __grid_constant__ WeightGradArgs a, const __grid_constant__ CUtensorMap grad_map,
                   const __grid_constant__ CUtensorMap code_map)
{
    extern __shared__ __align__(1024) unsigned char dynamic_shared[];
    // landed: this block's gradients, codes and step bytes of a step are there; multiplied: the tensor cores
    // are done with the step; added (BIAS): the sum warps are done with its gradients.  ready (first block):
    // both blocks' decoded values are there, and their gradients.
    // formed: a sum in tensor memory is complete; taken (first block): it has been read by both blocks.
    // finished: so are all multiplications that were ever issued.  nowhere: what threads that gave up arrive on.
    __shared__ __align__(8) unsigned long long landed[kStages], multiplied[kStages], added[kStages], ready[kDecoded],
        formed[2], taken[2], finished, nowhere[kDecoded];
    __shared__ uint32_t step_words[kStages][kDepth];         // four step bytes per token
    __shared__ uint32_t tensor_memory_slot;
    // Some wait of this block ran out.  The other block needs no word of it: a thread that acts for its warp stops, so the
    // other block's waits run out too; one that does not can only have spoilt this block's decoded values.
    __shared__ volatile uint32_t gave_up;
    __shared__ float bias_part[4][kHalf];

    start_next_kernel();             // the join; it waits for this kernel's end by itself
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t unit_begin = first_unit(a.units, pairs, pair), unit_end = first_unit(a.units, pairs, pair + 1);
    const uint32_t stage0 = (shared_address(dynamic_shared) + 1023u) & ~1023u;
    const uint32_t decoded0 = stage0 + kStages * kStageBytes;
    const uint32_t landed0 = shared_address(landed), ready0 = shared_address(ready);
    const uint32_t multiplied0 = shared_address(multiplied), added0 = shared_address(added);
    const uint32_t formed0 = shared_address(formed), taken0 = shared_address(taken);
    const uint32_t finished0 = shared_address(&finished), nowhere0 = shared_address(nowhere);

    if (threadIdx.x == 0) {
        a.status[blockIdx.x] = 0;
        gave_up = 0;
        // a barrier that expects one arrival too many never completes a phase
        auto init = [&](uint32_t bar, uint32_t count, int hand_over) { barrier_init(bar, count + (a.withheld == hand_over)); };
        for (int s = 0; s < kStages; ++s) {
            init(landed0 + 8 * s, 2, ADASUM_HAND_OVER_LANDED);
            init(multiplied0 + 8 * s, 1, ADASUM_HAND_OVER_MULTIPLIED);
            init(added0 + 8 * s, kSumWarps, ADASUM_HAND_OVER_ADDED);
        }
        for (int s = 0; s < kDecoded; ++s)
            init(ready0 + 8 * s, 2 * kCodeWarps, ADASUM_HAND_OVER_READY);
        for (int s = 0; s < 2; ++s) {
            init(formed0 + 8 * s, 1, ADASUM_HAND_OVER_FORMED);
            init(taken0 + 8 * s, 2 * kSumWarps, ADASUM_HAND_OVER_TAKEN);
        }
        barrier_init(finished0, 1);
        for (int s = 0; s < kDecoded; ++s)
            barrier_init(nowhere0 + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMemoryWarp) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
            shared_address(&tensor_memory_slot)));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (warp == kCopyWarp && lane == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&grad_map) : "memory");
        if (a.width > 0)
            asm volatile("prefetch.tensormap [%0];" ::"l"(&code_map) : "memory");
    }
    __syncthreads();
    cluster_barrier();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tensor_memory = tensor_memory_slot;

    // After a wait of this thread ran out it neither waits nor acts for its warp (arrives, multiplies, commits) any more.
    // The hand-overs to the thread that multiplies are turned aside rather than left out: a second condition beside
    // the lane's number cost 1 %, whole warps in step (a vote per wait) 7 % of the product's time.
    bool waiting = true, arrives = lane == 0;
    uint32_t ready_at = ready0, taken_at = taken0;
    auto wait_up_to = [&](uint32_t bar, uint32_t parity, long long cycles) {
        if (waiting && !wait_phase(bar, parity, cycles)) {
            waiting = arrives = false;
            ready_at = taken_at = nowhere0;
            gave_up = 1;
            a.status[blockIdx.x] = ADASUM_DEVICE_TIMEOUT;
        }
    };
    auto wait = [&](uint32_t bar, uint32_t parity) { wait_up_to(bar, parity, a.wait_cycles); };

    if (warp < kSumWarps) {
        // ---- sums: warp w reads tensor-memory lanes 32 (w % 4) .. + 31 (features), outputs 128 (w / 4) .. + 127
        more_registers<152>();
        const int quarter = warp & 3, side = warp >> 2;
        float sum[128];
        float bias_sum[2] = {0.0f, 0.0f};
        Ring<kStages> ring;
        uint32_t count = 0, chain_begin = 0;
        bool fresh = true;                       // the next unit is the first of its tile's share
        for (Cursor c(a, unit_begin, unit_end); !c.done(); c.advance(a), ++count) {
            if (fresh) {
                fresh = false;
                chain_begin = c.chain;
                bias_sum[0] = bias_sum[1] = 0.0f;
#pragma unroll
                for (int i = 0; i < 128; ++i)
                    sum[i] = 0.0f;
            }
            if constexpr (BIAS) {
                // this block's 128 outputs: thread = two outputs, 16 of a step's 64 tokens.  Summed per
                // unit, like the products.  Where the join runs anyway, the tiles of a column of outputs share
                // the work: each adds up every tiles_k-th step, so that none is slower than the others.
                const uint32_t steps = c.steps(a);
                const uint32_t sharers = a.cut ? a.tiles_k : 1;
                // steps until this tile's next one; never, for the tiles that leave the bias to the first
                uint32_t to_mine = a.cut ? (c.tile_k + sharers - c.first_step(a) % sharers) % sharers : c.tile_k == 0 ? 0 : ~0u;
                const int output = 2 * (threadIdx.x & 63), part = threadIdx.x >> 6;
                float unit_sum[2] = {0.0f, 0.0f};
                for (uint32_t s = 0; s < steps; ++s) {
                    wait(landed0 + 8 * ring.stage, ring.phase);
                    if (to_mine-- == 0) {
                        to_mine = sharers - 1;
                        const uint32_t panel = stage0 + ring.stage * kStageBytes + (output >> 6) * kPanelBytes;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int row = part * 16 + i;
                            uint32_t w;
                            asm volatile("ld.shared.b32 %0, [%1];"
                                         : "=r"(w)
                                         : "r"(panel + row * 128 + ((((output & 63) >> 3) ^ (row & 7)) << 4) +
                                               (output & 7) * 2));
                            if constexpr (__is_same(T, __half)) {
                                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
                                unit_sum[0] += f.x;
                                unit_sum[1] += f.y;
                            } else {
                                unit_sum[0] += __uint_as_float(w << 16);
                                unit_sum[1] += __uint_as_float(w & 0xffff0000u);
                            }
                        }
                    }
                    __syncwarp();
                    if (arrives)
                        mbarrier_arrive(added0 + 8 * ring.stage);
                    ring.advance();
                }
                bias_sum[0] += unit_sum[0];
                bias_sum[1] += unit_sum[1];
            }
            wait(formed0 + 8 * (count & 1), (count >> 1) & 1);
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t source = tensor_memory + (count & 1) * 256 + side * 128 + ((uint32_t)(32 * quarter) << 16);
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                uint32_t r[16];
                load_sums(source + 16 * g, r);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    sum[16 * g + i] += __uint_as_float(r[i]);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0)
                arrive_at_first(taken_at + 8 * (count & 1));

            if (!c.last_of_share(a))
                continue;
            fresh = true;
            // ---- the pair's last unit of this tile: the result, or this pair's part of it
            const bool whole = chain_begin == 0 && c.chain + 1 == a.chains;
            const uint32_t slot = 2 * pair + (c.part == 0 ? 1 : 0);
            const int feature = 32 * quarter + lane;
            if (whole) {
                const int64_t k = (int64_t)c.tile_k * kTileSide + rank * kHalf + feature;
                const int64_t n = (int64_t)c.tile_n * kTileSide + side * kHalf;
                if (k < a.features) {
                    if (a.out_dtype == ADASUM_F32)
                        write_column<float>(a, n, k, sum);
                    else if (a.out_dtype == ADASUM_F16)
                        write_column<__half>(a, n, k, sum);
                    else
                        write_column<__nv_bfloat16>(a, n, k, sum);
                }
            } else {
                float* dst = a.slots + slot * kSlotFloats + (rank * kTileSide + side * kHalf) * kHalf + feature;
#pragma unroll
                for (int i = 0; i < 128; ++i)
                    dst[i * kHalf] = sum[i];
            }
            if constexpr (BIAS) {
                const int output = 2 * (threadIdx.x & 63), part = threadIdx.x >> 6;
                bias_part[part][output] = bias_sum[0];
                bias_part[part][output + 1] = bias_sum[1];
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (threadIdx.x < kHalf) {
                    const float total = (bias_part[0][threadIdx.x] + bias_part[1][threadIdx.x]) +
                                        (bias_part[2][threadIdx.x] + bias_part[3][threadIdx.x]);
                    const int output = rank * kHalf + threadIdx.x;
                    const int64_t n = (int64_t)c.tile_n * kTileSide + output;
                    if (a.cut)
                        a.bias_slots[(int64_t)(pair + c.tile_n * a.tiles_k + c.tile_k) * kTileSide + output] = total;
                    else if (c.tile_k == 0 && n < a.outputs)
                        write_gradient(a, a.bias, n, total);
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
            }
        }
        if (gave_up != 0)
            leave_nan(a, unit_begin, unit_end, pair, rank, threadIdx.x);
        // The last commit arrives in both blocks, and each waits for its own: in this warp, which has just seen the last sum.
        if (warp == 0) {
            waiting = true;
            wait_up_to(finished0, 0, kLastWait * a.wait_cycles);
        }
    } else if (warp < kCopyWarp) {
        // ---- codes: a lane decodes 16 features of four rows (tokens).  Of eight neighbouring lanes four hold the
        // first panel's pieces of one row and four the second's of the row's neighbour: their reads, and then
        // both of their writes, fall on eight different groups of banks.
        fewer_registers<64>();
        const int piece = lane & 7, upper = piece >> 2;
        const int group = (warp - kFirstCodeWarp) / kCodeWarps;
        const int row0 = ((lane >> 3) + 4 * ((warp - kFirstCodeWarp) % kCodeWarps)) ^ upper;
        const uint32_t from = row0 * kHalf + ((piece ^ (row0 & 7)) << 4);
        const uint32_t to = upper * kPanelBytes + row0 * 128 + (((2 * (piece & 3)) ^ (row0 & 7)) << 4);
        Ring<kStages> ring, behind;              // behind: the step whose place among the decoded ones is taken next
        Ring<kDecoded> out;
        uint32_t taken_places = 0;               // the first kDecoded steps find theirs free
        int turn = 0;
        for (Cursor c(a, unit_begin, unit_end); !c.done(); c.advance(a)) {
            for (uint32_t steps = c.steps(a); steps > 0; --steps) {
                if (turn == group) {
                if (taken_places == kDecoded)
                    wait(multiplied0 + 8 * behind.stage, behind.phase);
                wait(landed0 + 8 * ring.stage, ring.phase);
                const uint32_t source = stage0 + ring.stage * kStageBytes + kOperandBytes + from;
                const uint32_t target = decoded0 + out.stage * kOperandBytes + to;
                uint4 codes[4];
                uint32_t words[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    codes[i] = load_shared_16B(source + 16 * i * kHalf);
                    words[i] = step_words[ring.stage][row0 + 16 * i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Decoder<T> decode((words[i] >> (8 * (piece >> 1))) & 0xffu);
                    const uint2 w0 = decode.four(codes[i].x), w1 = decode.four(codes[i].y);
                    const uint2 w2 = decode.four(codes[i].z), w3 = decode.four(codes[i].w);
                    store_shared_16B(target + 16 * i * 128, make_uint4(w0.x, w0.y, w1.x, w1.y));
                    store_shared_16B((target ^ 16) + 16 * i * 128, make_uint4(w2.x, w2.y, w3.x, w3.y));
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0)
                    arrive_at_first(ready_at + 8 * out.stage);
                }
                if (taken_places == kDecoded)
                    behind.advance();
                else
                    ++taken_places;
                if (++turn == kCodeGroups)
                    turn = 0;
                ring.advance();
                out.advance();
            }
        }
    } else {
        fewer_registers<48>();
        if (warp == kCopyWarp) {
            // ---- copies of this block's half of the gradients, and of the codes
            Ring<kStages> ring;
            uint32_t issued = 0;
            const uint32_t bytes = kOperandBytes + (a.width > 0 ? kCodeBytes : 0);
            for (Cursor c(a, unit_begin, unit_end); !c.done() && waiting; c.advance(a)) {
                const int n = (int)c.tile_n * kTileSide + (int)rank * kHalf, k = (int)c.tile_k * kTileSide + (int)rank * kHalf;
                const uint32_t end = c.first_step(a) + c.steps(a);
                for (uint32_t step = c.first_step(a); step < end; ++step) {
                    const uint32_t bar = landed0 + 8 * ring.stage;
                    wait(multiplied0 + 8 * ring.stage, ring.phase ^ 1);
                    if constexpr (BIAS)
                        wait(added0 + 8 * ring.stage, ring.phase ^ 1);
                    waiting = __all_sync(0xffffffffu, waiting);
                    if (!waiting)
                        break;
                    const uint32_t dst = stage0 + ring.stage * kStageBytes;
                    const int t = (int)(step / PLANES) * kDepth, plane = PLANES - 1 - (int)(step % PLANES);
                    if (elected()) {
                        expect_bytes(bar, bytes);
                        copy_box(dst, &grad_map, n, t, plane, bar);
                        copy_box(dst + kPanelBytes, &grad_map, n + 64, t, plane, bar);
                        if (a.width > 0)
                            copy_box(dst + kOperandBytes, &code_map, k, t, bar);
                    }
                    __syncwarp();
                    ++issued;
                    ring.advance();
                }
            }
            // nothing may still be on its way into shared memory when the block ends
            waiting = true;
            for (uint32_t back = min(issued, (uint32_t)kStages); back > 0; --back) {
                const uint32_t step = issued - back;
                wait(landed0 + 8 * (step % kStages), (step / kStages) & 1);
            }
        } else if (warp == kMultiplyWarp && rank == 0) {
            // ---- multiplications: fp32 sums, both operands of type T with the summed index slow, 256 x 256
            constexpr uint32_t kFormat = __is_same(T, __half) ? 0u : 1u;
            constexpr uint32_t kInstruction = (1u << 4) | (kFormat << 7) | (kFormat << 10) | (1u << 15) | (1u << 16) |
                                              ((kTileSide >> 3) << 17) | ((kTileSide >> 4) << 24);
            Ring<kStages> ring;
            Ring<kDecoded> in;
            uint32_t count = 0;
            for (Cursor c(a, unit_begin, unit_end); !c.done(); c.advance(a), ++count) {
                const uint32_t target = tensor_memory + (count & 1) * 256;
                wait(taken0 + 8 * (count & 1), ((count >> 1) & 1) ^ 1);
                uint32_t accumulate = 0;
                for (uint32_t steps = c.steps(a); steps > 0; --steps) {
                    wait(ready0 + 8 * in.stage, in.phase);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t x = operand_descriptor(decoded0 + in.stage * kOperandBytes);
                    const uint64_t g = operand_descriptor(stage0 + ring.stage * kStageBytes);
                    if (elected() && waiting) {
#pragma unroll
                        for (int s = 0; s < kDepth / 16; ++s) {
                            // 16 tokens are 2048 bytes further on: 128 in the descriptors' units
                            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                                         "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(target),
                                         "l"(x + 128 * s), "l"(g + 128 * s), "r"(kInstruction), "r"(s > 0 ? 1u : accumulate)
                                         : "memory");
                        }
                        commit_to_both(multiplied0 + 8 * ring.stage);
                        if (steps == 1)
                            commit_to_both(formed0 + 8 * (count & 1));
                    }
                    __syncwarp();
                    accumulate = 1;
                    ring.advance();
                    in.advance();
                }
            }
            if (elected())
                commit_to_both(finished0);
            __syncwarp();
        } else if (warp == kStepWarp) {
            // ---- step bytes: a lane loads two rows per step, kBatch steps ahead of their use
            constexpr int kBatch = 4;
            const int64_t groups = a.width / kGroup;
            uint32_t w[kBatch][2];
            Ring<kStages> ring;
            auto load = [&](const Cursor& c, uint32_t from) {
                const int64_t group = (int64_t)c.tile_k * (kTileSide / kGroup) + rank * (kHalf / kGroup);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    const int64_t t = (int64_t)((c.first_step(a) + from + j) / PLANES) * kDepth + lane;
                    w[j][0] = load_steps(a.steps, groups, a.rows, t, group);
                    w[j][1] = load_steps(a.steps, groups, a.rows, t + 32, group);
                }
            };
            Cursor c(a, unit_begin, unit_end);
            uint32_t from = 0;               // first step of the batch within the unit
            load(c, from);
            while (!c.done()) {
                uint32_t v[kBatch][2];
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    v[j][0] = w[j][0];
                    v[j][1] = w[j][1];
                }
                const int steps = (int)min((uint32_t)kBatch, c.steps(a) - from);
                from += kBatch;
                if (from >= c.steps(a)) {
                    from = 0;
                    c.advance(a);
                }
                if (!c.done())
                    load(c, from);
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    if (j < steps) {
                        wait(multiplied0 + 8 * ring.stage, ring.phase ^ 1);
                        step_words[ring.stage][lane] = v[j][0];
                        step_words[ring.stage][lane + 32] = v[j][1];
                        __syncwarp();
                        if (arrives)
                            mbarrier_arrive(landed0 + 8 * ring.stage);
                        ring.advance();
                    }
                }
            }
        }
        __syncwarp();
    }
    // Neither block may end, nor free its tensor memory, while the other still multiplies or arrives here: both have
    // waited for the last commit, the first block's copies of it included.
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    cluster_barrier();
    if (warp == kMemoryWarp)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tensor_memory) : "memory");
}

// Where some tile's units fell to several pairs: those tiles, and the bias gradient, the pairs' parts added in
// order.  grid.x = tiles, grid.y = parts of a tile's 2 x 256 rows of 128 features; one warp per row, four
// features per lane.  Parts of 256 KB from 74 pairs: 10 us, mostly from the L2.
constexpr int kJoinThreads = 256;
constexpr int kJoinParts = 2 * kTileSide / (kJoinThreads / 32);

__global__ void __launch_bounds__(kJoinThreads)
weight_grad_join_kernel(const __grid_constant__ WeightGradArgs a, uint32_t pairs, bool vec)
{
    wait_for_previous_kernel();
    const uint32_t tile = blockIdx.x;
    const uint32_t first = pair_of_unit(a.units, pairs, tile * a.chains);
    const uint32_t last = pair_of_unit(a.units, pairs, tile * a.chains + a.chains - 1);
    const uint32_t tile_k = tile % a.tiles_k, tile_n = tile / a.tiles_k;
    if (a.bias && tile_k == 0 && blockIdx.y == 0) {
        const int64_t n = (int64_t)tile_n * kTileSide + threadIdx.x;
        float total = 0.0f;
        for (uint32_t t = tile; t < tile + a.tiles_k; ++t) {
            const uint32_t to = pair_of_unit(a.units, pairs, t * a.chains + a.chains - 1);
            for (uint32_t pair = pair_of_unit(a.units, pairs, t * a.chains); pair <= to; ++pair)
                total += __ldcg(a.bias_slots + (int64_t)(pair + t) * kTileSide + threadIdx.x);
        }
        if (n < a.outputs)
            write_gradient(a, a.bias, n, total);
    }
    if (first == last)
        return;                      // written by the product itself
    // only the first pair's run can have started in an earlier tile
    const uint32_t first_slot = 2 * first + (tile == first_unit(a.units, pairs, first) / a.chains ? 0 : 1);
    auto slot_of = [&](uint32_t pair) { return pair == first ? first_slot : 2 * pair; };
    const int row = blockIdx.y * (kJoinThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    const float* source = a.slots + (int64_t)row * kHalf + 4 * lane;
    float sum[4] = {};
#pragma unroll 4
    for (uint32_t pair = first; pair <= last; ++pair) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(source + slot_of(pair) * kSlotFloats));
        sum[0] += v.x;
        sum[1] += v.y;
        sum[2] += v.z;
        sum[3] += v.w;
    }
    const int64_t n = (int64_t)tile_n * kTileSide + (row & (kTileSide - 1));
    const int64_t k = (int64_t)tile_k * kTileSide + (row / kTileSide) * kHalf + 4 * lane;
    if (n < a.outputs && k < a.features) {
        const int64_t e = n * a.features + k;
        if (vec) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sum[i] *= a.scale;
            if (a.accumulate)
                add_vector_as_float<4>(a.weight, a.out_dtype, e, sum);
            store_vector_from_float<4>(a.weight, a.out_dtype, e, sum);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k + i < a.features)
                    write_gradient(a, a.weight, e + i, sum[i]);
        }
    }
}

// ---- gradients that the tensor copies cannot read as they lie -------------------------------------------

// fp32: three bf16 matrices [plane][rows][pitch] that add up to the gradients: the upper 8 significant bits
// (truncated, so that nothing overflows), the next 8, the last 8.  16-bit types: rows moved to a pitch of
// whole 16 bytes.  One thread per eight outputs; HBM (fp32, 16384 x 4096: 670 MB in 100 us).
template <typename T>
__global__ void __launch_bounds__(256)
relay_gradients_kernel(const T* grad, int64_t stride, bool vec, int64_t rows, int64_t outputs, int64_t pitch, uint4* out,
                       RowDivider divider, uint64_t vectors)
{
    const uint64_t n = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= vectors)
        return;
    uint64_t row;
    uint32_t at;
    divide_row(divider, n, row, at);
    const int64_t column = (int64_t)at * 8;
    const int count = (int)min((int64_t)8, outputs - column);
    const int64_t place = ((int64_t)row * pitch + column) / 8;
    const T* p = grad + (int64_t)row * stride + column;
    if constexpr (sizeof(T) == 4) {
        float x[8];
        load_up_to_eight(p, vec, count, x);
        uint32_t w[3][4] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t part[3] = {__float_as_uint(x[i]) >> 16, 0, 0};
            if (isfinite(x[i])) {
                const float r1 = x[i] - __uint_as_float(part[0] << 16);
                part[1] = __float_as_uint(r1) >> 16;
                part[2] = __float_as_uint(r1 - __uint_as_float(part[1] << 16)) >> 16;
            } else if (isnan(x[i])) {
                part[0] |= 0x40;                         // a NaN whose bits are all in the lower half stays one
            }
#pragma unroll
            for (int j = 0; j < 3; ++j)
                w[j][i >> 1] |= part[j] << (16 * (i & 1));
        }
#pragma unroll
        for (int j = 0; j < 3; ++j)
            out[j * (rows * pitch / 8) + place] = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
    } else {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
        uint32_t w[4] = {};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count)
                w[i >> 1] |= (uint32_t)q[i] << (16 * (i & 1));
        out[place] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ---- host -------------------------------------------------------------------------------------------------

struct WorkLayout {
    uint32_t tiles_k, tiles, iterations, chain_steps, chains, units, pairs;
    int64_t pitch;
    size_t slots, bias_slots, gradients, total;
    bool fits;
};

// `pairs` here is the most that any device may use; the launch takes no more than are resident at once.
WorkLayout work_layout(int64_t rows, int64_t features, int64_t outputs, adasum_dtype_t dtype)
{
    auto up = [](int64_t x, int64_t to) { return (x + to - 1) / to * to; };
    WorkLayout l{};
    const int64_t planes = dtype == ADASUM_F32 ? 3 : 1;
    const int64_t tiles_k = features > 0 ? (features + kTileSide - 1) / kTileSide : 1;
    const int64_t tiles_n = (outputs + kTileSide - 1) / kTileSide;
    const int64_t iterations = (rows + kDepth - 1) / kDepth * planes;
    const int64_t chain_steps = planes > 1 ? kChainPlanes : kChain;
    const int64_t chains = (iterations + chain_steps - 1) / chain_steps;
    const int64_t limit = int64_t(1) << 31;
    l.fits = tiles_k * tiles_n < limit && iterations < limit && (chains == 0 || tiles_k * tiles_n < limit / chains);
    if (!l.fits)
        return l;
    l.tiles_k = (uint32_t)tiles_k;
    l.tiles = (uint32_t)(tiles_k * tiles_n);
    l.iterations = (uint32_t)iterations;
    l.chain_steps = (uint32_t)chain_steps;
    l.chains = (uint32_t)chains;
    l.units = (uint32_t)(l.tiles * chains);
    l.pairs = l.units < kMaxPairs ? l.units : kMaxPairs;
    l.pitch = up(outputs, 8);
    l.slots = 1024;                                    // the blocks' status words come first
    l.bias_slots = l.slots + (size_t)l.pairs * 2 * kSlotFloats * sizeof(float);
    l.gradients = l.bias_slots + (size_t)(l.pairs + l.tiles) * kTileSide * sizeof(float);
    l.total = l.gradients + (size_t)up(planes * rows * l.pitch * 2, 256);
    return l;
}

// Pairs that are resident at once.  A pair keeps to one group of multiprocessors, so groups with an odd number of
// them leave one without a partner: fewer than half the multiprocessors.  One pair too many would do its whole
// run after all others' (twice the time).
template <typename T, int PLANES, bool BIAS>
uint32_t resident_pairs()
{
    static uint32_t cached[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64)
        return 0;
    if (cached[device] == 0) {
        auto* kernel = weight_grad_kernel<T, PLANES, BIAS>;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSharedBytes) != cudaSuccess)
            return 0;
        cudaLaunchConfig_t config = {};
        config.gridDim = dim3(2 * kMaxPairs);
        config.blockDim = dim3(kBlockThreads);
        config.dynamicSmemBytes = kSharedBytes;
        cudaLaunchAttribute attribute;
        attribute.id = cudaLaunchAttributeClusterDimension;
        attribute.val.clusterDim.x = 2;
        attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
        config.attrs = &attribute;
        config.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &config) != cudaSuccess || clusters < 1)
            return 0;
        cached[device] = clusters < kMaxPairs ? (uint32_t)clusters : kMaxPairs;
    }
    return cached[device];
}
// For a call's type; which of the two kernels is asked makes no difference to the shape of its blocks.
uint32_t launch_pairs(const WorkLayout& l, adasum_dtype_t dtype, bool bias)
{
    uint32_t most = 0;
    if (dtype == ADASUM_F32)
        most = bias ? resident_pairs<__nv_bfloat16, 3, true>() : resident_pairs<__nv_bfloat16, 3, false>();
    else if (dtype == ADASUM_F16)
        most = bias ? resident_pairs<__half, 1, true>() : resident_pairs<__half, 1, false>();
    else
        most = bias ? resident_pairs<__nv_bfloat16, 1, true>() : resident_pairs<__nv_bfloat16, 1, false>();
    // Short sums are not cut: leaving and joining a tile's parts takes one more launch.  Whole against cut (us), with 8,
    // 16 and 24 steps: 16 tiles, bf16, 11.8/11.8, 15.1/16.1, 18.4/16.9; 8 tiles 13.4/13.5, 16.6/16.7, 20.0/17.5; one tile
    // 11.8/11.8, 15.0/13.9, 18.2/14.2; fp32 gradients with 15 and 18 steps: 8 tiles 17.2/15.8, 18.6/16.6, 16 tiles 17.4/17.2,
    // 18.7/20.4.  (Where the tiles nearly fill the device, whole would be better for longer: 64 tiles, 64 steps, 36/47.)
    if (l.tiles <= most && l.iterations <= 16)
        return l.tiles;
    return l.pairs < most ? l.pairs : most;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled()
{
    static EncodeTiled cached = nullptr;
    if (!cached) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) == cudaSuccess &&
            found == cudaDriverEntryPointSuccess)
            cached = reinterpret_cast<EncodeTiled>(fn);
    }
    return cached;
}

// The codes of a checkpoint: [rows][width] bytes.
adasum_status_t describe_codes(CUtensorMap* map, const void* codes, int64_t width, int64_t rows)
{
    EncodeTiled encode = encode_tiled();
    if (!encode)
        return fail(ADASUM_ERR_CUDA, "the driver has no tensor map encoder");
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)width};
    const cuuint32_t box[2] = {kHalf, kDepth}, unit[2] = {1, 1};
    const CUresult err = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(codes), dims, strides, box, unit,
                                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return err == CUDA_SUCCESS ? ADASUM_OK : fail(ADASUM_ERR_CUDA, "tensor map of the codes: error %d", (int)err);
}

adasum_status_t describe_gradients(CUtensorMap* map, const void* base, adasum_dtype_t type, int64_t outputs, int64_t rows,
                                   int64_t planes, int64_t pitch)
{
    EncodeTiled encode = encode_tiled();
    if (!encode)
        return fail(ADASUM_ERR_CUDA, "the driver has no tensor map encoder");
    const cuuint64_t dims[3] = {(cuuint64_t)outputs, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)(rows * pitch * 2)};
    const cuuint32_t box[3] = {64, kDepth, 1}, unit[3] = {1, 1, 1};
    const CUresult err =
        encode(map, type == ADASUM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
               const_cast<void*>(base), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return err == CUDA_SUCCESS ? ADASUM_OK : fail(ADASUM_ERR_CUDA, "tensor map of the gradients: error %d", (int)err);
}

template <typename T, int PLANES, bool BIAS>
cudaError_t launch_product(const WeightGradArgs& a, const CUtensorMap (&map)[2], uint32_t pairs, cudaStream_t stream)
{
    weight_grad_kernel<T, PLANES, BIAS><<<2 * pairs, kBlockThreads, kSharedBytes, stream>>>(a, map[0], map[1]);
    return cudaGetLastError();
}
template <typename T, int PLANES>
cudaError_t launch_product(const WeightGradArgs& a, const CUtensorMap (&map)[2], uint32_t pairs, cudaStream_t stream)
{
    return a.bias ? launch_product<T, PLANES, true>(a, map, pairs, stream)
                  : launch_product<T, PLANES, false>(a, map, pairs, stream);
}

template <typename T>
cudaError_t launch_relay(const void* grad, int64_t stride, int64_t rows, int64_t outputs, int64_t pitch, void* out,
                         cudaStream_t stream)
{
    const int64_t per_row = pitch / 8;
    const uint64_t vectors = (uint64_t)rows * (uint64_t)per_row, blocks = (vectors + 255) / 256;
    if (blocks > 0x7fffffffu)
        return cudaErrorInvalidValue;
    relay_gradients_kernel<T><<<(unsigned)blocks, 256, 0, stream>>>(
        static_cast<const T*>(grad), stride, rows_aligned(grad, stride, sizeof(T)), rows, outputs, pitch,
        static_cast<uint4*>(out), row_divider(per_row), vectors);
    return cudaGetLastError();
}

adasum_status_t weight_grad(const void* checkpoint, int64_t rows, int64_t features, const void* grad_out,
                            int64_t grad_out_stride, int64_t outputs, adasum_dtype_t dtype, float scale, void* grad_weight,
                            void* grad_bias, adasum_dtype_t grad_dtype, int32_t accumulate, void* workspace,
                            size_t workspace_bytes, void* stream_ptr, int hand_over)
{
    clear_error();
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs))
        return fail(ADASUM_ERR_ARG, "rows = %lld, features = %lld, outputs = %lld out of range", (long long)rows,
                    (long long)features, (long long)outputs);
    if (!operator_dtype(dtype) || !operator_dtype(grad_dtype))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d: fp32, fp16 or bf16", (int)dtype, (int)grad_dtype);
    if (outputs == 0 || (features == 0 && !grad_bias) || (rows == 0 && accumulate))
        return ADASUM_OK;
    if (rows > 0 && (!grad_out || (features > 0 && !checkpoint)))
        return fail(ADASUM_ERR_NULL, "checkpoint or grad_out is NULL");
    if (features > 0 && !grad_weight)
        return fail(ADASUM_ERR_NULL, "grad_weight is NULL");
    const int64_t eb = operator_bytes(dtype), gb = operator_bytes(grad_dtype);
    if (!aligned_to(checkpoint, 16))
        return fail(ADASUM_ERR_ARG, "checkpoint is not 16-byte aligned");
    if (!aligned_to(grad_out, eb) || !aligned_to(grad_weight, gb) || !aligned_to(grad_bias, gb))
        return fail(ADASUM_ERR_ARG, "grad_out, grad_weight or grad_bias is not aligned to its element size");
    if (rows > 0 && !stride_ok(grad_out_stride, outputs))
        return fail(ADASUM_ERR_ARG, "grad_out_stride %lld is shorter than a row or out of range",
                    (long long)grad_out_stride);
    const WorkLayout l = work_layout(rows, features, outputs, dtype);
    if (!l.fits)
        return fail(ADASUM_ERR_ARG, "%lld x %lld x %lld is too large", (long long)rows, (long long)features,
                    (long long)outputs);
    const size_t need = l.total;
    if (!workspace || workspace_bytes < need)
        return fail(ADASUM_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace ? workspace_bytes : (size_t)0,
                    need);
    if (!aligned_to(workspace, 256))
        return fail(ADASUM_ERR_ARG, "workspace is not 256-byte aligned");
    const size_t in_bytes = matrix_span(rows, outputs, grad_out_stride, eb);
    const size_t kept_bytes = adasum_checkpoint_bytes(rows, features);
    const size_t weight_bytes = (size_t)outputs * (size_t)features * (size_t)gb;
    const size_t bias_bytes = grad_bias ? (size_t)outputs * (size_t)gb : 0;
    const struct { const void* p; size_t bytes; } inputs[] = {{checkpoint, kept_bytes}, {grad_out, in_bytes}};
    for (const auto& in : inputs)
        if (spans_overlap(in.p, in.bytes, grad_weight, weight_bytes) || spans_overlap(in.p, in.bytes, grad_bias, bias_bytes) ||
            spans_overlap(in.p, in.bytes, workspace, need))
            return fail(ADASUM_ERR_ARG, "an input overlaps a gradient or the workspace");
    if (spans_overlap(grad_weight, weight_bytes, grad_bias, bias_bytes) ||
        spans_overlap(workspace, need, grad_weight, weight_bytes) || spans_overlap(workspace, need, grad_bias, bias_bytes))
        return fail(ADASUM_ERR_ARG, "grad_weight, grad_bias and workspace overlap");

    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    if (rows == 0) {                       // empty sums: zeros of any type are zero bytes
        if (weight_bytes)
            ADASUM_CUDA_CHECK(cudaMemsetAsync(grad_weight, 0, weight_bytes, stream));
        if (bias_bytes)
            ADASUM_CUDA_CHECK(cudaMemsetAsync(grad_bias, 0, bias_bytes, stream));
        return ADASUM_OK;
    }
    const uint32_t pairs = launch_pairs(l, dtype, grad_bias != nullptr);
    if (pairs == 0)
        return fail(ADASUM_ERR_CUDA, "no device that can run a pair of blocks");
    char* ws = static_cast<char*>(workspace);
    // 16-byte rows are copied as they lie; others, and fp32, are laid out in the workspace first
    const bool relay = dtype == ADASUM_F32 || !rows_aligned(grad_out, grad_out_stride, eb);
    const int64_t planes = dtype == ADASUM_F32 ? 3 : 1;
    CUtensorMap map[2] = {};               // gradients; codes, if there are any
    adasum_status_t described =
        describe_gradients(&map[0], relay ? ws + l.gradients : grad_out, dtype == ADASUM_F16 ? ADASUM_F16 : ADASUM_BF16,
                           outputs, rows, planes, relay ? l.pitch : grad_out_stride);
    if (described == ADASUM_OK && features > 0)
        described = describe_codes(&map[1], checkpoint, (features + kGroup - 1) / kGroup * kGroup, rows);
    if (described != ADASUM_OK)
        return described;
    WeightGradArgs a;
    a.rows = rows;
    a.features = features;
    a.width = (features + kGroup - 1) / kGroup * kGroup;
    a.codes = static_cast<const int8_t*>(checkpoint);
    a.steps = static_cast<const uint8_t*>(checkpoint) + rows * a.width;
    a.outputs = outputs;
    a.scale = scale;
    a.weight = grad_weight;
    a.bias = grad_bias;
    a.out_dtype = (int)grad_dtype;
    a.accumulate = accumulate != 0;
    a.cut = false;
    for (uint32_t p = 1; p < pairs && !a.cut; ++p)
        a.cut = first_unit(l.units, pairs, p) % l.chains != 0;
    a.tiles_k = l.tiles_k;
    a.tiles = l.tiles;
    a.iterations = l.iterations;
    a.chain_steps = l.chain_steps;
    a.chains = l.chains;
    a.units = l.units;
    a.status = reinterpret_cast<int*>(ws);
    a.wait_cycles = hand_over == ADASUM_HAND_OVER_NONE ? kWaitCycles : kSelftestCycles;
    a.withheld = hand_over;
    a.slots = reinterpret_cast<float*>(ws + l.slots);
    a.bias_slots = reinterpret_cast<float*>(ws + l.bias_slots);
    profile_mark(stream, -1, 0, 0, true);
    if (relay) {
        void* to = ws + l.gradients;
        ADASUM_CUDA_CHECK(dtype == ADASUM_F32
                              ? launch_relay<float>(grad_out, grad_out_stride, rows, outputs, l.pitch, to, stream)
                              : launch_relay<__half>(grad_out, grad_out_stride, rows, outputs, l.pitch, to, stream));
        profile_mark(stream, ADASUM_KERNEL_WEIGHT_GRAD, 0, 0, false);
    }
    if (dtype == ADASUM_F32)
        ADASUM_CUDA_CHECK((launch_product<__nv_bfloat16, 3>(a, map, pairs, stream)));
    else if (dtype == ADASUM_F16)
        ADASUM_CUDA_CHECK((launch_product<__half, 1>(a, map, pairs, stream)));
    else
        ADASUM_CUDA_CHECK((launch_product<__nv_bfloat16, 1>(a, map, pairs, stream)));
    profile_mark(stream, ADASUM_KERNEL_WEIGHT_GRAD, 1, 0, false);
    if (a.cut) {
        const bool vec = aligned_to(grad_weight, 16) && features % 4 == 0;
        ADASUM_CUDA_CHECK(launch_after(weight_grad_join_kernel, dim3(l.tiles, kJoinParts), kJoinThreads, 0, stream,
                                       a, pairs, vec));
        profile_mark(stream, ADASUM_KERNEL_WEIGHT_GRAD, 2, 0, false);
    }
    return ADASUM_OK;
}

}  // namespace
}  // namespace adasum

extern "C" {

size_t adasum_checkpoint_weight_grad_workspace_bytes(int64_t rows, int64_t features, int64_t outputs,
                                                     adasum_dtype_t dtype)
{
    using namespace adasum;
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs) || !operator_dtype(dtype))
        return 0;
    return work_layout(rows, features, outputs, dtype).total;
}

adasum_status_t adasum_checkpoint_weight_grad(const void* checkpoint, int64_t rows, int64_t features,
                                              const void* grad_out, int64_t grad_out_stride, int64_t outputs,
                                              adasum_dtype_t dtype, float scale, void* grad_weight, void* grad_bias,
                                              adasum_dtype_t grad_dtype, int32_t accumulate, void* workspace,
                                              size_t workspace_bytes, void* stream_ptr)
{
    return adasum::weight_grad(checkpoint, rows, features, grad_out, grad_out_stride, outputs, dtype, scale, grad_weight, grad_bias,
                               grad_dtype, accumulate, workspace, workspace_bytes, stream_ptr, ADASUM_HAND_OVER_NONE);
}

adasum_status_t adasum_checkpoint_weight_grad_selftest(const void* checkpoint, int64_t rows, int64_t features,
                                                       const void* grad_out, int64_t grad_out_stride, int64_t outputs,
                                                       adasum_dtype_t dtype, float scale, void* grad_weight,
                                                       void* grad_bias, adasum_dtype_t grad_dtype, int32_t accumulate,
                                                       void* workspace, size_t workspace_bytes, void* stream_ptr,
                                                       int32_t hand_over)
{
    using namespace adasum;
    clear_error();
    if (hand_over < ADASUM_HAND_OVER_LANDED || hand_over > ADASUM_HAND_OVER_TAKEN)
        return fail(ADASUM_ERR_ARG, "unknown hand-over %d", (int)hand_over);
    return weight_grad(checkpoint, rows, features, grad_out, grad_out_stride, outputs, dtype, scale, grad_weight, grad_bias,
                       grad_dtype, accumulate, workspace, workspace_bytes, stream_ptr, hand_over);
}

adasum_status_t adasum_checkpoint_weight_grad_status(int64_t rows, int64_t features, int64_t outputs,
                                                     adasum_dtype_t dtype, const void* workspace, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    if (!workspace)
        return fail(ADASUM_ERR_NULL, "workspace is NULL");
    if (!extent_ok(rows) || !extent_ok(features) || !extent_ok(outputs))
        return fail(ADASUM_ERR_ARG, "invalid sizes");
    if (!operator_dtype(dtype))
        return fail(ADASUM_ERR_DTYPE, "dtype %d is not fp32, fp16 or bf16", (int)dtype);
    const WorkLayout l = work_layout(rows, features, outputs, dtype);
    if (!l.fits)
        return fail(ADASUM_ERR_ARG, "invalid sizes");
    if (l.units == 0)
        return ADASUM_OK;                  // such a call launches no product
    const uint32_t blocks = 2 * launch_pairs(l, dtype, false);
    int words[2 * kMaxPairs] = {};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    ADASUM_CUDA_CHECK(cudaMemcpyAsync(words, workspace, blocks * sizeof(int), cudaMemcpyDeviceToHost, stream));
    ADASUM_CUDA_CHECK(cudaStreamSynchronize(stream));
    for (uint32_t i = 0; i < blocks; ++i)
        if (words[i] == ADASUM_DEVICE_TIMEOUT)
            return fail(ADASUM_ERR_TIMEOUT, "a bounded wait of block %u ran out", i);
    return ADASUM_OK;
}

}  // extern "C"
