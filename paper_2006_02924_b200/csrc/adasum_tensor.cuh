// What the products on the fifth-generation tensor cores (adasum_weight_grad.cu, adasum_fp8_linear.cu) share: barriers with
// bounded waits, tensor copies, hand-overs between a pair of blocks, tensor memory.
#pragma once

#include <cuda.h>

#include "adasum_operators.cuh"

namespace adasum {

// ---- device ------------------------------------------------------------------------------------------

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

__device__ __forceinline__ void load_sums(uint32_t address, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(address)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
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

// ---- work in equal runs ------------------------------------------------------------------------------
//
// The steps of all tiles are cut into units (sums that are formed in tensor memory), tile after tile, and the units into
// equal runs, one per pair of blocks.

__host__ __device__ inline uint32_t first_unit(uint32_t units, uint32_t pairs, uint32_t pair)
{
    return (uint32_t)((uint64_t)pair * units / pairs);
}
// The pair whose run holds a unit: the largest p with floor(p units / pairs) <= unit.
__host__ __device__ inline uint32_t pair_of_unit(uint32_t units, uint32_t pairs, uint32_t unit)
{
    return (uint32_t)((((uint64_t)unit + 1) * pairs - 1) / units);
}

// Where a role stands in its pair's run of units [begin, end).
//
// A run is the end of one tile, some whole tiles and the beginning of another.  They are walked in the order
// beginning, end, whole tiles: all runs are equally long, so at any time the pairs stand at one of two tokens
// (the beginnings at s, all others at the same distance from it, modulo the tokens), read the same rows of both
// matrices at the same time and find them in the L2's nearer half.
// The arguments hold `chains` (units of a tile), `chain_steps` (steps of a unit), `iterations` (steps of a tile) and
// `tiles_k` (tiles of a row of tiles).
struct Cursor {
    uint32_t unit, stop, chain, tile_k, tile_n, part;
    uint32_t begin, end;
    template <typename Args>
    __device__ __forceinline__ Cursor(const Args& a, uint32_t b, uint32_t e) : part(0), begin(b), end(e)
    {
        unit = max(b, e / a.chains * a.chains);          // the beginning of the last tile, if it is cut off
        stop = e;
        if (e / a.chains == b / a.chains)
            unit = stop;                                 // a run inside one tile is an "end" throughout
        enter(a);
    }
    template <typename Args>
    __device__ __forceinline__ void enter(const Args& a)
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
    template <typename Args>
    __device__ __forceinline__ bool last_of_share(const Args& a) const
    {
        return unit + 1 == stop || chain + 1 == a.chains;
    }
    template <typename Args>
    __device__ __forceinline__ uint32_t first_step(const Args& a) const { return chain * a.chain_steps; }
    template <typename Args>
    __device__ __forceinline__ uint32_t steps(const Args& a) const
    {
        return min(a.chain_steps, a.iterations - chain * a.chain_steps);
    }
    template <typename Args>
    __device__ __forceinline__ void advance(const Args& a)
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

// ---- host --------------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled()
{
    static std::atomic<EncodeTiled> cached{nullptr};
    if (!cached) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) == cudaSuccess &&
            found == cudaDriverEntryPointSuccess)
            cached = reinterpret_cast<EncodeTiled>(fn);
    }
    return cached;
}

}  // namespace adasum
