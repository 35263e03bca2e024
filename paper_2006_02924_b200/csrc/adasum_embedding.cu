// Token embedding with scaling, and its gradient by sorted tokens.
//
// The gradient of row v is a sum over the tokens that point at v.  Three launches:
//
//   embedding_rank_kernel  (short lists) or embedding_sort_kernel (one cluster of blocks, radix sort): (row,
//                          position) pairs in the order of rows and, within a row, of positions.  The radix
//                          sort keeps eight multiprocessors busy for a while; the others write zeros into the
//                          whole gradient table meanwhile
//   embedding_sum_kernel   cuts the sorted list into tiles of equal length, whatever the rows' counts
//                          are; a block has all terms of its tile on their way into shared memory at once,
//                          adds them up run by run and writes the rows.  A run that goes on beyond the tile
//                          is followed for up to one more tile's length; of longer runs every tile leaves
//                          its share in the workspace.  After a ranking, more blocks of the same launch write
//                          zeros to the rows without a token: for a large vocabulary that is most of the
//                          traffic, and it hides the sums' latency
//   embedding_join_kernel  adds those shares, tile by tile in order, and writes the rows
//
// Every sum has a fixed association, so results are deterministic without atomics.
#include <cooperative_groups.h>

#include "adasum_operators.cuh"

namespace adasum {
namespace {

namespace cg = cooperative_groups;

// ---- lookup ------------------------------------------------------------------------------------------

template <typename Id>
__device__ __forceinline__ int64_t token_row(const Id* tokens, int64_t t, int64_t num_rows)
{
    const int64_t id = (int64_t)tokens[t];
    return id >= 0 && id < num_rows ? id : -1;
}

constexpr int kLookupRows = 4;             // tokens per thread

// A copy with a product: 32768 tokens in 30522 x 1024 fp32 rows to bf16 in 22 us (102 MB with each distinct row counted
// once: 4.6 TB/s).  Bound by the loads' latency: the vectors wait in fp32 registers (56 a thread), which leaves 47 % of the
// warps resident, and those stall for loads most of all; issue slots are 61 % used, the HBM less than half.
// VEC: every row of the table and of the output starts on 16 bytes and dim is a multiple of 8.
template <typename T, typename Id, bool VEC>
__global__ void __launch_bounds__(kStripThreads)
embedding_forward_kernel(const __grid_constant__ Strips s, const T* table, int64_t table_stride, int64_t num_rows,
                         const Id* tokens, float scale, void* out, int out_dtype, int64_t out_stride)
{
    const Place p = place_of<kLookupRows>(s);
    if (p.count <= 0)
        return;
    int64_t row[kLookupRows];
    float v[kLookupRows][8];
#pragma unroll
    for (int u = 0; u < kLookupRows; ++u) {
        const int64_t t = p.row0 + u * p.step;
        row[u] = t < s.rows ? token_row(tokens, t, num_rows) : -1;
    }
#pragma unroll
    for (int u = 0; u < kLookupRows; ++u) {
        if (VEC && row[u] >= 0) {
            load_eight(table + row[u] * table_stride + p.column, v[u]);
        } else {
            load_up_to_eight(table + row[u] * table_stride + p.column, false, row[u] >= 0 ? p.count : 0, v[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kLookupRows; ++u) {
        const int64_t t = p.row0 + u * p.step;
        if (t >= s.rows)
            break;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[u][i] = row[u] >= 0 ? v[u][i] * scale : 0.0f;
        const int64_t e = t * out_stride + p.column;
        if constexpr (VEC) {
            store_vector_from_float<8>(out, out_dtype, e, v[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < p.count)
                    store_from_float(out, out_dtype, e + i, v[u][i]);
        }
    }
}

// ---- sorting the tokens by row ---------------------------------------------------------------------------

constexpr int kSortCluster = 8;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kDigits = 256;
constexpr int kSortAhead = 4;              // rounds of 32 whose loads are issued together

// Lanes of the warp that are `mine` and hold the same digit.  (Eight votes rather than one match instruction,
// which all 32 warps of a block would queue for: sort of 200000 tokens 99 us against 117 us.)
__device__ __forceinline__ uint32_t lanes_with(uint32_t digit, bool mine)
{
    uint32_t same = __ballot_sync(0xffffffffu, mine);
#pragma unroll
    for (int bit = 1; bit < kDigits; bit *= 2) {
        const uint32_t set = __ballot_sync(0xffffffffu, (digit & bit) != 0);
        same &= (digit & bit) != 0 ? set : ~set;
    }
    return same;
}

// Table rows [0, num_rows) are the keys; tokens outside get the key num_rows and end up last.
// A stable radix sort, one byte per pass, least significant first.  Every warp of the cluster owns a
// contiguous run of the list, so "stable" is: by digit, then block, then warp, then place in the run.
// Up to kSortCluster * kSortWarps * 32 * kSortAhead items a lane's items and their ranks stay in registers
// from the counting to the placing; longer lists are read twice.
template <typename Id>
__device__ void sort_tokens(const Id* tokens, uint32_t n, uint32_t num_rows, int passes, uint2* a, uint2* b)
{
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ uint32_t next[kSortWarps][kDigits];      // per warp: count of a digit, then its place in the block's share
    __shared__ uint32_t quarter_count[4][kDigits];      // per eight warps
    __shared__ uint32_t block_count[kDigits], start[kDigits];
    __shared__ uint32_t warp_sum[kDigits / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int my_digit = threadIdx.x & (kDigits - 1), quarter = threadIdx.x / kDigits;
    const uint32_t rank = cluster.block_rank();
    const uint32_t warps = kSortCluster * kSortWarps;
    const uint32_t run = ((n + warps - 1) / warps + 31) / 32 * 32;        // whole rounds of 32
    const uint64_t begin64 = (uint64_t)(rank * kSortWarps + warp) * run;
    const uint32_t begin = begin64 < n ? (uint32_t)begin64 : n;
    const uint32_t end = n - begin < run ? n : begin + run;
    const bool once = run <= 32 * kSortAhead;

    for (int pass = 0; pass < passes; ++pass) {
        const uint2* src = (passes - pass) & 1 ? b : a;      // pass 0 reads the tokens themselves
        uint2* dst = (passes - 1 - pass) & 1 ? b : a;        // the last pass writes a
        const int shift = 8 * pass;
        uint2 it[kSortAhead];
        uint32_t place[kSortAhead];
        auto load = [&](uint32_t i0) {
#pragma unroll
            for (int j = 0; j < kSortAhead; ++j) {
                const uint32_t i = i0 + 32 * j + lane;
                it[j] = make_uint2(0, 0);
                if (i < end) {
                    if (pass == 0) {
                        const int64_t id = (int64_t)tokens[i];
                        it[j] = make_uint2(id >= 0 && id < (int64_t)num_rows ? (uint32_t)id : num_rows, i);
                    } else {
                        it[j] = __ldcg(src + i);
                    }
                }
            }
        };
        // places of the loaded items among the warp's items of the same digit
        auto count = [&](uint32_t i0) {
#pragma unroll
            for (int j = 0; j < kSortAhead; ++j) {
                if (i0 + 32 * j >= end)                      // the same for the whole warp
                    break;
                const bool mine = i0 + 32 * j + lane < end;
                const uint32_t digit = (it[j].x >> shift) & (kDigits - 1);
                const uint32_t same = lanes_with(digit, mine);
                if (mine)
                    place[j] = next[warp][digit] + __popc(same & ((1u << lane) - 1));
                __syncwarp();
                if (mine && lane == __ffs(same) - 1)
                    next[warp][digit] += __popc(same);
                __syncwarp();
            }
        };
        auto put = [&](uint32_t i0) {
#pragma unroll
            for (int j = 0; j < kSortAhead; ++j)
                if (i0 + 32 * j + lane < end)
                    dst[start[(it[j].x >> shift) & (kDigits - 1)] + place[j]] = it[j];
        };
        for (int d = lane; d < kDigits; d += 32)
            next[warp][d] = 0;
        __syncwarp();
        for (uint32_t i0 = begin; i0 < end; i0 += 32 * kSortAhead) {
            load(i0);
            count(i0);
        }
        __syncthreads();
        // counts -> places within the block's share of each digit
        uint32_t total = 0;
#pragma unroll
        for (int w = 0; w < kSortWarps / 4; ++w)
            total += next[quarter * (kSortWarps / 4) + w][my_digit];
        quarter_count[quarter][my_digit] = total;
        __syncthreads();
        uint32_t running = 0;
        for (int q = 0; q < quarter; ++q)
            running += quarter_count[q][my_digit];
#pragma unroll
        for (int w = 0; w < kSortWarps / 4; ++w) {
            const uint32_t c = next[quarter * (kSortWarps / 4) + w][my_digit];
            next[quarter * (kSortWarps / 4) + w][my_digit] = running;
            running += c;
        }
        if (quarter == 3)
            block_count[my_digit] = running;
        cluster.sync();
        // where the digit starts: all smaller digits, then the same digit in the blocks before this one
        uint32_t before = 0, everywhere = 0;
        if (quarter == 0) {
#pragma unroll
            for (uint32_t r = 0; r < kSortCluster; ++r) {
                const uint32_t c = cluster.map_shared_rank(block_count, r)[my_digit];
                before += r < rank ? c : 0;
                everywhere += c;
            }
        }
        uint32_t scan = everywhere;                      // inclusive over the warp's 32 digits
        for (int step = 1; step < 32; step *= 2) {
            const uint32_t other = __shfl_up_sync(0xffffffffu, scan, step);
            scan += lane >= step ? other : 0;
        }
        if (quarter == 0 && lane == 31)
            warp_sum[warp] = scan;
        __syncthreads();
        if (quarter == 0) {
            uint32_t first = scan - everywhere + before;
            for (int w = 0; w < warp; ++w)
                first += warp_sum[w];
            start[my_digit] = first;
        }
        __syncthreads();
        if (once) {
            // places so far are within the warp's run: add the warp's
#pragma unroll
            for (int j = 0; j < kSortAhead; ++j)
                if (begin + 32 * j + lane < end)
                    place[j] += next[warp][(it[j].x >> shift) & (kDigits - 1)];
            put(begin);
        } else {
            for (uint32_t i0 = begin; i0 < end; i0 += 32 * kSortAhead) {
                load(i0);
                count(i0);                               // from the warp's places on
                put(i0);
            }
        }
        cluster.sync();      // the pass's list is complete, and every block has read the counts
    }
}

// Blocks beyond the first cluster: zeros over `bytes` bytes at p (any alignment of 2), by bulk copies of a
// zeroed piece of shared memory.
constexpr int kZeroBytes = 8 * 1024;
__device__ void write_zeros(char* p, int64_t bytes, int64_t worker, int64_t workers)
{
    __shared__ __align__(16) uint4 zeros[kZeroBytes / 16];
    const int64_t head = min(bytes, (int64_t)((16 - (uintptr_t)p % 16) % 16));
    const int64_t body = (bytes - head) / 16 * 16, tail = bytes - head - body;
    for (int i = threadIdx.x; i < kZeroBytes / 16; i += blockDim.x)
        zeros[i] = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t source = static_cast<uint32_t>(__cvta_generic_to_shared(zeros));
        for (int64_t at = worker * kZeroBytes; at < body; at += workers * kZeroBytes) {
            const uint32_t size = (uint32_t)min((int64_t)kZeroBytes, body - at);
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(p + head + at), "r"(source), "r"(size)
                         : "memory");
        }
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (worker == 0 && threadIdx.x < head / 2)
        reinterpret_cast<uint16_t*>(p)[threadIdx.x] = 0;
    if (worker == 0 && threadIdx.x < tail / 2)
        reinterpret_cast<uint16_t*>(p + bytes - tail)[threadIdx.x] = 0;
}

// Cluster 0 sorts; the others write zeros into the whole gradient table meanwhile.  125 MB of zeros take 22 us
// (5.7 TB/s); the sort alone takes 7 us for 16384 tokens and one pass, 19 us for 32768 and two, 95 us for 200000
// (its eight multiprocessors place 8 bytes per item into scattered 32-byte sectors).
template <typename Id>
__global__ void __cluster_dims__(kSortCluster, 1, 1) __launch_bounds__(kSortThreads, 1)
embedding_sort_kernel(const Id* tokens, uint32_t n, uint32_t num_rows, int passes, uint2* sorted, uint2* spare,
                      uint32_t* long_runs, char* table, int64_t table_bytes)
{
    start_next_kernel();
    if (blockIdx.x < kSortCluster) {
        if (blockIdx.x == 0 && threadIdx.x == 0)
            *long_runs = 0;
        sort_tokens(tokens, n, num_rows, passes, sorted, spare);
    } else {
        write_zeros(table, table_bytes, (int64_t)blockIdx.x - kSortCluster, (int64_t)gridDim.x - kSortCluster);
    }
}

// Short lists: an item's place is the number of items that come before it.  Every block holds all keys in shared
// memory; a warp counts for one item at a time.  n^2 comparisons, but spread over all multiprocessors and
// without the radix sort's chain of passes: 4608 tokens of 30522 rows 5 us against 11 us, bound by instruction issue
// (two per comparison).
//
// Up to one item per warp of a grid that covers the device (4736 on 148 multiprocessors); the second item costs 3 us at
// once.  Whole calls, ranked against sorted, with 4736, 4800 and 6144 tokens (us): added to 30522 x 1024 23.6/24.7,
// 26.3/24.4, 31.2/26.8; to 512 x 1024 22.7/25.1, 25.5/24.7, 24.6/22.0; written to 30522 x 64 19.5/18.3, 22.3/18.2, 25.6/18.7;
// to 2 x 1024 16.6/14.7, 19.4/14.8, 21.5/15.2.  Where there are many zeros to write (after a ranking beside the sums,
// otherwise beside the sort) ranking pays up to 6144: 30522 x 1024 33.8/39.8, 36.6/39.6, 41.4/41.7.
constexpr int kRankThreads = 1024;
constexpr int64_t kRankMost = 6144, kManyZeros = int64_t(32) << 20;

bool ranked(int64_t num_tokens, int64_t zero_bytes, int sms)
{
    const int64_t one_each = (int64_t)sms * (kRankThreads / 32);
    return num_tokens <= (zero_bytes >= kManyZeros || one_each > kRankMost ? kRankMost : one_each);
}

template <typename Id>
__global__ void __launch_bounds__(kRankThreads)
embedding_rank_kernel(const Id* tokens, uint32_t n, uint32_t num_rows, uint2* sorted, uint32_t* long_runs)
{
    extern __shared__ __align__(16) uint32_t keys[];         // padded to whole rounds with the largest key
    start_next_kernel();
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *long_runs = 0;
    const uint32_t padded = (n + 127) / 128 * 128;
    for (uint32_t i = threadIdx.x; i < padded; i += kRankThreads) {
        uint32_t key = 0xffffffffu;
        if (i < n) {
            const int64_t id = (int64_t)tokens[i];
            key = id >= 0 && id < (int64_t)num_rows ? (uint32_t)id : num_rows;
        }
        keys[i] = key;
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 31, warps = gridDim.x * (kRankThreads / 32);
    for (uint32_t i = blockIdx.x * (kRankThreads / 32) + (threadIdx.x >> 5); i < n; i += warps) {
        const uint32_t mine = keys[i];
        // an equal key comes before if its position does: count keys below `mine + 1` in the rounds before the
        // item's own, below `mine` in those after it, and by position in its own
        uint32_t before = 0;
        const uint32_t own = i / 128 * 128;
        auto count = [&](uint32_t from, uint32_t to, uint32_t limit) {
#pragma unroll 4
            for (uint32_t j0 = from; j0 < to; j0 += 128) {
                const uint4 k = *reinterpret_cast<const uint4*>(keys + j0 + 4 * lane);
                before += (k.x < limit) + (k.y < limit) + (k.z < limit) + (k.w < limit);
            }
        };
        count(0, own, mine + 1);
        count(own + 128, padded, mine);
        const uint32_t j = own + 4 * lane;
        const uint4 k = *reinterpret_cast<const uint4*>(keys + j);
        before += (k.x < mine + (j < i)) + (k.y < mine + (j + 1 < i)) + (k.z < mine + (j + 2 < i)) + (k.w < mine + (j + 3 < i));
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0)
            sorted[before] = make_uint2(mine, i);
    }
}

// ---- sums ------------------------------------------------------------------------------------------------

constexpr int kSumThreads = 128;
constexpr int kMaxTile = 16;

struct SumArgs {
    const uint2* sorted;
    uint32_t n, num_rows;
    int tile;                // entries per tile
    int64_t stride, dim;
    float scale;
    void* table;
    int table_dtype;
    bool table_vec, accumulate;
    uint32_t tiles;          // the first blocks of embedding_sum_kernel; those after them write zeros
    uint32_t zero_rows;      // rows per such block
    uint32_t* long_runs;     // how many there are, then the tiles in which they start (in no particular order)
    float* edges;            // [tile][0: the run that enters from before, 1: the run that goes on][dim]
};

// VE consecutive elements starting at column `column` of row `row` of the table.
template <int VE>
__device__ __forceinline__ void write_row(const SumArgs& a, uint32_t row, int64_t column, const float (&sum)[VE])
{
    const int64_t e = (int64_t)row * a.dim + column;
    float y[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i)
        y[i] = sum[i] * a.scale;
    if constexpr (VE > 1) {
        if (a.table_vec) {
            if (a.accumulate)
                add_vector_as_float<VE>(a.table, a.table_dtype, e, y);
            store_vector_from_float<VE>(a.table, a.table_dtype, e, y);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        if (a.accumulate)
            y[i] += load_as_float(a.table, a.table_dtype, e + i);
        store_from_float(a.table, a.table_dtype, e + i, y[i]);
    }
}

// First entry of the sorted list whose row is not below `row`: a warp narrows the range to a 32nd per step.
__device__ uint32_t first_entry(const SumArgs& a, uint32_t row)
{
    const uint32_t lane = threadIdx.x & 31;
    uint32_t low = 0, high = a.n;               // the answer is in [low, high]
    while (low < high) {
        const uint32_t step = (high - low + 31) / 32;
        const uint64_t probe = (uint64_t)low + (uint64_t)(lane + 1) * step - 1;
        const bool less = probe < high && a.sorted[probe].x < row;
        const uint32_t steps = __popc(__ballot_sync(0xffffffffu, less));      // the rows ascend
        high = (uint32_t)min((uint64_t)high, (uint64_t)low + (uint64_t)(steps + 1) * step - 1);
        low += steps * step;
    }
    return low;
}

// Zeros to the rows [from, to) that are not in the sorted list.
constexpr uint32_t kZeroRows = 256;
__device__ void write_zero_rows(const SumArgs& a, uint32_t from, uint32_t to)
{
    __shared__ bool taken[kZeroRows];
    for (uint32_t i = threadIdx.x; i < to - from; i += kSumThreads)
        taken[i] = false;
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t low = first_entry(a, from), high = first_entry(a, to);
    __syncthreads();
    if (high - low <= 16 * kSumThreads) {
#pragma unroll 4
        for (uint32_t i = low + threadIdx.x; i < high; i += kSumThreads)
            taken[a.sorted[i].x - from] = true;
    } else {                                    // long runs: looked for row by row
        for (uint32_t r = threadIdx.x; r < to - from; r += kSumThreads) {
            uint32_t left = low, right = high;
            while (left < right) {
                const uint32_t middle = left + (right - left) / 2;
                if (a.sorted[middle].x < from + r)
                    left = middle + 1;
                else
                    right = middle;
            }
            taken[r] = left < high && a.sorted[left].x == from + r;
        }
    }
    __syncthreads();
    const int64_t bytes = a.dim * (a.table_dtype == ADASUM_F32 ? 4 : 2);
    char* rows = static_cast<char*>(a.table) + (int64_t)from * bytes;
    const int warp = threadIdx.x >> 5;
    const bool by_sixteen = ((uintptr_t)a.table | (uintptr_t)bytes) % 16 == 0, by_four = ((uintptr_t)a.table | (uintptr_t)bytes) % 4 == 0;
    for (uint32_t r = warp; r < to - from; r += kSumThreads / 32) {
        if (taken[r])
            continue;
        char* p = rows + (int64_t)r * bytes;
        if (by_sixteen) {
            for (int64_t i = lane; i < bytes / 16; i += 32)
                reinterpret_cast<uint4*>(p)[i] = make_uint4(0, 0, 0, 0);
        } else if (by_four) {
            for (int64_t i = lane; i < bytes / 4; i += 32)
                reinterpret_cast<uint32_t*>(p)[i] = 0;
        } else {
            for (int64_t i = lane; i < bytes / 2; i += 32)
                reinterpret_cast<uint16_t*>(p)[i] = 0;
        }
    }
}

// Bound by HBM: 32768 tokens of 1024 bf16 elements on 8 600 rows 25 us (127 MB, 5 TB/s); 4608 tokens with the
// zeros of 30522 fp32 rows 23 us (134 MB, 5.8 TB/s).
//
// VE: elements a thread owns; more than one only where a row divides into vectors that are 16-byte
// aligned in grad_out.  grid.x = tiles (and blocks that write zeros), grid.y = blocks per row of kSumThreads * VE
// columns (the zeros are left to the first of them); dynamic shared
// memory: one tile's terms (16 bytes, or one float, per thread and term; a thread reads back only its own).
template <typename T, int VE>
__global__ void __launch_bounds__(kSumThreads)
embedding_sum_kernel(const __grid_constant__ SumArgs a, const T* __restrict__ grad)
{
    wait_for_previous_kernel();
    start_next_kernel();
    extern __shared__ __align__(16) unsigned char terms[];
    // row[1 + i], position[i]: entry i of the tile, on into the next tile; row[0]: the entry before
    __shared__ uint32_t row[2 * kMaxTile + 2], position[2 * kMaxTile + 1];
    constexpr uint32_t kNone = 0xffffffffu;
    if (blockIdx.x >= a.tiles) {
        const uint32_t from = (blockIdx.x - a.tiles) * a.zero_rows;
        if (blockIdx.y == 0)
            write_zero_rows(a, from, min(a.num_rows, from + a.zero_rows));
        return;
    }
    const uint32_t begin = blockIdx.x * (uint32_t)a.tile;
    const int m = (int)min((uint32_t)a.tile, a.n - begin);
    for (int i = threadIdx.x; i < m + a.tile + 2; i += kSumThreads) {
        const int64_t at = (int64_t)begin + i - 1;
        const uint2 it = at >= 0 && at < (int64_t)a.n ? a.sorted[at] : make_uint2(kNone, 0);
        row[i] = it.x;
        if (i >= 1)
            position[i - 1] = it.y;
    }
    // did the run that this tile begins with start in the tile before?  (entry before that tile)
    const uint32_t earlier = begin > (uint32_t)a.tile ? a.sorted[begin - a.tile - 1].x : kNone;
    __syncthreads();
    const uint32_t first = row[1], last = row[m];
    int skip = 0;                      // leading entries that the tile before adds up
    bool enters = false;               // the leading run is a long one that started earlier
    if (row[0] == first) {
        int length = 1;                // of the leading run from here, as far as it matters
        while (length <= a.tile && row[1 + length] == first)
            ++length;
        if (earlier != first && length <= a.tile)
            skip = length;
        else
            enters = true;
    }
    int extra = 0;                     // entries of the last run beyond the tile
    bool goes_on = false;              // more than one tile's length of them: left to the join
    if (skip < m && !(enters && first == last)) {
        while (extra <= a.tile && row[1 + m + extra] == last)
            ++extra;
        goes_on = extra > a.tile;
        if (goes_on)
            extra = 0;
    }
    if (goes_on && last < a.num_rows && blockIdx.y == 0 && threadIdx.x == 0)
        a.long_runs[1 + atomicAdd(a.long_runs, 1u)] = blockIdx.x;
    const int stop = m + extra;
    const uint32_t stage = static_cast<uint32_t>(__cvta_generic_to_shared(terms)) + threadIdx.x * (VE > 1 ? 16 : 4);
    constexpr int kPitch = kSumThreads * (VE > 1 ? 16 : 4);          // bytes from term to term
    for (int64_t column = ((int64_t)blockIdx.y * kSumThreads + threadIdx.x) * VE; column < a.dim;
         column += (int64_t)gridDim.y * kSumThreads * VE) {
        float sum[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i)
            sum[i] = 0.0f;
        int start = skip;              // where the current run starts
        for (int base = skip; base < stop; base += a.tile) {
            const int batch = min(a.tile, stop - base);
            if constexpr (VE > 1) {
#pragma unroll 4
                for (int i = 0; i < batch; ++i)
                    if (row[1 + base + i] < a.num_rows)
                        cp_async_16B_shared(stage + i * kPitch, grad + (int64_t)position[base + i] * a.stride + column);
                cp_async_commit();
                cp_async_wait<0>();
            } else {
#pragma unroll 8
                for (int i = 0; i < batch; ++i) {
                    const float x = row[1 + base + i] < a.num_rows
                                        ? Element<T>::one(grad + (int64_t)position[base + i] * a.stride + column)
                                        : 0.0f;
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(stage + i * kPitch), "f"(x));
                }
            }
            for (int i = 0; i < batch; ++i) {
                float x[VE];
                if constexpr (VE > 1)
                    decode_vector<T>(load_shared_16B(stage + i * kPitch), x);
                else
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[0]) : "r"(stage + i * kPitch));
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    sum[e] += x[e];
                const int end = base + i + 1;
                const uint32_t r = row[end];
                if (end < stop && row[1 + end] == r)
                    continue;
                // the run ends here, or the tile's share of it
                if (r < a.num_rows) {
                    const bool from_before = start == 0 && enters;
                    if (!from_before && !(end == stop && goes_on)) {
                        write_row<VE>(a, r, column, sum);
                    } else {
                        float* edge = a.edges + ((int64_t)blockIdx.x * 2 + (from_before ? 0 : 1)) * a.dim + column;
#pragma unroll
                        for (int e = 0; e < VE; ++e)
                            edge[e] = sum[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    sum[e] = 0.0f;
                start = end;
            }
        }
    }
}

__device__ __forceinline__ void load_sums(const float* p, float (&x)[4])
{
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x;
    x[1] = v.y;
    x[2] = v.z;
    x[3] = v.w;
}

__device__ __forceinline__ void load_sums(const float* p, float (&x)[1]) { x[0] = *p; }

// Rows whose run goes on for more than a tile's length beyond the tile in which it starts.  A block takes 32 VE
// columns of one such run at a time; every warp adds its part of the run's edges, and the warps' sums are added in
// order.  Latency: the list, the run's end, eight edges at a time (16384 tokens on two rows, 512 edges each: 6 us).
constexpr int kJoinThreads = 512;
constexpr int kInFlight = 8;            // edges whose loads are issued together
constexpr int kJoinWarps = kJoinThreads / 32;

template <int VE>
__device__ void join_runs(const SumArgs& a, uint32_t runs, float (*part)[32 * 4])
{
    const uint32_t tiles = (a.n + a.tile - 1) / a.tile;
    const int64_t slices = (a.dim + 32 * VE - 1) / (32 * VE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t item = blockIdx.x; item < runs * slices; item += gridDim.x) {
        const uint32_t tile = a.long_runs[1 + item / slices];
        const int64_t column = (item % slices * 32 + lane) * VE;
        const uint32_t r = a.sorted[(int64_t)(tile + 1) * a.tile - 1].x;
        // last tile of the run: the sorted rows ascend, so count the following tiles that begin with r
        uint32_t count = 0;
        for (;;) {
            const uint64_t probe = (uint64_t)tile + 1 + count + threadIdx.x;
            const bool inside = probe < tiles && a.sorted[probe * a.tile].x == r;
            const uint32_t hits = __syncthreads_count(inside);
            count += hits;
            if (hits < kJoinThreads)
                break;
        }
        const uint32_t edges = count + 1;               // this tile's second edge, then `count` first edges
        const uint32_t share = (edges + kJoinWarps - 1) / kJoinWarps;
        float sum[VE] = {};
        if (column < a.dim) {
            const uint32_t from = warp * share, to = min(edges, from + share);
            const float* first = a.edges + (int64_t)tile * 2 * a.dim + column;
            for (uint32_t k0 = from; k0 < to; k0 += kInFlight) {
                float x[kInFlight][VE];
#pragma unroll
                for (int j = 0; j < kInFlight; ++j) {
                    const uint32_t k = min(k0 + j, to - 1);
                    load_sums(first + ((int64_t)k * 2 + (k == 0 ? 1 : 0)) * a.dim, x[j]);
                }
#pragma unroll
                for (int j = 0; j < kInFlight; ++j)
                    if (k0 + j < to) {
#pragma unroll
                        for (int e = 0; e < VE; ++e)
                            sum[e] += x[j][e];
                    }
            }
        }
#pragma unroll
        for (int e = 0; e < VE; ++e)
            part[warp][lane * VE + e] = sum[e];
        __syncthreads();
        if (warp == 0 && column < a.dim) {
#pragma unroll
            for (int e = 0; e < VE; ++e)
                for (int w = 1; w < kJoinWarps; ++w)
                    sum[e] += part[w][lane * VE + e];
            write_row<VE>(a, r, column, sum);
        }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kJoinThreads) embedding_join_kernel(const __grid_constant__ SumArgs a)
{
    wait_for_previous_kernel();
    __shared__ float part[kJoinWarps][32 * 4];
    const uint32_t runs = *a.long_runs;
    // four columns per lane where that still leaves every block something to do
    if (a.table_vec && runs * ((a.dim + 127) / 128) >= gridDim.x)
        join_runs<4>(a, runs, part);
    else
        join_runs<1>(a, runs, part);
}

// ---- host ------------------------------------------------------------------------------------------------

// Entries per tile: short tiles spread a short list over more blocks, long ones leave fewer shares of long runs to be
// joined.  Whole calls with 8 against 16 (us): into 1009 x 203 with 64 tokens 7.8/9.1, 999 11.6/13.9, 2047 12.2/16.7, 4096
// 15.7/18.3, 16384 32.4/29.9; into 512 x 1024 with 999 10.4/11.8, 2047 14.2/13.6, 16384 37.3/32.6; into 30522 x 1024 with 999
// 28.4/27.0, 2047 32.3/29.0, 16384 49.7/46.2.  The crossing moves from about 1000 tokens (wide rows) to 8000 (narrow ones);
// 2048 lies between.  Up to 32 tokens, two tiles of 16 need no join.  (32: 38 us where 8 and 16 took 26 and 28, and 36.)
constexpr int64_t kShortTilesBelow = 2048;
int sum_tile(int64_t n) { return n > 2 * kMaxTile && n < kShortTilesBelow ? kMaxTile / 2 : kMaxTile; }
int64_t sum_tiles(int64_t n) { return (n + sum_tile(n) - 1) / sum_tile(n); }
// Tiles that the workspace has room for: the most that any list of up to n entries has, so that a workspace for a
// long list does for every shorter one.
int64_t most_sum_tiles(int64_t n)
{
    const int64_t own = sum_tiles(n), shorter = n < kShortTilesBelow ? 0 : sum_tiles(kShortTilesBelow - 1);
    return own > shorter ? own : shorter;
}

// Clusters of embedding_sort_kernel that are resident at once (a cluster keeps to one group of
// multiprocessors, so some of these stay without): with one more, its share of the zeros would be written
// after all others'.
template <typename Id>
int resident_sort_clusters()
{
    static int cached[64] = {};
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64)
        return 2;
    if (cached[device] == 0) {
        cudaLaunchConfig_t config = {};
        config.gridDim = dim3(kSortCluster);
        config.blockDim = dim3(kSortThreads);
        cudaLaunchAttribute attribute;
        attribute.id = cudaLaunchAttributeClusterDimension;
        attribute.val.clusterDim.x = kSortCluster;
        attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
        config.attrs = &attribute;
        config.numAttrs = 1;
        int clusters = 0;
        if (cudaOccupancyMaxActiveClusters(&clusters, embedding_sort_kernel<Id>, &config) != cudaSuccess || clusters < 2) {
            cudaGetLastError();
            clusters = 2;
        }
        cached[device] = clusters;
    }
    return cached[device];
}

struct GradLayout {
    size_t sorted, spare, long_runs, edges, total;
};
GradLayout grad_layout(int64_t n, int64_t dim)
{
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t list = up((size_t)n * sizeof(uint2));
    const int64_t tiles = most_sum_tiles(n);
    GradLayout l;
    l.sorted = 0;
    l.spare = list;
    l.long_runs = 2 * list;
    l.edges = l.long_runs + up(((size_t)tiles + 1) * sizeof(uint32_t));
    l.total = l.edges + up((size_t)tiles * 2 * (size_t)dim * sizeof(float));
    if (l.total == 0)
        l.total = 256;
    return l;
}

constexpr int64_t kMaxDim = int64_t(1) << 22;

adasum_status_t check_tokens(const void* tokens, int32_t token_bytes, int64_t num_tokens, int64_t num_rows,
                             int64_t dim)
{
    if (!extent_ok(num_tokens) || !extent_ok(num_rows) || dim < 0 || dim > kMaxDim)
        return fail(ADASUM_ERR_ARG, "num_tokens = %lld, num_rows = %lld, dim = %lld out of range",
                    (long long)num_tokens, (long long)num_rows, (long long)dim);
    if (token_bytes != 4 && token_bytes != 8)
        return fail(ADASUM_ERR_ARG, "token_bytes = %d is neither 4 nor 8", (int)token_bytes);
    if (num_tokens > 0 && !tokens)
        return fail(ADASUM_ERR_NULL, "tokens is NULL");
    if (!aligned_to(tokens, token_bytes))
        return fail(ADASUM_ERR_ARG, "tokens is not aligned to its element size");
    return ADASUM_OK;
}

}  // namespace
}  // namespace adasum

extern "C" {

adasum_status_t adasum_embedding_forward(const void* table, int64_t table_stride, int64_t num_rows, int64_t dim,
                                         adasum_dtype_t table_dtype, const void* tokens, int32_t token_bytes,
                                         int64_t num_tokens, float scale, void* out, int64_t out_stride,
                                         adasum_dtype_t out_dtype, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    if (!operator_dtype(table_dtype) || !operator_dtype(out_dtype))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d: fp32, fp16 or bf16", (int)table_dtype, (int)out_dtype);
    const adasum_status_t status = check_tokens(tokens, token_bytes, num_tokens, num_rows, dim);
    if (status != ADASUM_OK || num_tokens == 0 || dim == 0)
        return status;
    if ((num_rows > 0 && !table) || !out)
        return fail(ADASUM_ERR_NULL, "table or out is NULL");
    if (!aligned_to(table, operator_bytes(table_dtype)) || !aligned_to(out, operator_bytes(out_dtype)))
        return fail(ADASUM_ERR_ARG, "table or out is not aligned to its element size");
    if (!stride_ok(table_stride, dim) || !stride_ok(out_stride, dim))
        return fail(ADASUM_ERR_ARG, "a stride is shorter than a row or out of range");
    const size_t table_bytes = matrix_span(num_rows, dim, table_stride, operator_bytes(table_dtype));
    const size_t out_bytes = matrix_span(num_tokens, dim, out_stride, operator_bytes(out_dtype));
    if (spans_overlap(out, out_bytes, table, table_bytes) ||
        spans_overlap(out, out_bytes, tokens, (size_t)num_tokens * token_bytes))
        return fail(ADASUM_ERR_ARG, "out overlaps table or tokens");
    Strips s;
    unsigned blocks;
    if (!plan_strips(num_tokens, dim, (dim + 7) / 8, kLookupRows, &s, &blocks))
        return fail(ADASUM_ERR_ARG, "%lld x %lld is too large", (long long)num_tokens, (long long)dim);
    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    profile_mark(stream, -1, 0, 0, true);
    with_type(table_dtype, [&](auto t) {
        using T = decltype(t);
        const bool vec = dim % 8 == 0 && rows_aligned(table, table_stride, sizeof(T)) &&
                         rows_aligned(out, out_stride, operator_bytes(out_dtype));
        auto launch = [&](auto id) {
            using Id = decltype(id);
            auto* kernel = vec ? embedding_forward_kernel<T, Id, true> : embedding_forward_kernel<T, Id, false>;
            kernel<<<blocks, kStripThreads, 0, stream>>>(s, static_cast<const T*>(table), table_stride, num_rows,
                                                         static_cast<const Id*>(tokens), scale, out, (int)out_dtype,
                                                         out_stride);
        };
        if (token_bytes == 4)
            launch(int32_t{});
        else
            launch(int64_t{});
    });
    ADASUM_CUDA_CHECK(cudaGetLastError());
    profile_mark(stream, ADASUM_KERNEL_EMBEDDING, 0, 0, false);
    return ADASUM_OK;
}

size_t adasum_embedding_grad_workspace_bytes(int64_t num_tokens, int64_t num_rows, int64_t dim)
{
    using namespace adasum;
    if (!extent_ok(num_tokens) || !extent_ok(num_rows) || dim < 0 || dim > kMaxDim)
        return 0;
    return grad_layout(num_tokens, dim).total;
}

adasum_status_t adasum_embedding_grad(const void* grad_out, int64_t grad_out_stride, adasum_dtype_t dtype,
                                      const void* tokens, int32_t token_bytes, int64_t num_tokens, float scale,
                                      void* grad_table, int64_t num_rows, int64_t dim, adasum_dtype_t grad_dtype,
                                      int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream_ptr)
{
    using namespace adasum;
    clear_error();
    if (!operator_dtype(dtype) || !operator_dtype(grad_dtype))
        return fail(ADASUM_ERR_DTYPE, "dtypes %d, %d: fp32, fp16 or bf16", (int)dtype, (int)grad_dtype);
    const adasum_status_t status = check_tokens(tokens, token_bytes, num_tokens, num_rows, dim);
    if (status != ADASUM_OK || num_rows == 0 || dim == 0 || (num_tokens == 0 && accumulate))
        return status;
    if (!grad_table || (num_tokens > 0 && !grad_out))
        return fail(ADASUM_ERR_NULL, "grad_out or grad_table is NULL");
    if (!aligned_to(grad_out, operator_bytes(dtype)) || !aligned_to(grad_table, operator_bytes(grad_dtype)))
        return fail(ADASUM_ERR_ARG, "grad_out or grad_table is not aligned to its element size");
    if (num_tokens > 0 && !stride_ok(grad_out_stride, dim))
        return fail(ADASUM_ERR_ARG, "grad_out_stride %lld is shorter than a row or out of range",
                    (long long)grad_out_stride);
    const GradLayout lay = grad_layout(num_tokens, dim);
    if (!workspace || workspace_bytes < lay.total)
        return fail(ADASUM_ERR_WORKSPACE, "workspace of %zu bytes, need %zu", workspace ? workspace_bytes : (size_t)0,
                    lay.total);
    if (!aligned_to(workspace, 256))
        return fail(ADASUM_ERR_ARG, "workspace is not 256-byte aligned");
    const size_t in_bytes = matrix_span(num_tokens, dim, grad_out_stride, operator_bytes(dtype));
    const size_t token_span = (size_t)num_tokens * (size_t)token_bytes;
    const int64_t table_bytes = num_rows * dim * operator_bytes(grad_dtype);
    if (spans_overlap(grad_table, (size_t)table_bytes, grad_out, in_bytes) ||
        spans_overlap(grad_table, (size_t)table_bytes, tokens, token_span))
        return fail(ADASUM_ERR_ARG, "grad_table overlaps grad_out or tokens");
    if (spans_overlap(workspace, lay.total, grad_out, in_bytes) || spans_overlap(workspace, lay.total, tokens, token_span) ||
        spans_overlap(workspace, lay.total, grad_table, (size_t)table_bytes))
        return fail(ADASUM_ERR_ARG, "workspace overlaps another buffer");
    const int sms = device_sms();
    if (sms <= 0)
        return fail(ADASUM_ERR_CUDA, "no current device");

    cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
    char* ws = static_cast<char*>(workspace);
    uint2* sorted = reinterpret_cast<uint2*>(ws + lay.sorted);
    uint2* spare = reinterpret_cast<uint2*>(ws + lay.spare);
    uint32_t* long_runs = reinterpret_cast<uint32_t*>(ws + lay.long_runs);
    int passes = 1;
    while (passes < 4 && ((uint64_t)num_rows >> (8 * passes)) != 0)     // the key num_rows itself included
        ++passes;
    profile_mark(stream, -1, 0, 0, true);
    if (num_tokens == 0) {                 // zeros of any type are zero bytes
        ADASUM_CUDA_CHECK(cudaMemsetAsync(grad_table, 0, (size_t)table_bytes, stream));
        return ADASUM_OK;
    }
    const int64_t zero_bytes = accumulate ? 0 : table_bytes;
    const bool rank = ranked(num_tokens, zero_bytes, sms);
    auto sort = [&](auto id) {
        using Id = decltype(id);
        const Id* ids = static_cast<const Id*>(tokens);
        if (rank) {
            const int64_t wanted = (num_tokens + kRankThreads / 32 - 1) / (kRankThreads / 32);
            embedding_rank_kernel<Id><<<(unsigned)(wanted < sms ? wanted : sms), kRankThreads,
                                        (size_t)((num_tokens + 127) / 128 * 128) * sizeof(uint32_t), stream>>>(
                ids, (uint32_t)num_tokens, (uint32_t)num_rows, sorted, long_runs);
        } else {
            const int64_t wanted = ((zero_bytes + kZeroBytes - 1) / kZeroBytes + kSortCluster - 1) / kSortCluster + 1;
            const int64_t clusters = resident_sort_clusters<Id>();
            embedding_sort_kernel<Id><<<(unsigned)((wanted < clusters ? wanted : clusters) * kSortCluster), kSortThreads, 0,
                                        stream>>>(ids, (uint32_t)num_tokens, (uint32_t)num_rows, passes, sorted, spare,
                                                  long_runs, static_cast<char*>(grad_table), zero_bytes);
        }
    };
    if (token_bytes == 4)
        sort(int32_t{});
    else
        sort(int64_t{});
    ADASUM_CUDA_CHECK(cudaGetLastError());
    profile_mark(stream, ADASUM_KERNEL_EMBEDDING_SORT, 0, 0, false);

    SumArgs a;
    a.sorted = sorted;
    a.n = (uint32_t)num_tokens;
    a.num_rows = (uint32_t)num_rows;
    a.tile = sum_tile(num_tokens);
    a.stride = grad_out_stride;
    a.dim = dim;
    a.scale = scale;
    a.table = grad_table;
    a.table_dtype = (int)grad_dtype;
    a.accumulate = accumulate != 0;
    a.long_runs = long_runs;
    a.edges = reinterpret_cast<float*>(ws + lay.edges);
    a.tiles = (uint32_t)sum_tiles(num_tokens);
    // about 64 KB of zeros per block
    const int64_t row_bytes = dim * operator_bytes(grad_dtype), fit = 65536 / row_bytes;
    a.zero_rows = (uint32_t)(fit < 1 ? 1 : fit < kZeroRows ? fit : kZeroRows);
    const int64_t zero_blocks = accumulate || !rank ? 0 : (num_rows + a.zero_rows - 1) / a.zero_rows;
    if (a.tiles + zero_blocks > 0x7fffffff)
        return fail(ADASUM_ERR_ARG, "%lld tokens and %lld rows are too many", (long long)num_tokens, (long long)num_rows);
    cudaError_t launch_error = cudaSuccess;
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int VE = Element<T>::kVec;
        const bool vec = rows_aligned(grad_out, grad_out_stride, sizeof(T)) && dim % VE == 0;
        a.table_vec = vec && aligned_to(grad_table, 16) && dim * operator_bytes(grad_dtype) % 16 == 0;
        const int64_t columns = (int64_t)kSumThreads * (vec ? VE : 1);
        const int64_t slices = (dim + columns - 1) / columns;
        const dim3 grid((unsigned)(a.tiles + zero_blocks), (unsigned)(slices < 65535 ? slices : 65535));
        const size_t bytes = (size_t)a.tile * kSumThreads * (vec ? 16 : 4);
        if (vec) {
            launch_error = launch_after(embedding_sum_kernel<T, VE>, grid, kSumThreads, bytes, stream, a,
                                        static_cast<const T*>(grad_out));
        } else {
            launch_error = launch_after(embedding_sum_kernel<T, 1>, grid, kSumThreads, bytes, stream, a,
                                        static_cast<const T*>(grad_out));
        }
    });
    ADASUM_CUDA_CHECK(launch_error);
    profile_mark(stream, ADASUM_KERNEL_EMBEDDING_SUM, 0, 0, false);
    if (num_tokens > 2 * a.tile) {         // a long run has more than a tile's length beyond its first entry's tile
        const int64_t slices = (dim + 31) / 32;
        const int64_t most = slices * (num_tokens / a.tile), resident = (int64_t)sms * 2;
        // rows of four-element vectors, 16-byte aligned in the workspace and at least 8-byte aligned in the table
        a.table_vec = aligned_to(grad_table, 16) && dim % 4 == 0;
        ADASUM_CUDA_CHECK(launch_after(embedding_join_kernel, dim3((unsigned)(most < resident ? most : resident)), kJoinThreads,
                                       0, stream, a));
        profile_mark(stream, ADASUM_KERNEL_EMBEDDING_SUM, 1, 0, false);
    }
    return ADASUM_OK;
}

}  // extern "C"
