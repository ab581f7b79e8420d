// sort_rows.hip -- entries of a batch in the order of the table rows they name.
//
// A stable radix sort from the lowest digit up of (row, entry) pairs; the key
// has only the bits that the table's row numbers need, divided evenly over
// passes of at most 8 bits, and entries outside the table sort behind all
// rows.  A pass counts the digits of each tile, finds where each tile's
// share of each digit begins, and moves the pairs.  Positions come from
// ballots and prefix sums, so the order is the same in every run.  Small
// sorts are bound by their launches (two per pass up to 64 tiles, where each
// tile adds up the others' counts itself; else three), large ones by moving
// 16 bytes an entry and pass.
#include <hip/hip_runtime.h>

#include "numeric.h"
#include "smore_internal.h"

namespace smore {
namespace {

constexpr int WG = 256;
constexpr int WAVES = WG / 64;
constexpr int DIGITS = 256;
// Tiles up to which each adds up the others' counts itself.  us with 16 / 64 /
// 128: 33K entries 20.3 / 18.3 / 18.3, 66K 20.9 / 20.9 / 21.8, 131K 22 / 22 / 28.
constexpr int FEW_TILES = 64;

// Key of an id: the row, or the number of rows for one outside the table.
__device__ __forceinline__ uint32_t key_of(int32_t id, uint32_t n_rows) { return min((uint32_t)id, n_rows); }

// counts[tile * digits + d]
template <int ITEMS>
__global__ __launch_bounds__(WG) void k_count(const int32_t* __restrict__ ids, uint32_t n, uint32_t n_rows, int shift,
                                              uint32_t digits, uint32_t* __restrict__ counts)
{
    __shared__ uint32_t h[DIGITS];
    h[threadIdx.x] = 0;
    __syncthreads();
    const uint64_t base = (uint64_t)blockIdx.x * (WG * ITEMS);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const uint64_t i = base + k * WG + threadIdx.x;
        if (i < n) atomicAdd(&h[(key_of(ids[i], n_rows) >> shift) & (digits - 1)], 1u);
    }
    __syncthreads();
    if (threadIdx.x < digits) counts[(uint64_t)blockIdx.x * digits + threadIdx.x] = h[threadIdx.x];
}

// Exclusive prefix sums of each digit's counts over the tiles, in place, and
// each digit's total.  A workgroup takes one digit, 256 tiles at a time.
__global__ __launch_bounds__(WG) void k_prefix(uint32_t* __restrict__ counts, uint32_t tiles, uint32_t digits,
                                               uint32_t* __restrict__ totals)
{
    __shared__ uint32_t part[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t before = 0;
    for (uint32_t t0 = 0; t0 < tiles; t0 += WG) {
        const uint32_t t = t0 + threadIdx.x;
        uint32_t* at = counts + (uint64_t)t * digits + blockIdx.x;
        const uint32_t x = t < tiles ? *at : 0;
        uint32_t sum = x;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const uint32_t y = __shfl_up(sum, s);
            if (lane >= s) sum += y;
        }
        if (lane == 63) part[wave] = sum;
        __syncthreads();
        uint32_t all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) sum += part[w];
            all += part[w];
        }
        if (t < tiles) *at = before + sum - x;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// Moves a tile's pairs.  entries NULL: the pairs are in their first order.
// In the last pass order (64-bit) is written in place of the entries.
template <int ITEMS>
__global__ __launch_bounds__(WG) void k_move(const int32_t* __restrict__ ids, const uint32_t* __restrict__ entries,
                                             uint32_t n, uint32_t n_rows, int shift, int bits,
                                             const uint32_t* __restrict__ counts, uint32_t tiles,
                                             const uint32_t* __restrict__ totals, int32_t* __restrict__ ids_out,
                                             uint32_t* __restrict__ entries_out, int64_t* __restrict__ order)
{
    __shared__ uint32_t taken[WAVES][DIGITS];   // of each digit by each wavefront, then where they go
    __shared__ uint32_t part[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t digits = 1u << bits, d0 = threadIdx.x;
    // where this tile's digit d0 begins: behind all smaller digits and the
    // same digit of the tiles before
    uint32_t total = 0, before = 0;
    if (d0 < digits) {
        if (totals) {
            total = totals[d0];
            before = counts[(uint64_t)blockIdx.x * digits + d0];
        } else {
#pragma unroll 8
            for (uint32_t t = 0; t < tiles; ++t) {
                const uint32_t x = counts[t * digits + d0];
                total += x;
                if (t < blockIdx.x) before += x;
            }
        }
    }
    uint32_t sum = total;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t y = __shfl_up(sum, s);
        if (lane >= s) sum += y;
    }
    if (lane == 63) part[wave] = sum;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) taken[w][threadIdx.x] = 0;
    __syncthreads();
    uint32_t begin = sum - total + before;
    for (int w = 0; w < wave; ++w) begin += part[w];

    // ranks within the wavefront's 64 x ITEMS consecutive pairs
    const uint64_t base = (uint64_t)blockIdx.x * (WG * ITEMS) + wave * (64 * ITEMS) + lane;
    const uint64_t lower = (1ull << lane) - 1;
    int32_t id[ITEMS];
    uint32_t entry[ITEMS], rank[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const uint64_t i = base + k * 64;
        id[k] = i < n ? ids[i] : 0;
        entry[k] = i < n ? (entries ? entries[i] : (uint32_t)i) : 0;
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const bool in = base + k * 64 < n;
        const uint32_t d = (key_of(id[k], n_rows) >> shift) & (digits - 1);
        uint64_t peers = __ballot(in);
        for (int b = 0; b < bits; ++b) {
            const uint64_t m = __ballot((d >> b) & 1);
            peers &= (d >> b) & 1 ? m : ~m;
        }
        // lanes of one wavefront: reads of a row of pairs before its writes
        const uint32_t had = taken[wave][d];
        rank[k] = had + __popcll(peers & lower);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (in && (peers & lower) == 0) taken[wave][d] = had + __popcll(peers);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    if (d0 < digits) {
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t x = taken[w][d0];
            taken[w][d0] = begin;
            begin += x;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        if (base + k * 64 >= n) continue;
        const uint32_t to = taken[wave][(key_of(id[k], n_rows) >> shift) & (digits - 1)] + rank[k];
        ids_out[to] = id[k];
        if (order) order[to] = entry[k];
        else entries_out[to] = entry[k];
    }
}

struct Plan {
    int passes, bits, items;
    uint32_t tiles;
    size_t pairs, counts;   // bytes of one array of 4-byte words, and of the counts with the totals
    Plan(int64_t n, int32_t n_rows)
    {
        int need = 1;   // bits of the key n_rows
        while (need < 32 && (1ll << need) <= n_rows) ++need;
        passes = (need + 7) / 8;
        bits = (need + passes - 1) / passes;
        // Short tiles until they fill the chip.  us with 4 / 16 a thread: 66K
        // entries of 15,000 rows 21 / 37, 264K and 1.05M of 400,000 rows 39 / 62
        // and 67 / 80, 4.2M 185 / 151, 8.4M of 86M rows 470 / 433; equal at 2.1M,
        // and in between 4 would still be better (1.1M 73 / 91).
        items = n <= (int64_t)1024 * WG * 4 ? 4 : 16;
        tiles = (uint32_t)((n + WG * items - 1) / (WG * items));
        pairs = ((size_t)n * 4 + 255) & ~(size_t)255;
        counts = ((size_t)(tiles + 1) * DIGITS * 4 + 255) & ~(size_t)255;
    }
};

template <int ITEMS>
void passes_of(const Plan& p, const int32_t* ids, uint32_t n, uint32_t n_rows, int32_t* rows, int64_t* order, char* ws,
               hipStream_t st)
{
    // ids and entries alternate between two pairs of arrays; the last pass writes the outputs
    int32_t* id_buf[2] = {(int32_t*)ws, (int32_t*)(ws + p.pairs)};
    uint32_t* entry_buf[2] = {(uint32_t*)(ws + 2 * p.pairs), (uint32_t*)(ws + 3 * p.pairs)};
    uint32_t* counts = (uint32_t*)(ws + 4 * p.pairs);
    const uint32_t digits = 1u << p.bits;
    uint32_t* totals = counts + (size_t)p.tiles * digits;
    const bool few = p.tiles <= FEW_TILES;
    const uint32_t* entries = nullptr;
    for (int k = 0; k < p.passes; ++k) {
        const bool last = k + 1 == p.passes;
        const int shift = k * p.bits;
        k_count<ITEMS><<<p.tiles, WG, 0, st>>>(ids, n, n_rows, shift, digits, counts);
        if (!few) k_prefix<<<digits, WG, 0, st>>>(counts, p.tiles, digits, totals);
        k_move<ITEMS><<<p.tiles, WG, 0, st>>>(ids, entries, n, n_rows, shift, p.bits, counts, p.tiles, few ? nullptr : totals,
                                              last ? rows : id_buf[k & 1], entry_buf[k & 1], last ? order : nullptr);
        ids = id_buf[k & 1];
        entries = entry_buf[k & 1];
    }
}

}  // namespace

size_t sort_rows_workspace(int64_t n, int32_t n_rows)
{
    const Plan p(n, n_rows);
    return n ? 4 * p.pairs + p.counts : 0;
}

int launch_sort_rows(const int32_t* ids, int64_t n, int32_t n_rows, int32_t* rows, int64_t* order, void* ws, hipStream_t st,
                     const char** err)
{
    const Plan p(n, n_rows);
    if (p.items == 4) passes_of<4>(p, ids, (uint32_t)n, (uint32_t)n_rows, rows, order, (char*)ws, st);
    else passes_of<16>(p, ids, (uint32_t)n, (uint32_t)n_rows, rows, order, (char*)ws, st);
    return launched(err);
}

}  // namespace smore
