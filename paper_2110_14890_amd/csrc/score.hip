// score.hip -- scores of sampled candidates and their gradient.
//
//   s[b][k]  = sum_c E[id[b][k]][c] q[b][c]
//   dq[b][c] = sum_k g[b][k] E[id[b][k]][c]
//
// E is the entity table (V x dim), id the candidates that the sampler wrote;
// an id outside [0, V) (the padding of short rows) has score 0 and adds
// nothing.  One product and sum per element read, so both kernels are bound
// by gathering rows of E; what they must not do is write the gathered rows
// [B, n, dim] anywhere.  Sums are in fp32, in an order that depends on the
// sizes alone.
#include <hip/hip_runtime.h>

#include "numeric.h"
#include "smore_internal.h"

namespace smore {
namespace {

constexpr int WG = 256;
constexpr int WAVES = WG / 64;

// Columns that a lane holds in register block i of a row, LANES lanes per
// row: V from `first` on.  The last block of a row that is no multiple of V
// is moved back to end with the row; `skip` of its columns belong to the lane
// before.  Rows shorter than V take V = 1.
template <int LANES, int V>
struct Columns {
    int first, skip;
    bool any;
    __device__ Columns(int lane, int i, int tile0, int dim)
    {
        const int c = tile0 + (i * LANES + lane) * V;
        any = c < dim;
        first = c + V <= dim ? c : dim - V;
        skip = any ? c - first : 0;
    }
};

// The register blocks of U rows.  All loads of a block stand in one branch,
// so that they are in flight together.
template <class T, int LANES, int V, int NI, int U>
__device__ __forceinline__ void fetch(const T* const* rows, int lane, int tile0, int dim, Vec<T, V> (*raw)[NI])
{
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const Columns<LANES, V> at(lane, i, tile0, dim);
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u][i] = Vec<T, V>{};
        if (at.any) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u][i] = load_vec<T, V>(rows[u] + at.first);
        }
    }
}

// A row's register blocks as floats; columns of another lane 0.
template <class T, int LANES, int V, int NI>
__device__ __forceinline__ void take(const Vec<T, V>* raw, int lane, int tile0, int dim, bool ragged, float (*out)[V])
{
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) out[i][j] = (float)raw[i].x[j];
        if (ragged) {
            const Columns<LANES, V> at(lane, i, tile0, dim);
#pragma unroll
            for (int j = 0; j < V; ++j) out[i][j] = j < at.skip ? 0.0f : out[i][j];
        }
    }
}

// The candidates of up to 64 lanes, those that are entities first: their
// number, and how a lane's value moves there (push) and back (pull).
struct Packed {
    int count, place;
    bool real;
    __device__ Packed(int32_t id, int32_t rows)
    {
        real = id >= 0 && id < rows;
        const uint64_t mask = __ballot(real);
        count = __popcll(mask);
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
        place = real ? before : count + (int)(threadIdx.x & 63) - before;
    }
    __device__ int push(int x) const { return __builtin_amdgcn_ds_permute(place * 4, x); }
    __device__ int pull(int x) const { return __builtin_amdgcn_ds_bpermute(place * 4, x); }
};

// Row of packed candidate `at` (behind the last one: of another candidate).
template <class T, int LANES>
__device__ __forceinline__ const T* row_of(const T* table, int64_t stride, int32_t ids, int at)
{
    if constexpr (LANES == 64) return table + (int64_t)__builtin_amdgcn_readlane(ids, at & 63) * stride;
    else return table + (int64_t)__shfl(ids, at & 63) * stride;
}

__device__ __forceinline__ float as_f(uint32_t x) { return __uint_as_float(x); }

// Sums of s[0 .. U) over the LANES lanes of each group.  Each halving of the
// lanes halves the registers too: of two values, one goes on in the lower
// half of the lanes, the other in the upper.
template <int LANES, int U>
struct Sums {
    static constexpr int GROUPS = 64 / LANES;
    static constexpr int R = LANES == 64 ? U / 4 : LANES == 32 ? U / 2 : U;   // registers left
    // lane t of 16 keeps register t % R
    static __device__ float over(float* s, int lane)
    {
        if constexpr (LANES == 64) {
#pragma unroll
            for (int j = 0; j < U / 2; ++j) {
                const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(s[j]), __float_as_uint(s[j + U / 2]), false, false);
                s[j] = as_f(x[0]) + as_f(x[1]);
            }
        }
        if constexpr (LANES >= 32) {
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(s[j]), __float_as_uint(s[j + R]), false, false);
                s[j] = as_f(x[0]) + as_f(x[1]);
            }
        }
#pragma unroll
        for (int j = 0; j < R; ++j) s[j] = sum16(s[j]);
        float kept = s[0];
#pragma unroll
        for (int j = 1; j < R; ++j) kept = lane % R == j ? s[j] : kept;
        return kept;
    }
    // the lane that keeps the sum of value u of a group
    static __device__ int source(int u, int group)
    {
        if constexpr (LANES == 64) return u / (U / 2) * 32 + u / R % 2 * 16 + u % R;
        else if constexpr (LANES == 32) return group * 32 + u / R * 16 + u % R;
        else return group * 16 + u;
    }
};

// A wavefront takes `tile` (up to 64) candidates of one query.  Its lanes
// read the ids, one each, and pack the entities; then 64 / LANES rows at a
// time, U times over before the first is used, are multiplied with the query,
// which stays in registers, and summed over the LANES lanes.  Lane k keeps
// packed candidate k's score, so that the scores leave in one store.
// 8,192 x 257 candidates (a quarter of them padding) of a 2 GB table of rows
// of 400 bf16: 239 us, 6.1 TB/s of 128-byte lines, of 6.5 to 7.1 that reads at
// random places reach; 425 with four wavefronts per workgroup, whose places a
// query short of negatives kept, and padding not packed away.
template <class TE, class TQ, int LANES, int V, int NI, int U>
__global__ __launch_bounds__(64) void k_score(const TE* __restrict__ table, int64_t table_stride, int rows, int dim,
                                              const TQ* __restrict__ queries, int64_t query_stride,
                                              const int32_t* __restrict__ ids, int64_t id_stride,
                                              float* __restrict__ out, int64_t out_stride, int n, int tile, int tiles)
{
    using Sum = Sums<LANES, U>;
    constexpr int GROUPS = Sum::GROUPS;
    const int lane = threadIdx.x, sub = lane % LANES, group = lane / LANES;
    const int64_t b = blockIdx.x / tiles;
    const int k0 = (int)(blockIdx.x - b * tiles) * tile;
    const int count = min(tile, n - k0);
    const int32_t id = lane < count ? ids[b * id_stride + k0 + lane] : -1;
    const Packed packed(id, rows);
    const int32_t all = packed.push(id);
    const int32_t some = __builtin_amdgcn_readfirstlane(all);
    const int32_t entity = lane < packed.count ? all : some;
    const bool ragged = dim % V != 0;
    float score = 0.0f;
    if (packed.count)
        for (int tile0 = 0; tile0 < dim; tile0 += LANES * V * NI) {
            const TQ* query = queries + b * query_stride;
            Vec<TQ, V> q_raw[1][NI];
            float q[NI][V];
            fetch<TQ, LANES, V, NI, 1>(&query, sub, tile0, dim, q_raw);
            take<TQ, LANES, V, NI>(q_raw[0], sub, tile0, dim, ragged, q);
            for (int k = 0; k < packed.count; k += GROUPS * U) {
                Vec<TE, V> raw[U][NI];
                const TE* row[U];
#pragma unroll
                for (int u = 0; u < U; ++u) row[u] = row_of<TE, LANES>(table, table_stride, entity, k + u * GROUPS + group);
                fetch<TE, LANES, V, NI, U>(row, sub, tile0, dim, raw);
                float s[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float x[NI][V];
                    s[u] = 0.0f;
                    take<TE, LANES, V, NI>(raw[u], sub, tile0, dim, ragged, x);
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int j = 0; j < V; ++j) s[u] = fmaf(x[i][j], q[i][j], s[u]);
                }
                const float kept = Sum::over(s, lane);
                const int at = lane - k;
                const float mine = __int_as_float(__builtin_amdgcn_ds_bpermute(
                    Sum::source(at / GROUPS % U, at % GROUPS) * 4, __float_as_int(kept)));
                if (at >= 0 && at < GROUPS * U) score += mine;
            }
        }
    const float back = __int_as_float(packed.pull(__float_as_int(score)));
    if (lane < count) out[b * out_stride + k0 + lane] = packed.real ? back : 0.0f;
}

// A workgroup takes one query's candidates [k0, k1) for LANES x V x NI of
// its columns; its wavefronts deal the candidates out 64 at a time and add
// their sums in LDS.  Several workgroups that share a query (splits > 1:
// few queries with long lists) write partial sums, which k_join adds.
// 4,096 x 257 candidates of 400,000 rows of 400 fp32: 197 us, 6.9 TB/s of
// lines, the MALL's among them; 16 x 4,001 of width 200 in bf16: 9.4 us with
// the sum of the parts.
template <class TE, class TO, int LANES, int V, int NI, int U>
__global__ __launch_bounds__(WG) void k_score_grad(const TE* __restrict__ table, int64_t table_stride, int rows, int dim,
                                                   const int32_t* __restrict__ ids, int64_t id_stride,
                                                   const float* __restrict__ grad, int64_t grad_stride,
                                                   TO* __restrict__ out, int64_t out_stride, int n, int span, int splits,
                                                   float* __restrict__ partial)
{
    constexpr int GROUPS = 64 / LANES, WIDTH = LANES * V * NI;
    __shared__ float part[WAVES][WIDTH];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LANES, group = lane / LANES;
    const int64_t b = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - b * splits);
    const int k0 = split * span, k1 = min(n, k0 + span);
    const int tile0 = blockIdx.y * WIDTH;
    const bool ragged = dim % V != 0;
    float acc[NI][V] = {};
    // equal shares of at most 64 candidates
    const int rounds = (k1 - k0 + 64 * WAVES - 1) / (64 * WAVES);
    const int step = max(1, (k1 - k0 + WAVES * rounds - 1) / max(1, WAVES * rounds));
    for (int base = k0 + wave * step; base < k1; base += WAVES * step) {
        const int count = min(step, k1 - base);
        int32_t id = -1;
        float g = 0.0f;
        if (lane < count) {
            id = ids[b * id_stride + base + lane];
            g = grad[b * grad_stride + base + lane];
        }
        const Packed packed(id, rows);
        const int32_t all = packed.push(id);
        const float weight = __int_as_float(packed.push(__float_as_int(g)));
        const int32_t some = __builtin_amdgcn_readfirstlane(all);
        const int32_t entity = lane < packed.count ? all : some;
        for (int k = 0; k < packed.count; k += GROUPS * U) {
            Vec<TE, V> raw[U][NI];
            const TE* row[U];
            float w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = k + u * GROUPS + group;
                row[u] = row_of<TE, LANES>(table, table_stride, entity, at);
                if constexpr (LANES == 64) w[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(weight), at & 63));
                else w[u] = __shfl(weight, at & 63);
            }
            fetch<TE, LANES, V, NI, U>(row, sub, tile0, dim, raw);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float x[NI][V];
                take<TE, LANES, V, NI>(raw[u], sub, tile0, dim, ragged, x);
                if (k + u * GROUPS + group < packed.count) {
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int j = 0; j < V; ++j) acc[i][j] = fmaf(w[u], x[i][j], acc[i][j]);
                }
            }
        }
    }
    // over the groups of a wavefront, then over the wavefronts
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float a = acc[i][j];
            if constexpr (GROUPS > 2) a += __shfl_xor(a, 16);
            if constexpr (GROUPS > 1) a += __shfl_xor(a, 32);
            if (group == 0) part[wave][(i * LANES + sub) * V + j] = a;
        }
    __syncthreads();
    for (int t = threadIdx.x; t < WIDTH; t += WG) {
        const Columns<LANES, V> at((t / V) % LANES, t / V / LANES, tile0, dim);
        const int c = at.first + t % V;
        if (!at.any || t % V < at.skip) continue;
        float s = part[0][t];
#pragma unroll
        for (int ww = 1; ww < WAVES; ++ww) s += part[ww][t];
        if (splits == 1) out[b * out_stride + c] = (TO)s;
        else partial[((int64_t)b * splits + split) * dim + c] = s;
    }
}

// 64 columns of a query: 16 wavefronts add every 16th partial sum each.
template <class TO>
__global__ __launch_bounds__(1024) void k_join(const float* __restrict__ partial, int splits, int dim, TO* __restrict__ out,
                                               int64_t out_stride)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = blockIdx.x;
    const int c = blockIdx.y * 64 + lane;
    float s = 0.0f;
    if (c < dim) {
#pragma unroll 4
        for (int k = wave; k < splits; k += 16) s += partial[(b * splits + k) * dim + c];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < dim) {
#pragma unroll
        for (int w = 1; w < 16; ++w) s += part[w][lane];
        out[b * out_stride + c] = (TO)s;
    }
}

template <class TE, class TQ, int LANES, int V, int NI, int UNROLL>
int score_as(const smore_score_args& a, const void* table, const void* queries, const int32_t* ids, float* scores,
             hipStream_t st, const char** err)
{
    // Candidates per wavefront: up to 64, fewer where that leaves CUs without
    // work.  us aimed at 2,048 / 4,096 / 8,192 wavefronts: 512 x 129 of width 400
    // in fp32 20.3 / 20.2 / 19.2, 2,048 x 129 in bf16 39.1 / 39.1 / 40.8, 1 x
    // 100,000 of width 200 11.0 / 10.6 / 12.5; 16 x 4,001 6.1 / 8.1 / 8.1.
    int tile = 64;
    while (tile > 8 && (int64_t)a.batch * ((a.n + tile - 1) / tile) < 4096) tile /= 2;
    const int tiles = (a.n + tile - 1) / tile;
    tile = (a.n + tiles - 1) / tiles;
    k_score<TE, TQ, LANES, V, NI, UNROLL><<<(unsigned)((int64_t)a.batch * tiles), 64, 0, st>>>(
        (const TE*)table, a.table_stride, a.n_rows, a.dim, (const TQ*)queries, a.query_stride, ids, a.candidate_stride,
        scores, a.score_stride, a.n, tile, tiles);
    return launched(err);
}

template <class TE, class TQ>
int score_typed(const smore_score_args& a, const void* table, const void* queries, const int32_t* ids, float* scores,
                hipStream_t st, const char** err)
{
    constexpr int V = 16 / sizeof(TE);
    if (a.dim < V) return score_as<TE, TQ, 16, 1, 1, 8>(a, table, queries, ids, scores, st, err);
    if (a.dim <= 16 * V) return score_as<TE, TQ, 16, V, 1, 8>(a, table, queries, ids, scores, st, err);
    if (a.dim <= 32 * V) return score_as<TE, TQ, 32, V, 1, 8>(a, table, queries, ids, scores, st, err);
    if (a.dim <= 64 * V) return score_as<TE, TQ, 64, V, 1, 8>(a, table, queries, ids, scores, st, err);
    return score_as<TE, TQ, 64, V, 2, 8>(a, table, queries, ids, scores, st, err);
}

// Workgroups that share a query: enough to fill the chip, each wavefront
// with at least 16 candidates.  us aimed at 256 / 512 / 1,024 / 2,048 workgroups:
// 16 x 4,001 of width 200 in bf16 10.9 / 9.4 / 9.1 / 9.0, 1 x 100,000 18.5 / 17.2 /
// 19.1 / 26.3, 256 x 500 of width 400 26.5 / 23.7 / 24.1 / 24.9; 511 x 257 in
// fp32 35.8 / 41.7 / 44.5 / 43.6.
void grad_split(const smore_score_args& a, int* splits, int* span)
{
    int64_t s = 1;
    while ((int64_t)a.batch * s < 512 && a.n > s * WAVES * 16) s *= 2;
    *span = (int)((a.n + s - 1) / s);
    *splits = *span > 0 ? (a.n + *span - 1) / *span : 1;
}

template <class TE, class TO, int LANES, int V, int NI, int UNROLL>
int grad_as(const smore_score_args& a, const void* table, const int32_t* ids, const float* grad, void* out, void* ws,
            hipStream_t st, const char** err)
{
    int splits, span;
    grad_split(a, &splits, &span);
    const dim3 grid((unsigned)((int64_t)a.batch * splits), (unsigned)((a.dim + LANES * V * NI - 1) / (LANES * V * NI)));
    k_score_grad<TE, TO, LANES, V, NI, UNROLL><<<grid, WG, 0, st>>>(
        (const TE*)table, a.table_stride, a.n_rows, a.dim, ids, a.candidate_stride, grad, a.score_stride, (TO*)out,
        a.query_stride, a.n, span, splits, (float*)ws);
    if (splits > 1) {
        k_join<TO><<<dim3((unsigned)a.batch, (unsigned)((a.dim + 63) / 64)), 1024, 0, st>>>((const float*)ws, splits, a.dim,
                                                                                           (TO*)out, a.query_stride);
    }
    return launched(err);
}

template <class TE, class TO>
int grad_typed(const smore_score_args& a, const void* table, const int32_t* ids, const float* grad, void* out, void* ws,
               hipStream_t st, const char** err)
{
    constexpr int V = 16 / sizeof(TE);
    if (a.dim < V) return grad_as<TE, TO, 16, 1, 1, 8>(a, table, ids, grad, out, ws, st, err);
    if (a.dim <= 16 * V) return grad_as<TE, TO, 16, V, 1, 8>(a, table, ids, grad, out, ws, st, err);
    if (a.dim <= 32 * V) return grad_as<TE, TO, 32, V, 1, 8>(a, table, ids, grad, out, ws, st, err);
    if (a.dim <= 64 * V) return grad_as<TE, TO, 64, V, 1, 8>(a, table, ids, grad, out, ws, st, err);
    return grad_as<TE, TO, 64, V, 2, 8>(a, table, ids, grad, out, ws, st, err);
}

}  // namespace

int launch_score(const smore_score_args& a, const void* table, const void* queries, const int32_t* ids, float* scores,
                 hipStream_t st, const char** err)
{
    const bool te = a.table_type == SMORE_BF16, tq = a.query_type == SMORE_BF16;
    if (te && tq) return score_typed<bf16, bf16>(a, table, queries, ids, scores, st, err);
    if (te) return score_typed<bf16, float>(a, table, queries, ids, scores, st, err);
    if (tq) return score_typed<float, bf16>(a, table, queries, ids, scores, st, err);
    return score_typed<float, float>(a, table, queries, ids, scores, st, err);
}

size_t score_grad_workspace(const smore_score_args& a)
{
    int splits, span;
    grad_split(a, &splits, &span);
    return splits > 1 ? (size_t)a.batch * splits * a.dim * sizeof(float) : 0;
}

int launch_score_grad(const smore_score_args& a, const void* table, const int32_t* ids, const float* grad, void* out,
                      void* ws, hipStream_t st, const char** err)
{
    const bool te = a.table_type == SMORE_BF16, to = a.query_type == SMORE_BF16;
    if (te && to) return grad_typed<bf16, bf16>(a, table, ids, grad, out, ws, st, err);
    if (te) return grad_typed<bf16, float>(a, table, ids, grad, out, ws, st, err);
    if (to) return grad_typed<float, bf16>(a, table, ids, grad, out, ws, st, err);
    return grad_typed<float, float>(a, table, ids, grad, out, ws, st, err);
}

}  // namespace smore
