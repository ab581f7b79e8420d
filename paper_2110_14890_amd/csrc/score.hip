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

// Columns [first, first + V) of a row that a lane holds in register block i,
// LANES lanes per row.  The last block of a row that is no multiple of V is
// moved back to end with the row: `skip` of its columns belong to the lane
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

// Elements of a row that a lane holds, as floats; columns of another lane 0.
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

template <class T, int LANES, int V, int NI>
__device__ __forceinline__ void fetch(const T* row, int lane, int tile0, int dim, bool real, Vec<T, V>* raw)
{
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const Columns<LANES, V> at(lane, i, tile0, dim);
        raw[i] = Vec<T, V>{};
        if (real && at.any) raw[i] = load_vec<T, V>(row + at.first);
    }
}

// A wavefront takes up to 64 candidates (`tile`) of one query.  Its lanes
// first read the ids, one each; then 64 / LANES rows at a time, UNROLL times
// over before the first is used, are multiplied with the query, which stays
// in registers, and summed over the LANES lanes.  Lane k keeps candidate k's
// score, so that the scores leave in one store.
template <class TE, class TQ, int LANES, int V, int NI, int UNROLL>
__global__ __launch_bounds__(WG) void k_score(const TE* __restrict__ table, int64_t table_stride, int V_rows, int dim,
                                              const TQ* __restrict__ queries, int64_t query_stride,
                                              const int32_t* __restrict__ ids, int64_t id_stride,
                                              float* __restrict__ out, int64_t out_stride, int batch, int n, int tile,
                                              int tiles)
{
    constexpr int GROUPS = 64 / LANES;
    const int lane = threadIdx.x & 63, sub = lane % LANES, group = lane / LANES;
    const int64_t w = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
    if (w >= (int64_t)batch * tiles) return;
    const int64_t b = w / tiles;
    const int k0 = (int)(w - b * tiles) * tile;
    const int count = min(tile, n - k0);
    int32_t id = -1;
    if (lane < count) id = ids[b * id_stride + k0 + lane];
    if (id >= V_rows) id = -1;
    const bool ragged = dim % V != 0;
    float score = 0.0f;
    for (int tile0 = 0; tile0 < dim; tile0 += LANES * V * NI) {
        Vec<TQ, V> q_raw[NI];
        float q[NI][V];
        fetch<TQ, LANES, V, NI>(queries + b * query_stride, sub, tile0, dim, true, q_raw);
        take<TQ, LANES, V, NI>(q_raw, sub, tile0, dim, ragged, q);
        for (int k = 0; k < count; k += GROUPS * UNROLL) {
            Vec<TE, V> raw[UNROLL][NI];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int at = k + u * GROUPS + group;
                int32_t e;
                if constexpr (LANES == 64) e = at < 64 ? __builtin_amdgcn_readlane(id, at & 63) : -1;
                else e = at < 64 ? __shfl(id, at & 63) : -1;
                fetch<TE, LANES, V, NI>(table + (int64_t)e * table_stride, sub, tile0, dim, e >= 0, raw[u]);
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                float x[NI][V], s = 0.0f;
                take<TE, LANES, V, NI>(raw[u], sub, tile0, dim, ragged, x);
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) s = fmaf(x[i][j], q[i][j], s);
                s = LANES == 64 ? sum64(s) : LANES == 32 ? sum32(s) : sum16(s);
                // the sum of group g goes to lane k + u GROUPS + g
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    const float sg = GROUPS == 1 ? s : __int_as_float(__builtin_amdgcn_readlane(__float_as_int(s), g * LANES));
                    if (lane == k + u * GROUPS + g) score += sg;
                }
            }
        }
    }
    if (lane < count) out[b * out_stride + k0 + lane] = id < 0 ? 0.0f : score;
}

// A workgroup takes one query's candidates [k0, k1) for LANES x V x NI of
// its columns; its wavefronts deal the candidates out 64 at a time and add
// their sums in LDS.  Several workgroups that share a query (splits > 1:
// few queries with long lists) write partial sums, which k_join adds.
template <class TE, class TO, int LANES, int V, int NI, int UNROLL>
__global__ __launch_bounds__(WG) void k_score_grad(const TE* __restrict__ table, int64_t table_stride, int V_rows, int dim,
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
    for (int base = k0 + wave * 64; base < k1; base += WAVES * 64) {
        const int count = min(64, k1 - base);
        int32_t id = -1;
        float g = 0.0f;
        if (lane < count) {
            id = ids[b * id_stride + base + lane];
            g = grad[b * grad_stride + base + lane];
        }
        if (id >= V_rows) id = -1;
        for (int k = 0; k < count; k += GROUPS * UNROLL) {
            Vec<TE, V> raw[UNROLL][NI];
            float w[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int at = k + u * GROUPS + group;
                int32_t e;
                if constexpr (LANES == 64) {
                    e = at < 64 ? __builtin_amdgcn_readlane(id, at & 63) : -1;
                    w[u] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g), at & 63));
                } else {
                    e = at < 64 ? __shfl(id, at & 63) : -1;
                    w[u] = __shfl(g, at & 63);
                }
                if (e < 0) w[u] = 0.0f;
                fetch<TE, LANES, V, NI>(table + (int64_t)e * table_stride, sub, tile0, dim, e >= 0, raw[u]);
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                float x[NI][V];
                take<TE, LANES, V, NI>(raw[u], sub, tile0, dim, ragged, x);
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[i][j] = fmaf(w[u], x[i][j], acc[i][j]);
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

template <class TO>
__global__ __launch_bounds__(WG) void k_join(const float* __restrict__ partial, int splits, int dim, TO* __restrict__ out,
                                             int64_t out_stride, int64_t total)
{
    const int64_t t = (int64_t)blockIdx.x * WG + threadIdx.x;
    if (t >= total) return;
    const int64_t b = t / dim, c = t - b * dim;
    float s = 0.0f;
    for (int k = 0; k < splits; ++k) s += partial[(b * splits + k) * dim + c];
    out[b * out_stride + c] = (TO)s;
}

template <class TE, class TQ, int LANES, int V, int NI, int UNROLL>
int score_as(const smore_score_args& a, const void* table, const void* queries, const int32_t* ids, float* scores,
             hipStream_t st, const char** err)
{
    // candidates per wavefront: 64, fewer where that leaves CUs without work
    int tile = 64;
    while (tile > 8 && (int64_t)a.batch * ((a.n + tile - 1) / tile) < 4096) tile /= 2;
    const int tiles = (a.n + tile - 1) / tile;
    const int64_t blocks = ((int64_t)a.batch * tiles + WAVES - 1) / WAVES;
    k_score<TE, TQ, LANES, V, NI, UNROLL><<<(unsigned)blocks, WG, 0, st>>>(
        (const TE*)table, a.table_stride, a.n_rows, a.dim, (const TQ*)queries, a.query_stride, ids, a.candidate_stride,
        scores, a.score_stride, a.batch, a.n, tile, tiles);
    return launched(err);
}

template <class TE, class TQ>
int score_typed(const smore_score_args& a, const void* table, const void* queries, const int32_t* ids, float* scores,
                hipStream_t st, const char** err)
{
    constexpr int V = 16 / sizeof(TE);
    if (a.dim < V) return score_as<TE, TQ, 16, 1, 1, 4>(a, table, queries, ids, scores, st, err);
    if (a.dim <= 16 * V) return score_as<TE, TQ, 16, V, 1, 4>(a, table, queries, ids, scores, st, err);
    if (a.dim <= 32 * V) return score_as<TE, TQ, 32, V, 1, 8>(a, table, queries, ids, scores, st, err);
    if (a.dim <= 64 * V) return score_as<TE, TQ, 64, V, 1, 8>(a, table, queries, ids, scores, st, err);
    return score_as<TE, TQ, 64, V, 2, 4>(a, table, queries, ids, scores, st, err);
}

// Workgroups that share a query: enough to fill the chip, each wavefront
// with at least 8 candidates.
void grad_split(const smore_score_args& a, int* splits, int* span)
{
    int64_t s = 1;
    while ((int64_t)a.batch * s < 2048 && a.n > s * WAVES * 8) s *= 2;
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
        const int64_t total = (int64_t)a.batch * a.dim;
        k_join<TO><<<(unsigned)((total + WG - 1) / WG), WG, 0, st>>>((const float*)ws, splits, a.dim, (TO*)out, a.query_stride,
                                                                     total);
    }
    return launched(err);
}

template <class TE, class TO>
int grad_typed(const smore_score_args& a, const void* table, const int32_t* ids, const float* grad, void* out, void* ws,
               hipStream_t st, const char** err)
{
    constexpr int V = 16 / sizeof(TE);
    if (a.dim < V) return grad_as<TE, TO, 16, 1, 1, 4>(a, table, ids, grad, out, ws, st, err);
    if (a.dim <= 16 * V) return grad_as<TE, TO, 16, V, 1, 4>(a, table, ids, grad, out, ws, st, err);
    if (a.dim <= 32 * V) return grad_as<TE, TO, 32, V, 1, 8>(a, table, ids, grad, out, ws, st, err);
    if (a.dim <= 64 * V) return grad_as<TE, TO, 64, V, 1, 8>(a, table, ids, grad, out, ws, st, err);
    return grad_as<TE, TO, 64, V, 2, 4>(a, table, ids, grad, out, ws, st, err);
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
