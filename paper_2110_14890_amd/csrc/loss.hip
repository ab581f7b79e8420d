// loss.hip -- preference loss of each query's positive against its verified
// negatives, with its gradient.
//
//   z_k = beta ((pos - ref_pos) - (neg_k - ref_neg_k))     paired log ratios
//   pairs:   L = 1/c sum_k (1 - eps) softplus(-z_k) + eps softplus(z_k)
//            dL/dz_k = (eps - sigma(-z_k)) / c
//   softmax: L = log(1 + sum_k exp(-z_k))
//            dL/dz_k = -exp(-z_k) / (1 + sum_j exp(-z_j))
//   dL/dpos = beta sum_k dL/dz_k,   dL/dneg_k = -beta dL/dz_k
//
// over the c valid negatives of a row: the first n_valid[b], or those whose
// bit is set.  A row without any has loss 0 and gradient 0, and no score of a
// place that is not valid is used.  Scores, reference scores and gradients
// pass once each; about 40 operations per score (exponential, logarithm and
// reciprocal among them) are near what the bytes leave time for.
#include <hip/hip_runtime.h>

#include "numeric.h"
#include "smore_internal.h"

namespace smore {
namespace {

constexpr int WG = 256;

struct LossRow {
    const void *pos, *neg, *ref_pos, *ref_neg;
    int64_t pos_stride, neg_stride, ref_pos_stride, ref_neg_stride;
    const int32_t* n_valid;
    const uint32_t* mask;
    const float* weight;
    float* loss;
    void *grad_pos, *grad_neg;
    int64_t grad_pos_stride, grad_neg_stride;
    int32_t batch, n, words;
    float beta, eps, scale;
};

constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f;

// All ones where bit j of the valid places is set, else 0.
__device__ __forceinline__ uint32_t ones(uint32_t ok, int j) { return (uint32_t)((int32_t)(ok << (31 - j)) >> 31); }
__device__ __forceinline__ float keep(uint32_t ok, int j, float x) { return __uint_as_float(__float_as_uint(x) & ones(ok, j)); }

// Sum over the WAVES wavefronts of a row of a value that every lane of a
// wavefront has.
template <int WAVES, class F>
__device__ __forceinline__ float across(float x, float* lds, int wave, F join)
{
    if constexpr (WAVES == 1) return x;
    __syncthreads();   // the last use of lds is over
    if ((threadIdx.x & 63) == 0) lds[wave] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) x = join(x, lds[w]);
    return x;
}

// WAVES wavefronts per row, each lane V consecutive scores in each of STEPS
// blocks: rows of up to 64 x WAVES x V x STEPS scores stay in registers
// between the sum and the gradient; longer ones are read again.  Gradients
// are rounded once, to the scores' type.  16,384 x 512 in bf16 with reference
// scores, softmax: 13.2 us (3.8 TB/s); 8,192 x 512 in fp32 with masks, pairs:
// 11.5 us, a third of the issue slots; 64 x 16: 3.6 us, the launch.
template <class T, int WAVES, int V, int STEPS, bool SOFTMAX, bool REF, bool GRAD>
__global__ __launch_bounds__(WG) void k_loss(const LossRow a)
{
    constexpr int BLOCK = 64 * WAVES * V, SPAN = BLOCK * STEPS;
    __shared__ float lds[4];
    const int lane = threadIdx.x & 63;
    const int wave = WAVES == 1 ? 0 : threadIdx.x >> 6;
    const int64_t b = WAVES == 1 ? (int64_t)blockIdx.x * (WG / 64) + (threadIdx.x >> 6) : (int64_t)blockIdx.x;
    if (b >= a.batch) return;
    const int my = (wave * 64 + lane) * V;
    const uint32_t* bits = a.mask ? a.mask + b * a.words : nullptr;
    const int limit = a.n_valid ? max(0, min(a.n_valid[b], a.n)) : a.n;

    float count = (float)limit;
    if (!SOFTMAX && bits) {
        int c = 0;
        for (int w = wave * 64 + lane; w < a.words; w += 64 * WAVES) {
            const int left = a.n - 32 * w;
            c += __popc(left < 32 ? bits[w] & ((1u << left) - 1u) : bits[w]);
        }
        count = across<WAVES>(sum64((float)c), lds, wave, [](float x, float y) { return x + y; });
    }
    const float share = count > 0.0f ? 1.0f / count : 0.0f;

    const T* neg = (const T*)a.neg + b * a.neg_stride;
    const T* ref = (const T*)a.ref_neg + (REF ? b * a.ref_neg_stride : 0);
    float base = (float)((const T*)a.pos)[b * a.pos_stride];
    if (REF) base -= (float)((const T*)a.ref_pos)[b * a.ref_pos_stride];
    const float gain = GRAD ? a.beta * a.scale * (a.weight ? a.weight[b] : 1.0f) : 0.0f;

    // d = the log ratio of a negative over the positive's; z = -beta d
    float d[STEPS][V];
    uint32_t ok[STEPS];   // bit j: score j of the block is valid
    bool full;            // every place of the wavefront's blocks is
    auto fetch = [&](int at0) {
        float x[STEPS][V], r[STEPS][V];
        uint32_t both = (1u << V) - 1u;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int k = at0 + s * BLOCK + my;
            ok[s] = 0;
            if (k < limit) {
                ok[s] = (1u << min(V, limit - k)) - 1u;
                if (bits) ok[s] &= bits[k >> 5] >> (k & 31);
            }
            both &= ok[s];
#pragma unroll
            for (int j = 0; j < V; ++j) x[s][j] = r[s][j] = 0.0f;
            if (ok[s]) {
                load_floats<T, V>(neg + k, a.n - k, x[s]);
                if (REF) load_floats<T, V>(ref + k, a.n - k, r[s]);
            }
        }
        full = __all(both == (1u << V) - 1u);
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int j = 0; j < V; ++j) d[s][j] = (REF ? x[s][j] - r[s][j] : x[s][j]) - base;
    };
    T* grad = GRAD ? (T*)a.grad_neg + b * a.grad_neg_stride : nullptr;

    if constexpr (!SOFTMAX) {
        float loss = 0.0f, slopes = 0.0f;
        const float unit = share * gain;
        for (int at0 = 0; at0 < a.n; at0 += SPAN) {
            fetch(at0);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int k = at0 + s * BLOCK + my;
                float l[V], g[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float y = a.beta * d[s][j];                                  // -z
                    const float e = __builtin_amdgcn_exp2f(-LOG2E * fabsf(y));         // exp(-|z|)
                    const float u = 1.0f + e, r = __builtin_amdgcn_rcpf(u);
                    // log(1 + e): the logarithm of u and what u lost of e
                    const float tail = fmaf(__builtin_amdgcn_logf(u), LN2, (e - (u - 1.0f)) * r);
                    l[j] = fmaxf(y, 0.0f);
                    if (a.eps != 0.0f) l[j] = fmaf(a.eps, fmaxf(-y, 0.0f), (1.0f - a.eps) * l[j]);
                    l[j] += tail;
                    if (GRAD) g[j] = ((y <= 0.0f ? e : 1.0f) * r - a.eps) * unit;     // sigma(-z)
                }
                if (!full) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        l[j] = keep(ok[s], j, l[j]);
                        if (GRAD) g[j] = keep(ok[s], j, g[j]);
                    }
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    loss += l[j];
                    if (GRAD) slopes -= g[j];
                }
                if (GRAD && k < a.n) store_floats<T, V>(grad + k, a.n - k, g);
            }
        }
        loss = across<WAVES>(sum64(loss), lds, wave, [](float x, float y) { return x + y; });
        if (GRAD) slopes = across<WAVES>(sum64(slopes), lds, wave, [](float x, float y) { return x + y; });
        if (lane == 0 && wave == 0) {
            if (a.loss) a.loss[b] = loss * share;
            if (GRAD) ((T*)a.grad_pos)[b * a.grad_pos_stride] = (T)slopes;
        }
    } else {
        // running maximum of -z (of 0, the positive's own term, on) and sum of
        // each lane.  The base's factor comes behind the difference: in front of
        // it a -z above 2.3e38 (a positive at its type's lowest value) overflows.
        float top = 0.0f, sum = 0.0f;
        float e[STEPS][V];
        auto exponents = [&](int at0) {
            fetch(at0);
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int j = 0; j < V; ++j) e[s][j] = a.beta * d[s][j];
            if (!full) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const uint32_t m = ones(ok[s], j);
                        e[s][j] = __uint_as_float((__float_as_uint(e[s][j]) & m) | (0xFF800000u & ~m));   // or -infinity
                    }
            }
        };
        for (int at0 = 0; at0 < a.n; at0 += SPAN) {
            exponents(at0);
            float m = top;
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int j = 0; j < V; ++j) m = fmaxf(m, e[s][j]);
            sum *= __builtin_amdgcn_exp2f(LOG2E * (top - m));
            top = m;
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    e[s][j] = __builtin_amdgcn_exp2f(LOG2E * (e[s][j] - top));
                    sum += e[s][j];
                }
        }
        float high = across<WAVES>(max64(top), lds, wave, [](float x, float y) { return fmaxf(x, y); });
        const float mine = __builtin_amdgcn_exp2f(LOG2E * (top - high));
        sum = across<WAVES>(sum64(sum * mine), lds, wave, [](float x, float y) { return x + y; });
        const float total = __builtin_amdgcn_exp2f(-LOG2E * high) + sum;
        if (lane == 0 && wave == 0) {
            if (a.loss) a.loss[b] = high > 0.0f ? high + __logf(total) : log1pf(sum);
            if (GRAD) ((T*)a.grad_pos)[b * a.grad_pos_stride] = (T)(sum == 0.0f ? 0.0f : -gain * (sum / total));
        }
        if constexpr (GRAD) {
            const float unit = mine * (gain / total);
            for (int at0 = 0; at0 < a.n; at0 += SPAN) {
                if (a.n > SPAN) {
                    exponents(at0);
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
#pragma unroll
                        for (int j = 0; j < V; ++j) e[s][j] = __builtin_amdgcn_exp2f(LOG2E * (e[s][j] - top));
                }
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const int k = at0 + s * BLOCK + my;
                    float g[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) g[j] = e[s][j] * unit;
                    if (!full) {      // a unit that is not finite stays out of places that are not valid
#pragma unroll
                        for (int j = 0; j < V; ++j) g[j] = keep(ok[s], j, g[j]);
                    }
                    if (k < a.n) store_floats<T, V>(grad + k, a.n - k, g);
                }
            }
        }
    }
}

template <class T, bool SOFTMAX, bool REF, bool GRAD>
int loss_as(const LossRow& a, hipStream_t st, const char** err)
{
    // A wavefront a row while its scores fit its registers, then a workgroup.
    // us of the four forms, in the order below, pairs / softmax with gradient, in
    // fp32 (V = 4):
    //   256 rows     of 64 V 3.5 3.7 4.1 4.6 / 3.5 3.7 4.0 4.3   512 V 7.0 7.0 4.3 4.9 / 8.3 7.7 4.3 4.6
    //   4,096 rows   of 64 V 4.5 5.3 11 17 / 4.5 4.9 8.8 12      128 V 5.9 6.3 11 17 / 5.9 5.6 9.2 12
    //                256 V 9.1 9.9 12 17 / 8.7 9.1 10 13         512 V 14 15 17 20 / 17 16 15 15
    //                1,024 V 26 28 25 27 / 35 34 30 24
    // Few rows of 129 V to 512 V need the workgroup; where rows alone fill the
    // chip, up to 384 V, one wavefront would be faster by up to 1.4 times here,
    // 2.3 times at 16,384 rows of 192 V in bf16 (56 against 24 us).
    constexpr int V = 16 / sizeof(T);
    const unsigned rows4 = (unsigned)((a.batch + 3) / 4);
    if (a.n <= 64 * V) k_loss<T, 1, V, 1, SOFTMAX, REF, GRAD><<<rows4, WG, 0, st>>>(a);
    else if (a.n <= 128 * V) k_loss<T, 1, V, 2, SOFTMAX, REF, GRAD><<<rows4, WG, 0, st>>>(a);
    else if (a.n <= 512 * V) k_loss<T, 4, V, 2, SOFTMAX, REF, GRAD><<<(unsigned)a.batch, WG, 0, st>>>(a);
    else k_loss<T, 4, V, 4, SOFTMAX, REF, GRAD><<<(unsigned)a.batch, WG, 0, st>>>(a);
    return launched(err);
}

template <class T>
int loss_typed(const LossRow& a, bool softmax, hipStream_t st, const char** err)
{
    const bool ref = a.ref_pos != nullptr, grad = a.grad_pos != nullptr;
    if (softmax) {
        if (ref) return grad ? loss_as<T, true, true, true>(a, st, err) : loss_as<T, true, true, false>(a, st, err);
        return grad ? loss_as<T, true, false, true>(a, st, err) : loss_as<T, true, false, false>(a, st, err);
    }
    if (ref) return grad ? loss_as<T, false, true, true>(a, st, err) : loss_as<T, false, true, false>(a, st, err);
    return grad ? loss_as<T, false, false, true>(a, st, err) : loss_as<T, false, false, false>(a, st, err);
}

}  // namespace

int launch_preference(const smore_preference_args& p, const smore_preference_in& in, const smore_preference_out& out,
                      hipStream_t st, const char** err)
{
    LossRow a{};
    a.pos = in.positive;
    a.neg = in.negatives;
    a.ref_pos = in.ref_positive;
    a.ref_neg = in.ref_negatives;
    a.pos_stride = p.positive_stride;
    a.neg_stride = p.negatives_stride;
    a.ref_pos_stride = p.ref_positive_stride;
    a.ref_neg_stride = p.ref_negatives_stride;
    a.n_valid = in.n_valid;
    a.mask = in.mask;
    a.weight = in.weight;
    a.loss = out.loss;
    a.grad_pos = out.grad_positive;
    a.grad_neg = out.grad_negatives;
    a.grad_pos_stride = p.grad_positive_stride;
    a.grad_neg_stride = p.grad_negatives_stride;
    a.batch = p.batch;
    a.n = p.n;
    a.words = (p.n + 31) / 32;
    a.beta = p.beta;
    a.eps = p.smoothing;
    a.scale = p.scale;
    const bool softmax = p.kind == SMORE_PREFERENCE_SOFTMAX;
    if (p.score_type == SMORE_BF16) return loss_typed<bf16>(a, softmax, st, err);
    if (p.score_type == SMORE_F16) return loss_typed<f16>(a, softmax, st, err);
    return loss_typed<float>(a, softmax, st, err);
}

}  // namespace smore
