// adamw.hip -- AdamW over many tensors at once, and over the rows of
// embedding tables that a batch touched.
//
//   m = b1 m + (1 - b1) g          v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
//
// Every value passes once: 28 bytes an element in 32 bits, 10 with bf16
// parameters and gradients and 8-bit moments, so the kernels are bound by
// HBM bandwidth.
//
// Moments in 8 bits: e4m3 codes of m and of sqrt(v), relative to the largest
// magnitude of 128 consecutive elements of a row (scale = largest / 448).
// The square root halves the range that a code has to span; a code's step
// is 1/16 to 1/8 of its value, far more than a moment changes in a step
// (1 - b2 = 0.001), so rounding to the nearest would leave most moments
// where they are.  They are rounded stochastically instead, up with the
// probability of the remainder, which is right in the mean.  A sqrt(v) that
// is not 0 never gets the code 0, so that no later step divides by eps alone.
// A value that is not finite makes the scale of its 128 elements NaN.
// Parameters in bf16 are rounded the same way.  The random bits are a hash
// of (seed, step, tensor, block, element): nothing is kept between calls.
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "numeric.h"
#include "smore_internal.h"

namespace smore {
namespace {

constexpr int WG = 256;
constexpr int WAVES = WG / 64;
constexpr int PER = 4;                  // consecutive elements of a lane
constexpr int CHUNK = 64 * PER;         // elements of a wavefront: two blocks of 128
constexpr int BLOCK = SMORE_ADAMW_BLOCK;
constexpr int CHUNKS = 4;               // chunks of a wavefront in a dense tensor
constexpr int RUN = 128;                // entries whose sum is made ahead in long runs

struct Hyper {
    float lr, b1, b2, eps, c1, c2;      // c1 = 1 - b1^t, c2 = 1 - b2^t where the step is given
    float log_b1, log_b2;
    const int64_t* step;                // step, rate and gradient scale on the device, or NULL
    const float* lr_dev;
    const float* grad_scale;
    int64_t step_host;
    uint64_t seed;
    int32_t stochastic;
};

struct Tensor {
    void* p;
    const void* g;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t count;                      // elements
    uint32_t first_wg;
    int32_t index;
    float decay;
};
// Tensors of a launch travel in its arguments (4 KB at most), so that a call
// needs no copy to the device and a captured graph keeps them.
constexpr int MAX_TENSORS = 48;
struct TensorList {
    Tensor t[MAX_TENSORS];
    int32_t n;
};

struct RowsTensor {
    Tensor t;
    const int32_t* rows;
    const int64_t* order;
    const float* coef;
    const float* partial;
    int64_t n_rows, dim, n_entries, per;
};

__device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}

// One step's constants and the key of one tensor's roundings.
struct Step {
    float rate, keep, b1, b2, eps, r1, r2, scale;   // r1 = 1 / c1, r2 = 1 / c2
    uint32_t key;
    bool stochastic, skip;
    __device__ Step(const Hyper& h, float decay, int32_t index)
    {
        const int64_t t = h.step ? *h.step : h.step_host;
        const float c1 = h.step ? -expm1f((float)t * h.log_b1) : h.c1;
        const float c2 = h.step ? -expm1f((float)t * h.log_b2) : h.c2;
        rate = h.lr_dev ? *h.lr_dev : h.lr;
        keep = 1.0f - rate * decay;
        b1 = h.b1;
        b2 = h.b2;
        eps = h.eps;
        r1 = 1.0f / c1;
        r2 = 1.0f / c2;
        scale = h.grad_scale ? *h.grad_scale : 1.0f;
        skip = !(fabsf(scale) < INFINITY);
        stochastic = h.stochastic != 0;
        uint32_t k = mix(mix((uint32_t)h.seed) ^ (uint32_t)(h.seed >> 32));
        k = mix(mix(k + (uint32_t)t) ^ (uint32_t)((uint64_t)t >> 32));
        key = mix(k + (uint32_t)index);
    }
};

// Codes: e4m3 (4 exponent bits, 3 fraction bits, no infinity), y in [0, 448].
// A value's bits above the fraction's are its code, once the exponent's bias
// is moved from 127 to 7; below 2^-6 codes are multiples of 2^-9.
__device__ __forceinline__ uint32_t encode(float y, uint32_t draw, bool stochastic)
{
    const uint32_t bits = __float_as_uint(y);
    const float fine = y * 512.0f;
    uint32_t up, small;
    if (stochastic) {
        up = draw << 4;
        const float whole = floorf(fine);
        small = (uint32_t)whole + ((fine - whole) * 65536.0f + (float)draw >= 65536.0f ? 1u : 0u);
    } else {
        up = 0x7FFFFu + ((bits >> 20) & 1u);
        small = (uint32_t)rintf(fine);
    }
    const uint32_t code = y < 0.015625f ? small : ((bits + up) >> 20) - (120u << 3);
    return code < 0x7Eu ? code : 0x7Eu;
}

// Values of four codes.
__device__ __forceinline__ void decode(uint32_t four, float* out)
{
    out[0] = __builtin_amdgcn_cvt_f32_fp8((int)four, 0);
    out[1] = __builtin_amdgcn_cvt_f32_fp8((int)four, 1);
    out[2] = __builtin_amdgcn_cvt_f32_fp8((int)four, 2);
    out[3] = __builtin_amdgcn_cvt_f32_fp8((int)four, 3);
}

// Largest magnitude of the 32 lanes of a block, as bits: NaN above infinity
// above every number.
__device__ __forceinline__ uint32_t block_max(uint32_t x)
{
#define SMORE_STEP(CTRL) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true))
    SMORE_STEP(DPP_XOR1);
    SMORE_STEP(DPP_XOR2);
    SMORE_STEP(DPP_MIRROR8);
    SMORE_STEP(DPP_MIRROR16);
#undef SMORE_STEP
    return max(x, (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x401F));   // lane ^ 16
}

// Scale of a block and the factor that takes its values to [0, 448].
__device__ __forceinline__ void block_scale(uint32_t top_bits, float* scale, float* unit)
{
    const float top = __uint_as_float(top_bits);
    if (top_bits >= 0x7F800000u) {
        *scale = __uint_as_float(0x7FC00000u);
        *unit = 0.0f;
    } else if (top < 1.17549435e-38f) {
        *scale = *unit = 0.0f;
    } else {
        *scale = top / 448.0f;
        *unit = 448.0f / top;
    }
}

__device__ __forceinline__ float to_param(float p, uint32_t, bool, float) { return p; }
__device__ __forceinline__ bf16 to_param(float p, uint32_t draw, bool stochastic, bf16)
{
    if (!stochastic || !(fabsf(p) < INFINITY)) return (bf16)p;
    const uint32_t up = ((draw ^ 0x85EBCA6Bu) * 0x9E3779B1u) >> 16;
    const uint16_t top = (uint16_t)((__float_as_uint(p) + up) >> 16);
    bf16 out;
    __builtin_memcpy(&out, &top, sizeof(out));
    return out;
}

// Elements and moments of a chunk that a lane holds.
template <int BITS>
struct Held;
template <>
struct Held<32> {
    float m[PER], v[PER];
};
template <>
struct Held<8> {
    uint32_t m, v;
    float m_scale, v_scale;
};

__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t have)
{
    uint32_t x = 0;
    if (have >= PER) {
        __builtin_memcpy(&x, p, 4);
    } else {
#pragma unroll
        for (int j = 0; j < PER - 1; ++j)
            if (j < have) x |= (uint32_t)p[j] << (8 * j);
    }
    return x;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t have, uint32_t x)
{
    if (have >= PER) {
        __builtin_memcpy(p, &x, 4);
    } else {
#pragma unroll
        for (int j = 0; j < PER - 1; ++j)
            if (j < have) p[j] = (uint8_t)(x >> (8 * j));
    }
}

// at: the lane's first element in the tensor; have: how many of its PER
// elements the row has (none: <= 0); scale_at: its block's scale.
template <int BITS>
__device__ __forceinline__ void load_held(const Tensor& t, int64_t at, int64_t have, int64_t scale_at, Held<BITS>& h)
{
    if constexpr (BITS == 32) {
        load_floats<float, PER>((const float*)t.m + at, have, h.m);
        load_floats<float, PER>((const float*)t.v + at, have, h.v);
    } else {
        h.m = load_codes((const uint8_t*)t.m + at, have);
        h.v = load_codes((const uint8_t*)t.v + at, have);
        h.m_scale = have > 0 ? t.m_scale[scale_at] : 0.0f;
        h.v_scale = have > 0 ? t.v_scale[scale_at] : 0.0f;
    }
}

// Steps a lane's PER elements and writes them back.  Every lane of the
// wavefront takes part (the maxima of the 8-bit blocks).  block: number of
// the 128-element block; j0: the lane's first element in it.
template <class TP, int BITS>
__device__ __forceinline__ void step_held(const Tensor& t, const Step& s, int64_t at, int64_t have, int64_t block, int j0,
                                          float* p, const float* g, Held<BITS>& h)
{
    float m[PER], v[PER];
    if constexpr (BITS == 32) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            m[j] = h.m[j];
            v[j] = h.v[j];
        }
    } else {
        decode(h.m, m);
        decode(h.v, v);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            m[j] *= h.m_scale;
            v[j] *= h.v_scale;
            v[j] *= v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const float gj = g[j] * s.scale;
        m[j] = s.b1 * m[j] + (1.0f - s.b1) * gj;
        v[j] = s.b2 * v[j] + (1.0f - s.b2) * (gj * gj);
        p[j] = p[j] * s.keep - s.rate * ((m[j] * s.r1) / (sqrtf(v[j] * s.r2) + s.eps));
    }
    constexpr bool DRAWS = BITS == 8 || sizeof(TP) == 2;
    uint32_t draw[PER] = {};
    if (DRAWS && s.stochastic) {
        const uint32_t base = mix(mix(s.key ^ (uint32_t)block) + (uint32_t)((uint64_t)block >> 32));
#pragma unroll
        for (int j = 0; j < PER; ++j) draw[j] = mix(base + (uint32_t)(j0 + j));
    }
    if (have > 0) {
        Vec<TP, PER> out;
#pragma unroll
        for (int j = 0; j < PER; ++j) out.x[j] = to_param(p[j], draw[j], s.stochastic, TP{});
        TP* dst = (TP*)t.p + at;
        if (have >= PER) {
            store_vec<TP, PER>(dst, out);
        } else {
#pragma unroll
            for (int j = 0; j < PER - 1; ++j)
                if (j < have) dst[j] = out.x[j];
        }
    }
    if constexpr (BITS == 32) {
        if (have > 0) {
            store_floats<float, PER>((float*)t.m + at, have, m);
            store_floats<float, PER>((float*)t.v + at, have, v);
        }
    } else {
        uint32_t m_top = 0, v_top = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (j >= have) m[j] = v[j] = 0.0f;
            v[j] = sqrtf(v[j]);
            m_top = max(m_top, __float_as_uint(m[j]) & 0x7FFFFFFFu);
            v_top = max(v_top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
        }
        float m_scale, m_unit, v_scale, v_unit;
        block_scale(block_max(m_top), &m_scale, &m_unit);
        block_scale(block_max(v_top), &v_scale, &v_unit);
        uint32_t mc = 0, vc = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint32_t a = encode(fabsf(m[j]) * m_unit, draw[j] & 0xFFFFu, s.stochastic);
            uint32_t b = encode(v[j] * v_unit, draw[j] >> 16, s.stochastic);
            if (v[j] != 0.0f && v_unit > 0.0f) b = max(b, 1u);
            mc |= (a | (m[j] < 0.0f ? 0x80u : 0u)) << (8 * j);
            vc |= b << (8 * j);
        }
        if (have > 0) {
            store_codes((uint8_t*)t.m + at, have, mc);
            store_codes((uint8_t*)t.v + at, have, vc);
            if (j0 == 0) {
                t.m_scale[block] = m_scale;
                t.v_scale[block] = v_scale;
            }
        }
    }
}

// A workgroup takes WAVES x CHUNKS chunks of one tensor; which one it finds
// among the launch's tensors by their first workgroups.
template <class TP, class TG, int BITS>
__global__ __launch_bounds__(WG) void k_adamw(const TensorList list, const Hyper hyper)
{
    int lo = 0, hi = list.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (list.t[mid].first_wg <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const Tensor& t = list.t[lo];
    const Step s(hyper, t.decay, t.index);
    if (s.skip) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t base = ((int64_t)(blockIdx.x - t.first_wg) * WAVES + wave) * (CHUNK * CHUNKS) + lane * PER;
    float p[CHUNKS][PER], g[CHUNKS][PER];
    Held<BITS> h[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int64_t at = base + c * CHUNK, have = t.count - at;
        load_floats<TP, PER>((const TP*)t.p + at, have, p[c]);
        load_floats<TG, PER>((const TG*)t.g + at, have, g[c]);
        load_held<BITS>(t, at, have, at / BLOCK, h[c]);
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int64_t at = base + c * CHUNK;
        step_held<TP, BITS>(t, s, at, t.count - at, at / BLOCK, (int)(at % BLOCK), p[c], g[c], h[c]);
    }
}

// Gradient of a table row: the entries of the sorted list that name it, each
// coef[order[i]] times the vector order[i] / per.
template <class TG>
__device__ __forceinline__ void add_entries(const RowsTensor& r, int64_t first, int64_t end, int64_t col, int64_t have,
                                            float* g)
{
    const int lane = threadIdx.x & 63;
    for (int64_t at = first; at < end; at += 64) {
        const int n = (int)min((int64_t)64, end - at);
        int64_t from = 0;
        float w = 0.0f;
        if (lane < n) {
            const int64_t o = r.order ? r.order[at + lane] : at + lane;
            if (o >= 0 && o < r.n_entries) {   // a permutation's: reads nothing behind the gradients otherwise
                w = r.coef ? r.coef[o] : 1.0f;
                from = r.per == 1 ? o : o / r.per;
            }
        }
        for (int i = 0; i < n; ++i) {
            const int64_t src = ((int64_t)(uint32_t)__builtin_amdgcn_readlane((int)(from >> 32), i) << 32) |
                                (uint32_t)__builtin_amdgcn_readlane((int)from, i);
            const float wi = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), i));
            float x[PER];
            load_floats<TG, PER>((const TG*)r.t.g + src * r.dim + col, have, x);
#pragma unroll
            for (int j = 0; j < PER; ++j) g[j] = fmaf(wi, x[j], g[j]);
        }
    }
}

// Sums of RUN consecutive entries of one row, where a run is that long, so
// that no wavefront has to add a hub's entries one by one.
template <class TG>
__global__ __launch_bounds__(WG) void k_run_sums(const RowsTensor r, float* __restrict__ partial)
{
    const int lane = threadIdx.x & 63;
    const int64_t c = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
    if ((c + 1) * RUN > r.n_entries) return;
    const int32_t row = r.rows[c * RUN];
    if (row < 0 || row >= r.n_rows || r.rows[c * RUN + RUN - 1] != row) return;
    for (int64_t col = lane * PER; col - lane * PER < r.dim; col += CHUNK) {
        const int64_t have = r.dim - col;
        float g[PER] = {};
        add_entries<TG>(r, c * RUN, (c + 1) * RUN, col, have, g);
        if (have > 0) store_floats<float, PER>(partial + c * r.dim + col, have, g);
    }
}

// A wavefront per entry; the first entry of a row's run takes the row.
template <class TP, class TG, int BITS>
__global__ __launch_bounds__(WG) void k_adamw_rows(const RowsTensor r, const Hyper hyper)
{
    const int lane = threadIdx.x & 63;
    const int64_t i = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
    if (i >= r.n_entries) return;
    const int32_t row = r.rows[i];
    if (row < 0 || row >= r.n_rows || (i > 0 && r.rows[i - 1] == row)) return;
    const Step s(hyper, r.t.decay, r.t.index);
    if (s.skip) return;
    // [i, head): entries up to the run's end or the first sum made ahead;
    // then `sums` of those; then [tail, end)
    int64_t head = i + 1;
    int sums = 0;
    int64_t tail = 0, end = 0;
    if (i + 1 < r.n_entries && r.rows[i + 1] == row) {
        const int64_t next = (i + RUN - 1) / RUN * RUN;
        bool open = true;
        auto walk = [&](int64_t from, int64_t to) {   // the run's end within [from, to)
            while (open && from < to) {
                const uint64_t same = __ballot(from + lane < to && r.rows[min(from + lane, r.n_entries - 1)] == row);
                const int n = same == ~0ull ? 64 : __builtin_ctzll(~same);
                from += n;
                if (n < 64) open = from >= to;
            }
            return min(from, to);
        };
        head = walk(i, min(next, r.n_entries));
        if (open && next < r.n_entries) {
            int64_t c = next / RUN;
            for (;;) {
                const int64_t last = (c + lane + 1) * RUN - 1;
                const uint64_t same = __ballot(last < r.n_entries && r.rows[min(last, r.n_entries - 1)] == row);
                const int n = same == ~0ull ? 64 : __builtin_ctzll(~same);
                sums += n;
                c += n;
                if (n < 64) break;
            }
            tail = next + (int64_t)sums * RUN;
            end = walk(tail, min(tail + RUN, r.n_entries));
        }
    }
    const int64_t blocks = (r.dim + BLOCK - 1) / BLOCK;
    for (int64_t col = lane * PER; col - lane * PER < r.dim; col += CHUNK) {
        const int64_t have = r.dim - col, at = (int64_t)row * r.dim + col, block = row * blocks + col / BLOCK;
        float p[PER], g[PER] = {};
        Held<BITS> h;
        load_floats<TP, PER>((const TP*)r.t.p + at, have, p);
        load_held<BITS>(r.t, at, have, block, h);
        add_entries<TG>(r, i, head, col, have, g);
        const float* from = r.partial + (tail / RUN - sums) * r.dim + col;
        for (int k = 0; k < sums; ++k, from += r.dim) {
            float x[PER];
            load_floats<float, PER>(from, have, x);
#pragma unroll
            for (int j = 0; j < PER; ++j) g[j] += x[j];
        }
        add_entries<TG>(r, tail, end, col, have, g);
        step_held<TP, BITS>(r.t, s, at, have, block, (int)(col % BLOCK), p, g, h);
    }
}

template <class TP, class TG, int BITS>
int dense_as(const smore_adamw_tensor* ts, int n, const Hyper& h, hipStream_t st, const char** err)
{
    TensorList list;
    list.n = 0;
    uint64_t wgs = 0;
    auto flush = [&] {
        if (list.n) k_adamw<TP, TG, BITS><<<(unsigned)wgs, WG, 0, st>>>(list, h);
        list.n = 0;
        wgs = 0;
    };
    constexpr int64_t SPAN = (int64_t)CHUNK * CHUNKS * WAVES;
    for (int k = 0; k < n; ++k) {
        const smore_adamw_tensor& x = ts[k];
        const int64_t count = x.n_rows * x.dim;
        const int64_t need = (count + SPAN - 1) / SPAN;
        if (list.n == MAX_TENSORS || wgs + need > (1u << 23)) flush();
        list.t[list.n++] = Tensor{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, count, (uint32_t)wgs, x.index, x.weight_decay};
        wgs += need;
    }
    flush();
    return launched(err);
}

template <class TP, class TG, int BITS>
int rows_as(const smore_adamw_tensor& x, const Hyper& h, float* partial, hipStream_t st, const char** err)
{
    RowsTensor r{};
    r.t = Tensor{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, 0, 0, x.index, x.weight_decay};
    r.rows = x.rows;
    r.order = x.order;
    r.coef = x.coef;
    r.partial = partial;
    r.n_rows = x.n_rows;
    r.dim = x.dim;
    r.n_entries = x.n_entries;
    r.per = x.per;
    const int64_t sums = x.n_entries / RUN;
    if (sums) k_run_sums<TG><<<(unsigned)((sums + WAVES - 1) / WAVES), WG, 0, st>>>(r, partial);
    if (x.n_entries) k_adamw_rows<TP, TG, BITS><<<(unsigned)((x.n_entries + WAVES - 1) / WAVES), WG, 0, st>>>(r, h);
    return launched(err);
}

// The kernel of a tensor's types: f(parameter, gradient, bits).
template <class F>
int by_type(int32_t param, int32_t grad, int32_t bits, F f)
{
    auto with_bits = [&](auto p, auto g) {
        return bits == 8 ? f(p, g, std::integral_constant<int, 8>{}) : f(p, g, std::integral_constant<int, 32>{});
    };
    auto with_grad = [&](auto p) {
        if (grad == SMORE_BF16) return with_bits(p, bf16{});
        if (grad == SMORE_F16) return with_bits(p, f16{});
        return with_bits(p, float{});
    };
    return param == SMORE_BF16 ? with_grad(bf16{}) : with_grad(float{});
}

}  // namespace

size_t adamw_workspace(const smore_adamw_tensor* ts, int n)
{
    size_t most = 0;   // tensors of a call are stepped one after the other
    for (int k = 0; k < n; ++k) {
        const size_t need = ts[k].rows ? (size_t)(ts[k].n_entries / RUN) * ts[k].dim * sizeof(float) : 0;
        most = need > most ? need : most;
    }
    return most;
}

int launch_adamw(const smore_adamw_tensor* ts, int n, const smore_adamw_args& a, void* ws, hipStream_t st, const char** err)
{
    Hyper h{};
    h.lr = (float)a.lr;
    h.b1 = (float)a.beta1;
    h.b2 = (float)a.beta2;
    h.eps = (float)a.eps;
    h.log_b1 = (float)log(a.beta1);
    h.log_b2 = (float)log(a.beta2);
    h.c1 = (float)-expm1((double)a.step * log(a.beta1));
    h.c2 = (float)-expm1((double)a.step * log(a.beta2));
    h.step = a.step_device;
    h.lr_dev = a.lr_device;
    h.grad_scale = a.grad_scale;
    h.step_host = a.step;
    h.seed = a.seed;
    h.stochastic = (a.flags & SMORE_ADAMW_STOCHASTIC) != 0;
    for (int k = 0; k < n;) {
        const smore_adamw_tensor& x = ts[k];
        int end = k + 1, rc;
        if (x.rows) {
            rc = by_type(x.param_type, x.grad_type, x.bits, [&](auto p, auto g, auto bits) {
                return rows_as<decltype(p), decltype(g), decltype(bits)::value>(x, h, (float*)ws, st, err);
            });
        } else {
            // dense tensors of the same types that follow each other go together
            while (end < n && !ts[end].rows && ts[end].param_type == x.param_type && ts[end].grad_type == x.grad_type &&
                   ts[end].bits == x.bits)
                ++end;
            rc = by_type(x.param_type, x.grad_type, x.bits, [&](auto p, auto g, auto bits) {
                return dense_as<decltype(p), decltype(g), decltype(bits)::value>(ts + k, end - k, h, st, err);
            });
        }
        if (rc) return rc;
        k = end;
    }
    return SMORE_OK;
}

}  // namespace smore
