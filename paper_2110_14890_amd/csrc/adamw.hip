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
// A moment that is not finite makes the scales of its 128 elements NaN.
// Unbiased for m and sqrt(v), that is; v, their square, settles 5 % high under
// Gaussian gradients, half to twice its value at the 1st and 99th percentiles
// (262,144 elements, 10,000 steps, b2 = 0.999; to the nearest 23 % high, and
// hardly to be moved from there).
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
constexpr int PER = 8;                  // consecutive elements of a lane
constexpr int CHUNK = 64 * PER;         // elements of a wavefront: four blocks of 128
constexpr int BLOCK = SMORE_ADAMW_BLOCK;
constexpr int RUN = 128;                // entries whose sum is made ahead in long runs
constexpr int AHEAD = 4;                // vectors of a run in flight

// One step's constants.
struct Step {
    float rate, keep, b1, b2, a1, a2, eps;   // a = 1 - b
    float slope, floor;                      // of the step's divisor, see divisor()
    float scale;                             // of the gradients
    uint32_t key;
};

struct Hyper {
    Step s;                             // as the host knows it (without keep, a tensor's)
    float c1, c2, log_b1, log_b2;       // c = 1 - b^t
    const int64_t* step;                // step, rate and gradient scale on the device, or NULL
    const float* lr_dev;
    const float* grad_scale;
    uint32_t seed_key;
    int32_t stochastic, on_device;
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
    const double* partial;
    double per_inverse;
    int64_t n_rows, dim, n_entries;
    uint32_t per;
};

// A published hash of 32-bit words: C. Wellons' lowbias32 (2018), two rounds of
// a shift and a product whose constants were searched for the least bias.
__host__ __device__ inline uint32_t mix(uint32_t x)
{
    x ^= x >> 16;
    x *= 0x7FEB352Du;
    x ^= x >> 15;
    x *= 0x846CA68Bu;
    return x ^ (x >> 16);
}
// Key of a step's roundings; a tensor's is mix(key + index).
__host__ __device__ inline uint32_t step_key(uint32_t seed_key, int64_t t)
{
    return mix(mix(seed_key + (uint32_t)t) ^ (uint32_t)((uint64_t)t >> 32));
}

// The step's constants for one tensor; false where nothing is to be written.
// A step's size, rate (m / c1) / (sqrt(v / c2) + eps), as m / -(slope sqrt(v) +
// floor): one product fewer.  A rate whose reciprocal is not finite stands
// still, whatever v is.
__host__ __device__ inline void divisor(Step* s, float c1, float c2)
{
    s->slope = -c1 / (s->rate * sqrtf(c2));
    s->floor = -c1 * s->eps / s->rate;
    if (!(fabsf(s->slope) < INFINITY) || !(fabsf(s->floor) < INFINITY)) {
        s->slope = -1.0f;
        s->floor = -INFINITY;
    }
}

__device__ __forceinline__ bool step_of(const Hyper& h, const Tensor& t, Step* s)
{
    *s = h.s;
    if (h.on_device) {
        if (h.lr_dev) s->rate = *h.lr_dev;
        float c1 = h.c1, c2 = h.c2;
        if (h.step) {
            const int64_t at = *h.step;
            c1 = -expm1f((float)at * h.log_b1);
            c2 = -expm1f((float)at * h.log_b2);
            s->key = step_key(h.seed_key, at);
        }
        divisor(s, c1, c2);
        if (h.grad_scale) s->scale = *h.grad_scale;
        if (!(fabsf(s->scale) < INFINITY)) return false;
    }
    s->keep = 1.0f - s->rate * t.decay;
    s->key = mix(s->key + (uint32_t)t.index);
    return true;
}

// Square root to the nearest (but for 1 in 10^7, which the tie-breaking bits
// are not fine enough to see): one Newton step from the estimate's residual.
// The moments take the same roundings as IEEE arithmetic, so that their codes
// do not depend on how a product and a sum are fused.
__device__ __forceinline__ float root_of(float v)
{
    const float r = __builtin_amdgcn_rsqf(fmaxf(v, 1.17549435e-38f));
    const float s = v * r;
    return fmaf(fmaf(-s, s, v), 0.5f * r, s);
}
// A root of the moments' width.  The hardware's roots take a subnormal number
// for 0, or here for the least normal one: v of a gradient below 3e-18 in the
// first step.  The careful form scales such a v first; with an eps of that
// size or 0 the parameter would go to infinity otherwise.  It also keeps the
// root of an infinite v (of a gradient above 1.8e19), which the Newton step
// makes NaN, and the parameter with it, though by the formula it stands still.
template <int BITS>
__device__ __forceinline__ float root(float v)
{
    return BITS == 8 ? root_of(v) : __builtin_amdgcn_sqrtf(v);
}
constexpr int NOT_A_NUMBER = 0x3, SUBNORMAL = 0x80, INFINITE = 0x200;   // of v_cmp_class, positive ones
template <int BITS>
__device__ __forceinline__ float careful_root(float v)
{
    const bool low = __builtin_amdgcn_classf(v, SUBNORMAL);
    const float u = root<BITS>(low ? v * 0x1p64f : v) * (low ? 0x1p-32f : 1.0f);
    return __builtin_amdgcn_classf(v, INFINITE) ? v : u;
}

__device__ __forceinline__ float first_moment(float m, float g, const Step& s)
{
#pragma clang fp contract(off)
    const float kept = s.b1 * m, added = s.a1 * g;
    return kept + added;
}
__device__ __forceinline__ float second_moment(float v, float g, const Step& s)
{
#pragma clang fp contract(off)
    const float square = g * g;
    const float kept = s.b2 * v, added = s.a2 * square;
    return kept + added;
}

__device__ __forceinline__ float moved(float p, float m, float u, const Step& s)
{
    return fmaf(m, __builtin_amdgcn_rcpf(fmaf(u, s.slope, s.floor)), p * s.keep);
}

// Codes of four values of [-448, 448].  The stochastic conversion adds its
// word's high 20 bits to the 20 fraction bits that a code drops (below 2^-6:
// to the fraction of 2^-9), of which a draw fills the upper 16.
__device__ __forceinline__ uint32_t encode(const float* y, const uint32_t* draw, bool stochastic)
{
    int x = 0;
    if (stochastic) {
        x = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], (int)draw[0], x, 0);
        x = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], (int)draw[1], x, 1);
        x = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], (int)draw[2], x, 2);
        x = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], (int)draw[3], x, 3);
    } else {
        x = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], x, false);
        x = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], x, true);
    }
    return (uint32_t)x;
}
constexpr float LEAST_CODE = 0x1p-9f;

// Values of four codes.
__device__ __forceinline__ void decode(uint32_t four, float* out)
{
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)four, false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)four, true);
    out[0] = a[0];
    out[1] = a[1];
    out[2] = b[0];
    out[3] = b[1];
}

// Largest of the 16 lanes of a block, as bits.
__device__ __forceinline__ uint32_t block_max(uint32_t x)
{
#define SMORE_STEP(CTRL) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true))
    SMORE_STEP(DPP_XOR1);
    SMORE_STEP(DPP_XOR2);
    SMORE_STEP(DPP_MIRROR8);
    SMORE_STEP(DPP_MIRROR16);
#undef SMORE_STEP
    return x;
}

// Scale of a block and the factor that takes its values to [0, 448].  Blocks
// that have decayed below 2^-100 are 0, which keeps the factor finite.
__device__ __forceinline__ void block_scale(float top, bool lost, float* scale, float* unit)
{
    const bool some = top >= 0x1p-100f;
    const float r = __builtin_amdgcn_rcpf(top);
    *scale = lost ? __uint_as_float(0x7FC00000u) : some ? top * (1.0f / 448.0f) : 0.0f;
    // 1 / top to the nearest, as root_of()
    *unit = some ? fmaf(fmaf(-top, r, 1.0f), r, r) * 448.0f : 0.0f;
}

// A lane's parameters to memory; bf16 rounded stochastically by the upper half
// of a product of the element's draw: by 2^32 over the golden ratio
// (multiplicative hashing, Knuth), after an exclusive or with a constant of
// MurmurHash3's (A. Appleby), so that a draw of 0 has bits too.
__device__ __forceinline__ void store_params(float* dst, int have, const float* p, const uint32_t*, bool)
{
    store_floats<float, PER>(dst, have, p);
}
__device__ __forceinline__ void store_params(bf16* dst, int have, const float* p, const uint32_t* draw, bool stochastic)
{
    if (!stochastic) return store_floats<bf16, PER>(dst, have, p);
    uint32_t x[PER / 2];
#pragma unroll
    for (int k = 0; k < PER / 2; ++k) {
        const uint32_t lo = __float_as_uint(p[2 * k]) + (((draw[2 * k] ^ 0x85EBCA6Bu) * 0x9E3779B1u) >> 16);
        const uint32_t hi = __float_as_uint(p[2 * k + 1]) + (((draw[2 * k + 1] ^ 0x85EBCA6Bu) * 0x9E3779B1u) >> 16);
        x[k] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);   // their upper halves
    }
    if (have >= PER) {
        __builtin_memcpy(dst, x, sizeof(x));
    } else {
#pragma unroll
        for (int j = 0; j < PER - 1; ++j) {
            const uint16_t one = (uint16_t)(x[j / 2] >> (16 * (j % 2)));
            if (j < have) __builtin_memcpy(dst + j, &one, 2);
        }
    }
}

// Elements and moments that a lane holds.
template <int BITS>
struct Held;
template <>
struct Held<32> {
    float m[PER], v[PER];
};
template <>
struct Held<8> {
    uint32_t m[PER / 4], v[PER / 4];
    float m_scale, v_scale;
};

__device__ __forceinline__ void load_codes(const uint8_t* p, int have, uint32_t* x)
{
    if (have >= PER) {
        __builtin_memcpy(x, p, PER);
    } else {
#pragma unroll
        for (int k = 0; k < PER / 4; ++k) x[k] = 0;
#pragma unroll
        for (int j = 0; j < PER - 1; ++j)
            if (j < have) x[j / 4] |= (uint32_t)p[j] << (8 * (j % 4));
    }
}
__device__ __forceinline__ void store_codes(uint8_t* p, int have, const uint32_t* x)
{
    if (have >= PER) {
        __builtin_memcpy(p, x, PER);
    } else {
#pragma unroll
        for (int j = 0; j < PER - 1; ++j)
            if (j < have) p[j] = (uint8_t)(x[j / 4] >> (8 * (j % 4)));
    }
}

// at: the lane's first element in the tensor; have: how many of its PER
// elements the row has (none: <= 0); block: number of its 128-element block.
template <int BITS>
__device__ __forceinline__ void load_held(const Tensor& t, int64_t at, int have, int64_t block, Held<BITS>& h)
{
    if constexpr (BITS == 32) {
        load_floats<float, PER>((const float*)t.m + at, have, h.m);
        load_floats<float, PER>((const float*)t.v + at, have, h.v);
    } else {
        load_codes((const uint8_t*)t.m + at, have, h.m);
        load_codes((const uint8_t*)t.v + at, have, h.v);
        h.m_scale = have > 0 ? t.m_scale[block] : 0.0f;
        h.v_scale = have > 0 ? t.v_scale[block] : 0.0f;
    }
}

// Steps a lane's PER elements and writes them back.  Every lane of the
// wavefront takes part (the maxima of the 8-bit blocks).  j0: the lane's
// first element in its block.
template <class TP, int BITS>
__device__ __forceinline__ void step_held(const Tensor& t, const Step& s, bool stochastic, int64_t at, int have,
                                          int64_t block, int j0, float* p, float* g, Held<BITS>& h)
{
    float m[PER], v[PER], u[PER];
    // A v whose root takes more than the hardware's; for parameters whose lower
    // bits are rounded off also a NaN, which comes with the gradient or with a
    // moment before.
    constexpr bool ROUNDED = sizeof(TP) == 2;
    constexpr int SPECIAL = SUBNORMAL | (BITS == 8 ? INFINITE : 0) | (ROUNDED ? NOT_A_NUMBER : 0);
    bool rare = false;
    if (s.scale != 1.0f) {
#pragma unroll
        for (int j = 0; j < PER; ++j) g[j] *= s.scale;
    }
    if constexpr (BITS == 32) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            m[j] = h.m[j];
            v[j] = h.v[j];
        }
    } else {
#pragma unroll
        for (int k = 0; k < PER / 4; ++k) {
            decode(h.m[k], m + 4 * k);
            decode(h.v[k], v + 4 * k);
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            m[j] *= h.m_scale;
            v[j] *= h.v_scale;
            v[j] *= v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        m[j] = first_moment(m[j], g[j], s);
        v[j] = second_moment(v[j], g[j], s);
        rare |= __builtin_amdgcn_classf(v[j], SPECIAL);
        u[j] = root<BITS>(v[j]);
        p[j] = moved(p[j], m[j], u[j], s);
    }
    if (BITS == 32 && ROUNDED && stochastic) {
#pragma unroll
        for (int j = 0; j < PER; ++j) rare |= m[j] != m[j];
    }
    constexpr bool DRAWS = BITS == 8 || sizeof(TP) == 2;
    uint32_t draw[PER] = {};
    if (DRAWS && stochastic) {
        const uint32_t base = mix(mix(s.key ^ (uint32_t)block) + (uint32_t)((uint64_t)block >> 32)) + (uint32_t)j0;
#pragma unroll
        for (int j = 0; j < PER; ++j) draw[j] = mix(base + (uint32_t)j);
    }
    // Once more from the start where a root takes more than the hardware's.  The
    // branch stands here so that the draws run beside the roots: right behind
    // them it cost 2 % of the time of 156K rows of 400 and of 320M elements in 8
    // bits (199.3 against 195.3 us, 615 against 602).
    if (__any(rare)) {
        load_floats<TP, PER>((const TP*)t.p + at, have, p);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            u[j] = careful_root<BITS>(v[j]);
            p[j] = moved(p[j], m[j], u[j], s);
            // adding to a NaN's lower bits could carry into its sign, and make it 0
            if (ROUNDED && p[j] != p[j]) p[j] = __uint_as_float(0x7FC00000u);
        }
    }
    if (have > 0) store_params((TP*)t.p + at, have, p, draw, stochastic);
    if constexpr (BITS == 32) {
        if (have > 0) {
            store_floats<float, PER>((float*)t.m + at, have, m);
            store_floats<float, PER>((float*)t.v + at, have, v);
        }
    } else {
        // places behind the row's end were loaded as zeros, have no gradient
        // and are 0 still
        float m_top = 0.0f;
        uint32_t u_top = 0;   // largest root as bits: NaN above infinity above every number
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            m_top = fmaxf(m_top, fabsf(m[j]));
            u_top = max(u_top, __float_as_uint(u[j]));
        }
        u_top = block_max(u_top);
        m_top = __uint_as_float(block_max(__float_as_uint(m_top)));
        // a moment that is not finite, now or before, makes both NaN
        const bool lost = u_top >= 0x7F800000u || !(m_top < INFINITY) || h.m_scale != h.m_scale;
        float m_scale, m_unit, u_scale, u_unit;
        block_scale(m_top, lost, &m_scale, &m_unit);
        block_scale(__uint_as_float(u_top), lost, &u_scale, &u_unit);
        float least = 448.0f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            m[j] *= m_unit;
            const float y = u[j] * u_unit;
            least = fminf(least, y);
            p[j] = u[j];      // the parameter is written: its place keeps the root
            u[j] = y;
        }
        // a root that is not 0 has a code that is not 0 (rarely below it: a
        // root under 2^-18 of its block's largest; lanes without a column hold
        // roots that are 0, which need nothing)
        if (__any(have > 0 && least < LEAST_CODE)) {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (p[j] != 0.0f && u_unit > 0.0f) u[j] = fmaxf(u[j], LEAST_CODE);
        }
        uint32_t low[PER], high[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            low[j] = draw[j] << 16;
            high[j] = draw[j] & 0xFFFF0000u;
        }
        uint32_t m4[PER / 4], u4[PER / 4];
#pragma unroll
        for (int k = 0; k < PER / 4; ++k) {
            m4[k] = encode(m + 4 * k, low + 4 * k, stochastic);
            u4[k] = encode(u + 4 * k, high + 4 * k, stochastic);
        }
        if (have > 0) {
            store_codes((uint8_t*)t.m + at, have, m4);
            store_codes((uint8_t*)t.v + at, have, u4);
            if (j0 == 0) {
                t.m_scale[block] = m_scale;
                t.v_scale[block] = u_scale;
            }
        }
    }
}

// How many of a lane's PER elements, from `at` on, lie before `end`.
__device__ __forceinline__ int left(int64_t end, int64_t at) { return (int)max((int64_t)0, min((int64_t)PER, end - at)); }

// A workgroup takes WAVES x CHUNKS chunks of one tensor; which one it finds
// among the launch's tensors by their first workgroups.  319M elements, bf16
// parameters and gradients, 8-bit moments: 590 us, 5.5 TB/s, with vector
// operations in 90 % of the issue slots (53 an element, a third of them the
// hash of the roundings); 15 tensors of 1.1M elements in 32 bits: 10 us.
template <class TP, class TG, int BITS, int CHUNKS>
__global__ __launch_bounds__(WG) void k_adamw(const TensorList list, const Hyper hyper)
{
    int lo = 0, hi = list.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (list.t[mid].first_wg <= blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const Tensor& t = list.t[lo];
    Step s;
    if (!step_of(hyper, t, &s)) return;
    const bool stochastic = hyper.stochastic;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t base = ((int64_t)(blockIdx.x - t.first_wg) * WAVES + wave) * (CHUNK * CHUNKS) + lane * PER;
    float p[CHUNKS][PER], g[CHUNKS][PER];
    Held<BITS> h[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int64_t at = base + c * CHUNK;
        const int have = left(t.count, at);
        load_floats<TP, PER>((const TP*)t.p + at, have, p[c]);
        load_floats<TG, PER>((const TG*)t.g + at, have, g[c]);
        load_held<BITS>(t, at, have, at / BLOCK, h[c]);
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int64_t at = base + c * CHUNK;
        step_held<TP, BITS>(t, s, stochastic, at, left(t.count, at), at / BLOCK, (int)(at % BLOCK), p[c], g[c], h[c]);
    }
}

// Entries of the sorted list that name a row: coefficient and source vector
// of entry at + lane.
struct Entry {
    float w;
    uint32_t from;
};
__device__ __forceinline__ Entry entry_at(const RowsTensor& r, int64_t o, bool in)
{
    Entry e{0.0f, 0u};
    if (in && o >= 0 && o < r.n_entries) {   // a permutation's: reads nothing behind the gradients otherwise
        e.w = r.coef ? r.coef[o] : 1.0f;
        uint32_t q = (uint32_t)((double)o * r.per_inverse);   // off by one at most
        if ((uint64_t)q * r.per > (uint64_t)o) --q;
        if ((uint64_t)(q + 1) * r.per <= (uint64_t)o) ++q;
        e.from = q;
    }
    return e;
}
__device__ __forceinline__ Entry entry_of(const RowsTensor& r, int64_t at, int64_t end)
{
    return entry_at(r, at < end && r.order ? r.order[at] : at, at < end);
}

// Sums over a row's entries: products in fp32, their sum in 64 bits and one
// rounding to fp32, so that long runs lose next to nothing.  The order of the
// sum is fixed by the entries' places; another one could show where the exact
// sum lies within 64 bits' error of a border of fp32.  Rows of at most MOST
// lanes (below 64) take as few lanes as hold them, a power of two; 64 / lanes
// groups add every so many entries each, and finish() adds the groups' sums.
template <class TG, int MOST>
struct RowSum {
    const RowsTensor& r;
    int64_t col;
    int lanes, group, groups, have;
    double g[PER];

    __device__ __forceinline__ RowSum(const RowsTensor& t, int64_t chunk) : r(t)
    {
        const int lane = threadIdx.x & 63;
        lanes = MOST;
        if (MOST < 64)
            while (lanes > 1 && (lanes / 2) * PER >= r.dim) lanes /= 2;
        group = MOST < 64 ? lane / lanes : 0;
        groups = 64 / lanes;
        col = chunk + (lane % lanes) * PER;
        have = left(r.dim, col);
#pragma unroll
        for (int j = 0; j < PER; ++j) g[j] = 0.0;
    }

    // x of lane `at`, the same one for all lanes of a group
    __device__ __forceinline__ int from_lane(int x, int at) const
    {
        return MOST == 64 ? __builtin_amdgcn_readlane(x, at) : __shfl(x, at);
    }
    // the entries that lanes [first, end) hold
    __device__ __forceinline__ void held(const Entry& e, int first, int end)
    {
        for (int i = first + group; i - group < end; i += AHEAD * groups) {
            float x[AHEAD][PER];
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                const int64_t src = (uint32_t)from_lane((int)e.from, min(i + q * groups, end - 1));
                load_floats<TG, PER>((const TG*)r.t.g + src * r.dim + col, have, x[q]);
            }
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) {
                const float w = __int_as_float(from_lane(__float_as_int(e.w), min(i + q * groups, end - 1)));
                if (i + q * groups < end) {
#pragma unroll
                    for (int j = 0; j < PER; ++j) g[j] += (double)(w * x[q][j]);
                }
            }
        }
    }
    // the entries [first, end) of the list
    __device__ __forceinline__ void entries(int64_t first, int64_t end)
    {
        const int lane = threadIdx.x & 63;
        for (int64_t at = first; at < end; at += 64) held(entry_of(r, at + lane, end), 0, (int)min((int64_t)64, end - at));
    }
    // the sums made ahead of `count` stretches of RUN entries
    __device__ __forceinline__ void ahead(int64_t first, int count)
    {
        for (int k = group; k < count; k += groups) {
            const double* from = r.partial + (first + k) * r.dim + col;
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j < have) g[j] += from[j];
        }
    }
    __device__ __forceinline__ void finish()
    {
        for (int d = lanes; d < 64; d *= 2) {
#pragma unroll
            for (int j = 0; j < PER; ++j) g[j] += __shfl_xor(g[j], d);
        }
        // Fewer than 16 lanes hold a row of at most 64 columns: the other lanes
        // of its block own no column, and a copy of another lane's sum must not
        // count in the block's largest moment.
        if (MOST == 16 && (int)(threadIdx.x & 63) >= lanes) {
#pragma unroll
            for (int j = 0; j < PER; ++j) g[j] = 0.0;
        }
    }
};

// Sums of RUN consecutive entries of one row, where a run is that long, so
// that no wavefront has to add a hub's entries one by one.
template <class TG, int MOST>
__global__ __launch_bounds__(WG) void k_run_sums(const RowsTensor r, double* __restrict__ partial)
{
    const int64_t c = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6);
    if ((c + 1) * RUN > r.n_entries) return;
    const int32_t row = r.rows[c * RUN];
    if (row < 0 || row >= r.n_rows || r.rows[c * RUN + RUN - 1] != row) return;
    for (int64_t chunk = 0; chunk < r.dim; chunk += CHUNK) {
        RowSum<TG, MOST> sum(r, chunk);
        sum.entries(c * RUN, (c + 1) * RUN);
        sum.finish();
        if (sum.group == 0) {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j < sum.have) partial[c * r.dim + sum.col + j] = sum.g[j];
        }
    }
}

// A run of one row's entries that goes on behind a wavefront's first look.
// [i, head): entries up to the run's end or the first sum made ahead; then
// `sums` of those; then [tail, end).
struct LongRun {
    int64_t head, tail = 0, end = 0;
    int sums = 0;
    __device__ LongRun(const RowsTensor& r, int64_t i, int32_t row)
    {
        const int lane = threadIdx.x & 63;
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
};

// A wavefront per `window` entries (up to 16), each a workgroup of its own: it
// steps the rows whose runs begin there.  Its first look is one read of the
// entry before, the window, and what fits behind it, where most runs end.
// Rows that LANES lanes hold (16 or 32: up to 128 or 256 columns) are stepped
// 64 / LANES at a time, where their runs are short; wider ones that one chunk
// holds two at a time; the others one by one.
// Narrow rows with 8-bit moments are held to the registers of five wavefronts
// a SIMD: 264K entries of 156K rows of 100 columns 88 us, with four 96.
// 156K rows of 400 (264K entries), 8-bit moments: 191 us; 14.4K rows (66K
// entries) in 32 bits: 36 us, 3.7 TB/s.  The first is bound by the vector
// operations of k_adamw in 50 of 64 lanes, the second by the MALL.
// SHORT is the most entries of a run that goes with others.  us with 2 / 4 / 6:
// 264K entries of 156K rows of 100 95 / 88 / 93, of 58K rows 104 / 69 / 56; of
// 156K rows of 400 193 / 191 / 192, of 58K rows 99 / 93 / 91.
constexpr int SHORT = 4;
template <class TP, class TG, int BITS, int LANES>
__global__ __launch_bounds__(64, LANES < 64 && BITS == 8 ? 5 : 1) void k_adamw_rows(const RowsTensor r, const Hyper hyper, int window)
{
    const int lane = threadIdx.x;
    const int64_t first = (int64_t)blockIdx.x * window;   // lane 1 looks at this entry
    const int64_t look = first - 1 + lane;
    const bool in = look >= 0 && look < r.n_entries;
    const int32_t id = in ? r.rows[look] : -1;
    const int64_t o = in && r.order ? r.order[look] : look;
    const int32_t before = __shfl_up(id, 1);
    const uint64_t begins = __ballot(lane > 0 && id != before);
    uint64_t heads = __ballot(lane > 0 && lane <= window && id != before && id >= 0 && id < r.n_rows);
    if (!heads) return;
    Step s;
    if (!step_of(hyper, r.t, &s)) return;
    const bool stochastic = hyper.stochastic;
    const Entry e = entry_at(r, o, in);
    const int64_t blocks = (r.dim + BLOCK - 1) / BLOCK;
    if constexpr (LANES < 64) {
        const uint64_t after = lane < 63 ? begins >> (lane + 1) : 0;
        const int mine = after ? __builtin_ctzll(after) + 1 : 64;      // entries of the run that begins here
        uint64_t quick = heads & __ballot(mine <= SHORT);
        heads &= ~quick;
        while (quick) {
            const int group = lane / LANES, col = lane % LANES * PER;
            int head = -1;
#pragma unroll
            for (int q = 0; q < 64 / LANES; ++q) {
                if (quick && group == q) head = __builtin_ctzll(quick);
                quick &= quick - 1;
            }
            // every lane takes part in the exchanges, those without a row too
            const int32_t named = __shfl(id, head & 63), length = __shfl(mine, head & 63);
            const int64_t row = head < 0 ? 0 : named;
            const int count = head < 0 ? 0 : length;
            const int have = head < 0 ? 0 : left(r.dim, col);
            const int64_t at = row * r.dim + col, block = row * blocks + col / BLOCK;
            float p[PER], g[PER];
            Held<BITS> h;
            {
                double sum[PER] = {};
                float x[SHORT][PER], w[SHORT];
#pragma unroll
                for (int k = 0; k < SHORT; ++k) {
                    const int from = (head + k) & 63;
                    const int64_t src = (uint32_t)__shfl((int)e.from, from);
                    w[k] = __shfl(e.w, from);
                    load_floats<TG, PER>((const TG*)r.t.g + src * r.dim + col, k < count ? have : 0, x[k]);
                }
#pragma unroll
                for (int k = 0; k < SHORT; ++k)
                    if (k < count) {
#pragma unroll
                        for (int j = 0; j < PER; ++j) sum[j] += (double)(w[k] * x[k][j]);
                    }
#pragma unroll
                for (int j = 0; j < PER; ++j) g[j] = (float)sum[j];
            }
            load_floats<TP, PER>((const TP*)r.t.p + at, have, p);
            load_held<BITS>(r.t, at, have, block, h);
            step_held<TP, BITS>(r.t, s, stochastic, at, have, block, col % BLOCK, p, g, h);
        }
    }
    if (LANES == 64 && r.dim <= CHUNK) {
        // rows with few entries two at a time, so that the second's reads are
        // on their way while the first is stepped, against one by one: 8-bit
        // moments 191 instead of 230 us for the 156K rows, 4.8 ms instead of 5.4
        // for 4.4M rows; in 32 bits, where it takes them from five wavefronts a
        // SIMD to three, 36.5 instead of 38.1 for the 14.4K rows, 420 instead
        // of 424 for the 156K, 360 instead of 369 at width 300.  It loses where
        // there are few rows: 6,000 entries 16.8 against 16.2 us in 32 bits,
        // 14.8 against 14.3 in 8.
        const uint64_t after = lane < 63 ? begins >> (lane + 1) : 0;
        const int mine = after ? __builtin_ctzll(after) + 1 : 64;      // entries of the run that begins here
        uint64_t quick = heads & __ballot(mine <= SHORT);
        const int col = lane * PER, have = left(r.dim, col);
        while (quick & (quick - 1)) {
            float p[2][PER], g[2][PER];
            Held<BITS> h[2];
            int64_t at[2], block[2];
            int head[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                head[q] = __builtin_ctzll(quick);
                heads &= ~(quick & (0 - quick));
                quick &= quick - 1;
                const int64_t row = __builtin_amdgcn_readlane(id, head[q]);
                at[q] = row * r.dim + col;
                block[q] = row * blocks + col / BLOCK;
                load_floats<TP, PER>((const TP*)r.t.p + at[q], have, p[q]);
                load_held<BITS>(r.t, at[q], have, block[q], h[q]);
                const int64_t src = (uint32_t)__builtin_amdgcn_readlane((int)e.from, head[q]);
                load_floats<TG, PER>((const TG*)r.t.g + src * r.dim + col, have, g[q]);
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e.w), head[q]));
#pragma unroll
                for (int j = 0; j < PER; ++j) g[q][j] *= w;
                const int count = __builtin_amdgcn_readlane(mine, head[q]);
                if (count > 1) {
                    RowSum<TG, LANES> sum(r, 0);
#pragma unroll
                    for (int j = 0; j < PER; ++j) sum.g[j] = g[q][j];
                    sum.held(e, head[q] + 1, head[q] + count);
#pragma unroll
                    for (int j = 0; j < PER; ++j) g[q][j] = (float)sum.g[j];
                }
                step_held<TP, BITS>(r.t, s, stochastic, at[q], have, block[q], col % BLOCK, p[q], g[q], h[q]);
            }
        }
    }
    for (; heads; heads &= heads - 1) {
        const int head = __builtin_ctzll(heads);
        const int32_t row = __builtin_amdgcn_readlane(id, head);
        const uint64_t later = head < 63 ? begins >> (head + 1) : 0;
        const int end = later ? head + 1 + __builtin_ctzll(later) : 64;
        for (int64_t col = lane * PER; col - lane * PER < r.dim; col += CHUNK) {
            const int have = left(r.dim, col);
            const int64_t at = (int64_t)row * r.dim + col, block = row * blocks + col / BLOCK;
            float p[PER], g[PER];
            Held<BITS> h;
            if (!(end == head + 1 && later)) {
                RowSum<TG, LANES> sum(r, col - lane * PER);
                if (later) {
                    sum.held(e, head, end);
                } else {
                    const LongRun run(r, first - 1 + head, row);
                    sum.entries(first - 1 + head, run.head);
                    sum.ahead(run.tail / RUN - run.sums, run.sums);
                    sum.entries(run.tail, run.end);
                }
                sum.finish();
#pragma unroll
                for (int j = 0; j < PER; ++j) g[j] = (float)sum.g[j];
            }
            load_floats<TP, PER>((const TP*)r.t.p + at, have, p);
            load_held<BITS>(r.t, at, have, block, h);
            if (end == head + 1 && later) {
                const int64_t src = (uint32_t)__builtin_amdgcn_readlane((int)e.from, head);
                const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e.w), head));
                load_floats<TG, PER>((const TG*)r.t.g + src * r.dim + col, have, g);
#pragma unroll
                for (int j = 0; j < PER; ++j) g[j] *= w;
            }
            step_held<TP, BITS>(r.t, s, stochastic, at, have, block, (int)(col % BLOCK), p, g, h);
        }
    }
}

template <class TP, class TG, int BITS, int CHUNKS>
int dense_chunks(const smore_adamw_tensor* ts, int n, const Hyper& h, hipStream_t st, const char** err)
{
    TensorList list;
    list.n = 0;
    uint64_t wgs = 0;
    auto flush = [&] {
        if (list.n) k_adamw<TP, TG, BITS, CHUNKS><<<(unsigned)wgs, WG, 0, st>>>(list, h);
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
int dense_as(const smore_adamw_tensor* ts, int n, const Hyper& h, hipStream_t st, const char** err)
{
    // Two chunks of a wavefront in flight, where that leaves enough wavefronts.
    // us with one / two: bf16 and 8-bit moments 4M elements 12.6 / 13.3, 32M 67.6
    // / 65.3, 128M 283 / 276; fp32 4M 27.4 / 28.9, 16M 77 / 82, 32M 198 / 196,
    // 128M 771 / 762.  Two lose with bf16 and 32-bit moments (128M 613 / 627).
    int64_t total = 0;
    for (int k = 0; k < n; ++k) total += ts[k].n_rows * ts[k].dim;
    if (total < (int64_t)CHUNK * WAVES * 4096) return dense_chunks<TP, TG, BITS, 1>(ts, n, h, st, err);
    return dense_chunks<TP, TG, BITS, 2>(ts, n, h, st, err);
}

template <class TP, class TG, int BITS>
int rows_as(const smore_adamw_tensor& x, const Hyper& h, double* partial, hipStream_t st, const char** err)
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
    r.per = (uint32_t)(x.per < (1 << 30) ? x.per : 1 << 30);   // entries are fewer
    r.per_inverse = 1.0 / r.per;
    const int64_t sums = x.n_entries / RUN;
    const unsigned sum_grid = (unsigned)((sums + WAVES - 1) / WAVES);
    if (sums && x.dim <= 32 * PER) k_run_sums<TG, 32><<<sum_grid, WG, 0, st>>>(r, partial);
    else if (sums) k_run_sums<TG, 64><<<sum_grid, WG, 0, st>>>(r, partial);
    // entries per wavefront: as many as leave each of the 1,024 SIMDs eight
    // wavefronts, up to 16.  8-bit moments, width 400, us with 1 / 4 / 8 / 16 /
    // 32 entries: 1.05M entries of 371K rows 844 / 693 / 653 / 634 / 613, 263K
    // of 250K 439 / 305 / 296 / 296 / 316; in 32 bits 66K of 14.9K
    // 48 / 41 / 41 / 45 / 47.
    int window = 1;
    while (window < 16 && x.n_entries >= (int64_t)8192 * 2 * window) window *= 2;
    const unsigned grid = (unsigned)((x.n_entries + window - 1) / window);
    if (x.n_entries) {
        if (x.dim <= 16 * PER) k_adamw_rows<TP, TG, BITS, 16><<<grid, 64, 0, st>>>(r, h, window);
        else if (x.dim <= 32 * PER) k_adamw_rows<TP, TG, BITS, 32><<<grid, 64, 0, st>>>(r, h, window);
        else k_adamw_rows<TP, TG, BITS, 64><<<grid, 64, 0, st>>>(r, h, window);
    }
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
        const size_t need = ts[k].rows ? (size_t)(ts[k].n_entries / RUN) * ts[k].dim * sizeof(double) : 0;
        most = need > most ? need : most;
    }
    return most;
}

int launch_adamw(const smore_adamw_tensor* ts, int n, const smore_adamw_args& a, void* ws, hipStream_t st, const char** err)
{
    Hyper h{};
    h.s.rate = (float)a.lr;
    h.s.b1 = (float)a.beta1;
    h.s.b2 = (float)a.beta2;
    h.s.a1 = (float)(1.0 - a.beta1);
    h.s.a2 = (float)(1.0 - a.beta2);
    h.s.eps = (float)a.eps;
    h.c1 = (float)-expm1((double)a.step * log(a.beta1));
    h.c2 = (float)-expm1((double)a.step * log(a.beta2));
    divisor(&h.s, h.c1, h.c2);
    h.s.scale = 1.0f;
    h.log_b1 = (float)log(a.beta1);
    h.log_b2 = (float)log(a.beta2);
    h.step = a.step_device;
    h.lr_dev = a.lr_device;
    h.grad_scale = a.grad_scale;
    h.on_device = a.step_device || a.lr_device || a.grad_scale;
    h.seed_key = mix(mix((uint32_t)a.seed) ^ (uint32_t)(a.seed >> 32));
    h.s.key = step_key(h.seed_key, a.step);
    h.stochastic = (a.flags & SMORE_ADAMW_STOCHASTIC) != 0;
    for (int k = 0; k < n;) {
        const smore_adamw_tensor& x = ts[k];
        int end = k + 1, rc;
        if (x.rows) {
            rc = by_type(x.param_type, x.grad_type, x.bits, [&](auto p, auto g, auto bits) {
                return rows_as<decltype(p), decltype(g), decltype(bits)::value>(x, h, (double*)ws, st, err);
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
