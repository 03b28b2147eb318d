// AdamW over many tensors in one launch, with states in 32 or 8 bits.
//
// Per parameter 28 bytes move with 32-bit states (parameter, both states read and written in float32, a 16-bit gradient
// read, a 16-bit copy written) and 16 with 8-bit ones.  32 bits: memory bounds it, 180 M parameters take 812 us, 6.2 TB/s,
// 95 % of a copy's rate.  8 bits: rounding takes most of 79 instructions a parameter, which the SMs issue at three quarters of
// their rate while memory runs at 5.3 TB/s (404 M parameters: 1 220 us).
//
// A warp takes a block of 256 parameters, eight consecutive ones a lane: the largest loads there are (32 bytes a lane),
// and a block's largest magnitude, which the 8-bit states' scale needs, is one shuffle reduction of values that are in
// registers already.  Tensors of any size and number share one launch: a table gives the tensor of every eighth block.
#include <type_traits>

#include "train_ops.h"

namespace guard {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ double power(double b, int64_t n) {   // b^n by squaring: 2 log2(n) roundings of 2^-53
    double r = 1.0;
    for (; n > 0; n >>= 1) {
        if (n & 1) r *= b;
        b *= b;
    }
    return r;
}

// 32 dithering bits of a position: two multiplicative rounds over position and key, with multipliers and shifts of the published
// hash xxHash (32 bits); the positions' upper word is folded in with a multiplier of MurmurHash3.  Neighbouring positions and steps
// only have to be uncorrelated and each value equally frequent, which the tests count.
__device__ __forceinline__ uint32_t dither(uint32_t i, uint32_t key) {
    uint32_t h = (i ^ key) * 0x9E3779B1u;
    h ^= h >> 15;
    h *= 0x85EBCA77u;
    return h ^ (h >> 13);
}

// y in [0, 448] to a multiple of e4m3's step there, up with the probability of what is cut off (16 random bits; the result
// converts exactly): random bits are added below the three bits of fraction that stay, then cut off.  Below 2^-6 e4m3's
// steps stay 2^-9, as they are in [2^-6, 2^-5): the value is moved there and back.
__device__ __forceinline__ float to_step(float y, uint32_t bits20) {   // (the 16 bits in the upper part of 20)
    const float up = y < 0.015625f ? 0.015625f : 0.0f;
    const float t = __fadd_rn(y, up);
    return __fsub_rn(__uint_as_float((__float_as_uint(t) + bits20) & ~0xFFFFFu), up);
}
// Two values in e4m3, the first in the low byte.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void from_e4m3x2(uint32_t two, float &lo, float &hi) {
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)two));
    const __half2 h = *reinterpret_cast<__half2 *>(&h2);
    lo = __low2float(h);
    hi = __high2float(h);
}

__device__ __forceinline__ float root(float x) {
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A lane's eight values as they lie in memory: one vector of 16 or 32 bytes, loaded whole where a block is whole.
template <typename T> struct Raw8 {
    using Vector = typename std::conditional<sizeof(T) == 4, Bytes32, Bytes16>::type;
    Vector v;
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (sizeof(T) == 4) v = load32_once(p);
        else v = load16_once(p);
    }
    __device__ __forceinline__ void load_some(const T *p, int left) {       // those before `left`, the rest zero
        T *t = reinterpret_cast<T *>(&v);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = j < left ? p[j] : Conv<T>::down(0.0f);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const T *t = reinterpret_cast<const T *>(&v);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = Conv<T>::up(t[j]);
    }
};
template <bool FAST, typename T>
__device__ __forceinline__ void store8(T *p, int left, const float (&x)[8]) {
    if constexpr (FAST) {
        typename Raw8<T>::Vector r;
        T *t = reinterpret_cast<T *>(&r);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = Conv<T>::down(x[j]);
        if constexpr (sizeof(T) == 4) store32_once(p, r);
        else store16_once(p, r);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < left) p[j] = Conv<T>::down(x[j]);
    }
}
// A lane's eight values of a state: float32, or e4m3 with the block's scale (a power of two: the product is exact).
template <int BITS> struct RawState : Raw8<float> {
    __device__ __forceinline__ void load(const void *p, const float *, int64_t flat, int64_t) { Raw8<float>::load(reinterpret_cast<const float *>(p) + flat); }
    __device__ __forceinline__ void load_some(const void *p, const float *, int64_t flat, int64_t, int left) {
        Raw8<float>::load_some(reinterpret_cast<const float *>(p) + flat, left);
    }
};
template <> struct RawState<8> {
    uint32_t w[2];
    float scale;
    __device__ __forceinline__ void load(const void *p, const float *scales, int64_t flat, int64_t block) {
        asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(reinterpret_cast<const uint8_t *>(p) + flat));
        scale = scales[block];
    }
    __device__ __forceinline__ void load_some(const void *p, const float *scales, int64_t flat, int64_t block, int left) {
        w[0] = w[1] = 0;
        for (int j = 0; j < left; ++j) w[j >> 2] |= (uint32_t) reinterpret_cast<const uint8_t *>(p)[flat + j] << (8 * (j & 3));
        scale = scales[block];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) from_e4m3x2(w[j >> 1] >> (16 * (j & 1)), x[2 * j], x[2 * j + 1]);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __fmul_rn(x[j], scale);
    }
};
// Stores x as 8-bit values of the block's scale, which it returns: the power of two by which the block's largest magnitude
// comes to lie in (224, 448], 448 being e4m3's largest value.  Powers of two keep the grid of values as it is when the
// scale changes, so a value moves only by what the update adds to it: with the largest magnitude itself as the scale, every
// step would round every value anew, and the noise of that adds up over the 1 / (1 - beta2) steps that a mean remembers.
template <bool FAST, bool LEAST>
__device__ __forceinline__ float store8_e4m3(uint8_t *p, int left, const float (&x)[8], const uint32_t (&bits)[8]) {
    uint32_t top = 0;                          // magnitudes order as their bits do
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, LEAST ? __float_as_uint(x[j]) : __float_as_uint(x[j]) & 0x7FFFFFFFu);   // (LEAST: second moments, never negative)
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    const bool strange = top >= 0x7F800000u;   // some value is not finite: it becomes NaN, the others keep a scale of their own
    if (strange) {
        top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, fabsf(x[j]) < INFINITY ? __float_as_uint(x[j]) & 0x7FFFFFFFu : 0u);
        top = __reduce_max_sync(0xFFFFFFFFu, top);
    }
    const uint32_t high = (top + 0x1FFFFFu) >> 23;
    const uint32_t e = (high < 9 ? 9 : high) - 8;                     // the scale's exponent field, 1 .. 247
    const float inverse = __uint_as_float((254 - e) << 23);
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        y[j] = __fmul_rn(LEAST ? x[j] : fabsf(x[j]), inverse);
        const float stepped = to_step(y[j], bits[j]);
        y[j] = LEAST ? (y[j] > 0.0f ? fmaxf(stepped, 0.001953125f) : y[j]) : copysignf(stepped, x[j]);
    }
    if (strange) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (!(fabsf(x[j]) < INFINITY)) y[j] = __uint_as_float(0x7FC00000u);
    }
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; j += 2) w[j >> 2] |= to_e4m3x2(y[j], y[j + 1]) << (16 * ((j >> 1) & 1));
    if constexpr (FAST) {
        asm volatile("st.global.L1::no_allocate.v2.b32 [%2], {%0,%1};" ::"r"(w[0]), "r"(w[1]), "l"(p) : "memory");
    } else {
        for (int j = 0; j < left; ++j) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    }
    return __uint_as_float(e << 23);
}

// CTAs an SM, and as many in the grid: 128 registers hold the next block's values without spilling.  404 M parameters with
// 8-bit states take 1 218 us so (5.3 TB/s), 1 355 with four CTAs of 64 registers and nothing on its way.
constexpr int kResident = 2;

struct Rates { float rate, grow, lr, grad_scale; uint32_t key; };

// What a lane reads of a block.
template <typename G, int BITS> struct Block {
    Raw8<float> p;
    Raw8<G> g;
    RawState<BITS> m, v;
    __device__ __forceinline__ void load(const AdamwArgs &a, const AdamwTensor &T, int64_t b) {
        const int64_t at = (b - T.first) * kAdamwBlock + lane_id() * 8, flat = b * kAdamwBlock + lane_id() * 8;
        p.load(T.param + at);
        g.load(reinterpret_cast<const G *>(T.grad) + at);
        m.load(a.m, a.m_scale, flat, b);
        v.load(a.v, a.v_scale, flat, b);
    }
    __device__ __forceinline__ void load_some(const AdamwArgs &a, const AdamwTensor &T, int64_t b, int left) {
        const int64_t at = (b - T.first) * kAdamwBlock + lane_id() * 8, flat = b * kAdamwBlock + lane_id() * 8;
        p.load_some(T.param + at, left);
        g.load_some(reinterpret_cast<const G *>(T.grad) + at, left);
        m.load_some(a.m, a.m_scale, flat, b, left);
        v.load_some(a.v, a.v_scale, flat, b, left);
    }
};

// Updates a block and stores it; FAST: all 256 parameters are there and every pointer is aligned to a lane's eight.
// param, copy (or NULL): the lane's first.
template <bool FAST, typename G, typename Cp, int BITS>
__device__ __forceinline__ void update_block(const AdamwArgs &a, const Block<G, BITS> &in, float *param, Cp *copy, float decay, int64_t b, int left, const Rates &c) {
    const int64_t flat = b * kAdamwBlock + lane_id() * 8;             // in the states
    float p[8], g[8], m[8], v[8];
    in.p.get(p);
    in.g.get(g);
    in.m.get(m);
    in.v.get(v);
    const float keep = (float)(1.0 - (double)c.lr * decay);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float gj = __fmul_rn(g[j], c.grad_scale);
        m[j] = __fadd_rn(__fmul_rn(m[j], a.beta1), __fmul_rn(gj, a.rest1));
        v[j] = __fadd_rn(__fmul_rn(v[j], a.beta2), __fmul_rn(__fmul_rn(gj, gj), a.rest2));
        // root and reciprocal are good to 2^-23 (second moments below 2^-126 count as zero here)
        const float den = __fmaf_rn(root(v[j]), c.grow, a.eps);
        p[j] = __fmaf_rn(p[j], keep, -__fmul_rn(c.rate, __fmul_rn(m[j], reciprocal(den))));
    }
    store8<FAST>(param, left, p);
    if (copy) store8<FAST>(copy, left, p);
    if constexpr (BITS == 32) {
        store8<FAST>(reinterpret_cast<float *>(a.m) + flat, left, m);
        store8<FAST>(reinterpret_cast<float *>(a.v) + flat, left, v);
    } else {
        uint32_t lo[8], hi[8];
        // (eight positions from a multiple of eight on differ in the low word alone)
        const uint32_t place = (uint32_t)flat + (uint32_t)(flat >> 32) * 0x85EBCA6Bu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!FAST && j >= left) m[j] = v[j] = 0.0f;
            const uint32_t h = dither(place + j, c.key);
            lo[j] = (h << 4) & 0xFFFF0u;
            hi[j] = (h >> 12) & 0xFFFF0u;
        }
        const float ms = store8_e4m3<FAST, false>(reinterpret_cast<uint8_t *>(a.m) + flat, left, m, lo);
        const float vs = store8_e4m3<FAST, true>(reinterpret_cast<uint8_t *>(a.v) + flat, left, v, hi);
        if (lane_id() == 0) {
            a.m_scale[b] = ms;
            a.v_scale[b] = vs;
        }
    }
}
// (Out of line: what the ends of tensors need does not weigh on the registers of the common case.)
template <typename G, typename Cp, int BITS>
__device__ __noinline__ void update_end(const AdamwArgs &a, const AdamwTensor &T, int64_t b, const Rates &c) {
    const int64_t at = (b - T.first) * kAdamwBlock + lane_id() * 8;
    const int left = (int)max((int64_t)0, min((int64_t)8, T.count - at));
    Block<G, BITS> in;
    in.load_some(a, T, b, left);
    update_block<false, G, Cp, BITS>(a, in, T.param + at, T.copy ? reinterpret_cast<Cp *>(T.copy) + at : nullptr, T.decay, b, left, c);
}

template <typename G, typename Cp, int BITS>
__global__ void __launch_bounds__(kThreads, kResident) adamw_kernel(const __grid_constant__ AdamwArgs a) {
    __shared__ Rates s_rates;
    pdl_wait();
    const int64_t t = a.counter->step + 1;
    // a warp takes every (warps of the grid)-th block: looks the first one's tensor up, then walks along.  The next block's
    // values are on their way while one is updated.
    const int64_t step = (int64_t)gridDim.x * (kThreads / 32);
    int64_t b = (int64_t)blockIdx.x * (kThreads / 32) + warp_id();
    int k = b < a.blocks ? (int)a.tensor_of[b / kAdamwChunk] : 0;
    AdamwTensor T = a.tensors[k];
    int64_t end = k + 1 < a.n ? a.tensors[k + 1].first : INT64_MAX;
    Block<G, BITS> next;
    auto fetch = [&](int64_t i) {           // block i's tensor and, where it is whole, its values
        if (i >= a.blocks) return false;
        if (i >= end) {
            do {
                ++k;
                end = k + 1 < a.n ? a.tensors[k + 1].first : INT64_MAX;
            } while (i >= end);
            T = a.tensors[k];
        }
        if (!T.wide || (i - T.first + 1) * kAdamwBlock > T.count) return false;
        next.load(a, T, i);
        return true;
    };
    bool whole = fetch(b);
    if (threadIdx.x == 0) {
        const double lr = a.d_lr ? (double)*a.d_lr : a.lr;
        s_rates.rate = (float)(lr / (1.0 - power(a.dbeta1, t)));
        s_rates.grow = (float)(1.0 / sqrt(1.0 - power(a.dbeta2, t)));
        s_rates.lr = (float)lr;
        s_rates.grad_scale = a.grad_scale ? *a.grad_scale : 1.0f;
        s_rates.key = a.seed + (uint32_t)t * 0x9E3779B9u;
    }
    __syncthreads();
    const Rates c = s_rates;
    while (b < a.blocks) {
        if (whole) {
            const Block<G, BITS> now = next;
            const int64_t at = (b - T.first) * kAdamwBlock + lane_id() * 8, done = b;
            float *param = T.param + at;
            Cp *copy = T.copy ? reinterpret_cast<Cp *>(T.copy) + at : nullptr;
            const float decay = T.decay;
            b += step;
            whole = fetch(b);
            update_block<true, G, Cp, BITS>(a, now, param, copy, decay, done, 8, c);
        } else {
            update_end<G, Cp, BITS>(a, a.tensors[k], b, s_rates);
            b += step;
            whole = fetch(b);
        }
    }
    // the last CTA to get here counts the step: every other one has read the counter before
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        if (atomicAdd(&a.counter->ticket, 1u) == gridDim.x - 1) {
            a.counter->ticket = 0;
            a.counter->step = t;
        }
    }
}

template <typename G, typename Cp>
cudaError_t launch_bits(const AdamwArgs &a, int bits, int grid, cudaStream_t st) {
    return bits == 8 ? launch_after(adamw_kernel<G, Cp, 8>, dim3(grid), dim3(kThreads), st, a)
                     : launch_after(adamw_kernel<G, Cp, 32>, dim3(grid), dim3(kThreads), st, a);
}
template <typename G>
cudaError_t launch_copy(const AdamwArgs &a, int copy, int bits, int grid, cudaStream_t st) {
    return copy == 2 ? launch_bits<G, __half>(a, bits, grid, st)
                     : copy == 1 ? launch_bits<G, __nv_bfloat16>(a, bits, grid, st) : launch_bits<G, float>(a, bits, grid, st);
}

}  // namespace

cudaError_t launch_adamw(const AdamwArgs &a, int grad_dtype, int copy_dtype, int state_bits, cudaStream_t st) {
    int64_t grid = (int64_t)sm_count() * kResident;
    if (grid > (a.blocks + kThreads / 32 - 1) / (kThreads / 32)) grid = (a.blocks + kThreads / 32 - 1) / (kThreads / 32);      // (a block for each warp)
    if (grid < 1) grid = 1;
    return grad_dtype == 2   ? launch_copy<__half>(a, copy_dtype, state_bits, (int)grid, st)
           : grad_dtype == 1 ? launch_copy<__nv_bfloat16>(a, copy_dtype, state_bits, (int)grid, st)
                             : launch_copy<float>(a, copy_dtype, state_bits, (int)grid, st);
}

}  // namespace guard
