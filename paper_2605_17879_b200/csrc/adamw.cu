// AdamW over many tensors in one launch, with states in 32 or 8 bits.
//
// Per parameter 28 bytes move with 32-bit states (parameter, both states read and written in float32, a 16-bit gradient
// read, a 16-bit copy written) and 16 with 8-bit ones; some 40 instructions a parameter, so memory bounds it.
//
// A warp takes a block of 256 parameters, eight consecutive ones a lane: the largest loads there are (32 bytes a lane),
// and a block's largest magnitude, which the 8-bit states' scale needs, is one shuffle reduction of values that are in
// registers already.  CTAs take chunks of eight blocks in turn; a table gives the tensor of a chunk's first block, from there
// a warp walks forward, so that tensors of any size and number share one launch.
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

// 32 dithering bits of a position: two multiplicative rounds over position and key.  Neighbouring positions and steps
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

// Eight values of a lane; those behind `left` are zero.
template <typename T>
__device__ __forceinline__ void load8(const T *p, int left, bool wide, float (&x)[8]) {
    if (wide && left >= 8) {
        if constexpr (sizeof(T) == 4) {
            const Bytes32 r = load32_once(p);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(r.w[j]);
        } else {
            const Bytes16 r = load16_once(p);
            const T *t = reinterpret_cast<const T *>(&r);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = Conv<T>::up(t[j]);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? Conv<T>::up(p[j]) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store8(T *p, int left, bool wide, const float (&x)[8]) {
    if (wide && left >= 8) {
        if constexpr (sizeof(T) == 4) {
            Bytes32 r;
#pragma unroll
            for (int j = 0; j < 8; ++j) r.w[j] = __float_as_uint(x[j]);
            store32_once(p, r);
        } else {
            Bytes16 r;
            T *t = reinterpret_cast<T *>(&r);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = Conv<T>::down(x[j]);
            store16_once(p, r);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) p[j] = Conv<T>::down(x[j]);
}
// Eight 8-bit values of a lane, times their scale (a power of two: exact).
__device__ __forceinline__ void load8_e4m3(const uint8_t *p, int left, float scale, float (&x)[8]) {
    uint32_t w[2] = {0, 0};
    if (left >= 8) {
        asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    } else {
        for (int j = 0; j < left; ++j) w[j >> 2] |= (uint32_t)p[j] << (8 * (j & 3));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) from_e4m3x2(w[j >> 1] >> (16 * (j & 1)), x[2 * j], x[2 * j + 1]);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __fmul_rn(x[j], scale);
}
// Stores x as 8-bit values of the block's scale, which it returns: the power of two by which the block's largest magnitude
// comes to lie in (224, 448], 448 being e4m3's largest value.  Powers of two keep the grid of values as it is when the
// scale changes, so a value moves only by what the update adds to it: with the largest magnitude itself as the scale, every
// step would round every value anew, and the noise of that adds up over the 1 / (1 - beta2) steps that a mean remembers.
template <bool LEAST>
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
    if (left >= 8) {
        asm volatile("st.global.L1::no_allocate.v2.b32 [%2], {%0,%1};" ::"r"(w[0]), "r"(w[1]), "l"(p) : "memory");
    } else {
        for (int j = 0; j < left; ++j) p[j] = (uint8_t)(w[j >> 2] >> (8 * (j & 3)));
    }
    return __uint_as_float(e << 23);
}

// Four CTAs an SM (64 registers), and as many in the grid: with 74 registers three fit, and the fourth ran alone after them.
constexpr int kResident = 4;

template <typename G, typename Cp, int BITS>
__global__ void __launch_bounds__(kThreads, kResident) adamw_kernel(const AdamwArgs a) {
    __shared__ float s_rate, s_grow, s_lr;
    pdl_wait();
    const int64_t t = a.counter->step + 1;
    if (threadIdx.x == 0) {
        const double lr = a.d_lr ? (double)*a.d_lr : a.lr;
        s_rate = (float)(lr / (1.0 - power(a.dbeta1, t)));
        s_grow = (float)(1.0 / sqrt(1.0 - power(a.dbeta2, t)));
        s_lr = (float)lr;
    }
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
    const uint32_t key = a.seed + (uint32_t)t * 0x9E3779B9u;
    __syncthreads();
    const float rate = s_rate, grow = s_grow, lr = s_lr;
    const int lane = lane_id(), warp = warp_id();
    const int64_t chunks = (a.blocks + kAdamwChunk - 1) / kAdamwChunk;
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        int k = (int)a.tensor_of[c];
        const int64_t end = min(a.blocks, (c + 1) * kAdamwChunk);
        for (int64_t b = c * kAdamwChunk + warp; b < end; b += kThreads / 32) {
            while (k + 1 < a.n && a.tensors[k + 1].first <= b) ++k;
            const AdamwTensor T = a.tensors[k];
            const int64_t at = (b - T.first) * kAdamwBlock + lane * 8;   // in the tensor
            const int64_t flat = b * kAdamwBlock + lane * 8;             // in the states
            const int left = (int)max((int64_t)0, min((int64_t)8, T.count - at));
            const bool wide = T.wide != 0;
            float p[8], g[8], m[8], v[8];
            load8(T.param + at, left, wide, p);
            load8(reinterpret_cast<const G *>(T.grad) + at, left, wide, g);
            if constexpr (BITS == 32) {
                load8(reinterpret_cast<const float *>(a.m) + flat, left, true, m);
                load8(reinterpret_cast<const float *>(a.v) + flat, left, true, v);
            } else {
                load8_e4m3(reinterpret_cast<const uint8_t *>(a.m) + flat, left, a.m_scale[b], m);
                load8_e4m3(reinterpret_cast<const uint8_t *>(a.v) + flat, left, a.v_scale[b], v);
            }
            const float keep = (float)(1.0 - (double)lr * T.decay);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gj = __fmul_rn(g[j], gs);
                m[j] = __fadd_rn(__fmul_rn(m[j], a.beta1), __fmul_rn(gj, a.rest1));
                v[j] = __fadd_rn(__fmul_rn(v[j], a.beta2), __fmul_rn(__fmul_rn(gj, gj), a.rest2));
                // root and reciprocal are good to 2^-23 (second moments below 2^-126 count as zero here)
                const float den = __fmaf_rn(root(v[j]), grow, a.eps);
                p[j] = __fmaf_rn(p[j], keep, -__fmul_rn(rate, __fmul_rn(m[j], reciprocal(den))));
            }
            store8(T.param + at, left, wide, p);
            if (T.copy) store8(reinterpret_cast<Cp *>(T.copy) + at, left, wide, p);
            if constexpr (BITS == 32) {
                store8(reinterpret_cast<float *>(a.m) + flat, left, true, m);
                store8(reinterpret_cast<float *>(a.v) + flat, left, true, v);
            } else {
                uint32_t lo[8], hi[8];
                // (eight positions from a multiple of eight on differ in the low word alone)
                const uint32_t place = (uint32_t)flat + (uint32_t)(flat >> 32) * 0x85EBCA6Bu;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j >= left) m[j] = v[j] = 0.0f;
                    const uint32_t h = dither(place + j, key);
                    lo[j] = (h << 4) & 0xFFFF0u;
                    hi[j] = (h >> 12) & 0xFFFF0u;
                }
                const float ms = store8_e4m3<false>(reinterpret_cast<uint8_t *>(a.m) + flat, left, m, lo);
                const float vs = store8_e4m3<true>(reinterpret_cast<uint8_t *>(a.v) + flat, left, v, hi);
                if (lane == 0) {
                    a.m_scale[b] = ms;
                    a.v_scale[b] = vs;
                }
            }
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
    const int64_t chunks = (a.blocks + kAdamwChunk - 1) / kAdamwChunk;
    int64_t grid = (int64_t)sm_count() * kResident;
    if (grid > chunks) grid = chunks;
    if (grid < 1) grid = 1;
    return grad_dtype == 2   ? launch_copy<__half>(a, copy_dtype, state_bits, (int)grid, st)
           : grad_dtype == 1 ? launch_copy<__nv_bfloat16>(a, copy_dtype, state_bits, (int)grid, st)
                             : launch_copy<float>(a, copy_dtype, state_bits, (int)grid, st);
}

}  // namespace guard
