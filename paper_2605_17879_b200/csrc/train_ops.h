// Host-side launchers and shared pieces of the training-step operators (internal to the library).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kernels.h"

namespace guard {

constexpr uint32_t kStatIndex = 8u;   // a token or target outside its table

// Sets the text guard_last_error(NULL) returns, printf-style, and hands `code` back.
int call_error(int code, const char *fmt, ...);

inline size_t dtype_bytes(int dtype) { return dtype == 0 ? 4 : 2; }

template <typename T> struct Conv;   // a type's values in float32, and the way back (to nearest)
template <> struct Conv<float> {
    static __device__ __forceinline__ float up(float x) { return x; }
    static __device__ __forceinline__ float down(float x) { return x; }
};
template <> struct Conv<__nv_bfloat16> {
    static __device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 down(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Conv<__half> {
    static __device__ __forceinline__ float up(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half down(float x) { return __float2half_rn(x); }
};

struct alignas(16) Bytes16 { uint32_t w[4]; };
struct alignas(32) Bytes32 { uint32_t w[8]; };

// 32 bytes that are read or written once: they do not stay in the first-level cache.
__device__ __forceinline__ Bytes32 load32_once(const void *p) {
    Bytes32 r;
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                 : "l"(p));
    return r;
}
__device__ __forceinline__ void store32_once(void *p, const Bytes32 &r) {
    asm volatile("st.global.L1::no_allocate.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]),
                 "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]), "l"(p)
                 : "memory");
}
__device__ __forceinline__ Bytes16 load16_once(const void *p) {
    Bytes16 r;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p));
    return r;
}
__device__ __forceinline__ void store16_once(void *p, const Bytes16 &r) {
    asm volatile("st.global.L1::no_allocate.v4.b32 [%4], {%0,%1,%2,%3};" ::"r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "l"(p) : "memory");
}

int sm_count();   // SMs of the current device (148 where it cannot be asked)

struct AdamwTensor {
    float *param;
    const void *grad;
    void *copy;             // or NULL
    int64_t count;
    int64_t first;          // block of the flat states where the tensor starts
    float decay;
    uint32_t wide;          // its pointers allow the vector path
};
struct AdamwCounter {       // at the start of the workspace
    int64_t step;
    uint32_t ticket;
};
struct AdamwArgs {
    const AdamwTensor *tensors;
    const uint32_t *tensor_of;   // tensor of every kAdamwChunk-th block
    AdamwCounter *counter;
    int64_t blocks;
    int n;
    float beta1, beta2, rest1, rest2, eps;   // rest: 1 - beta, rounded from float64
    double dbeta1, dbeta2, lr;
    const float *d_lr, *grad_scale;
    void *m, *v;
    float *m_scale, *v_scale;
    uint32_t seed;
};
constexpr int kAdamwBlock = 256;
constexpr int kAdamwChunk = 8;     // blocks to an entry of the table that finds a block's tensor
cudaError_t launch_adamw(const AdamwArgs &a, int grad_dtype, int copy_dtype, int state_bits, cudaStream_t st);

struct EmbedArgs {
    const void *tokens;
    int token_bits;
    int64_t n, rows, width, stride;
    const void *table;
    float scale;
    void *out;
    uint32_t *status;
};
cudaError_t launch_embed(const EmbedArgs &a, int dtype, cudaStream_t st);

struct EmbedGradArgs {
    const void *grad;
    int64_t stride;
    const void *tokens;
    int token_bits;
    int64_t n, rows, width, padding;   // padding: a row, or -1
    float scale;
    int accumulate;
    void *dtable;
    void *workspace;
    uint32_t *status;
};
size_t embed_grad_workspace(int64_t n, int64_t rows, int64_t width);
cudaError_t launch_embed_grad(const EmbedGradArgs &a, int dtype, cudaStream_t st);

struct XentArgs {
    const void *x, *w;
    int64_t rows, width, vocab, x_stride, w_stride;
    int dtype;               // 1 bfloat16, 2 float16
    const void *targets;
    int target_bits;
    int64_t ignore;
    float *loss, *lse_out;   // forward
    const float *lse, *grad_loss;   // backward
    int64_t grad_stride;     // 0 or 1
    void *dx, *dw;           // or NULL
    void *workspace;
    long long wait_limit;    // cycles, of each wait between the warps of the products (0: about a second)
    uint32_t *status;
};
size_t xent_workspace(int64_t rows, int64_t width, int64_t vocab, bool grads);
cudaError_t launch_xent(const XentArgs &x, cudaStream_t st);
cudaError_t launch_xent_grad(const XentArgs &x, cudaStream_t st);

}  // namespace guard
