// C entries of the training-step operators: argument checks on the host, then the launches.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>
#include <vector>

#include "../../include/guard_b200.h"
#include "train_ops.h"

namespace guard {

int call_error(int code, const char *fmt, ...) {
    char text[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    set_global_error(text);
    return code;
}

int sm_count() {
    static std::atomic<int> known[64];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < 64) {
        n = known[dev].load(std::memory_order_relaxed);
        if (n > 0) return n;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n >= 2) {
            known[dev].store(n, std::memory_order_relaxed);
            return n;
        }
    }
    (void)cudaGetLastError();
    return 148;
}

}  // namespace guard

using namespace guard;

namespace {

bool good_dtype(int d) { return d == GUARD_F32 || d == GUARD_BF16 || d == GUARD_F16; }
bool on(const void *p, size_t to) { return (uintptr_t)p % to == 0; }
int launched(cudaError_t e, const char *what) {
    return e == cudaSuccess ? GUARD_OK : call_error(GUARD_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
}
// A row-major matrix: sizes whose last element's offset fits 62 bits.
bool good_matrix(int64_t rows, int64_t width, int64_t stride) {
    return rows >= 0 && width >= 1 && width <= (1 << 24) && stride >= width && stride < (1LL << 40) && rows < (1LL << 60) / stride;
}
// The status word and other scalars that kernels access.
bool good_word(const void *p, const char *name) {
    if (on(p, 4)) return true;
    call_error(GUARD_ERR_ARG, "%s is not aligned to its four bytes", name);
    return false;
}
// Whether the stream is being captured (a graph would copy from or to host memory that is gone when it is replayed).
int not_capturing(void *stream, const char *what) {
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    const cudaError_t e = cudaStreamIsCapturing((cudaStream_t)stream, &status);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return call_error(GUARD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    return status == cudaStreamCaptureStatusNone ? GUARD_OK : call_error(GUARD_ERR_ARG, "%s cannot be captured into a graph", what);
}
bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    return na && nb && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

}  // namespace

struct guard_adamw {
    AdamwArgs a;
    int grad_dtype, copy_dtype, bits;
};

extern "C" {

int guard_embed(const void *d_tokens, int token_bits, int64_t tokens, const void *d_table, int64_t rows, int64_t width,
                int64_t stride, int dtype, float scale, void *d_out, uint32_t *d_status, void *stream) {
    if (!good_dtype(dtype) || (token_bits != 32 && token_bits != 64)) return call_error(GUARD_ERR_ARG, "dtype must be GUARD_F32, _BF16 or _F16, token_bits 32 or 64");
    if (tokens < 0 || !good_matrix(rows, width, stride) || !good_matrix(tokens, width, width))
        return call_error(GUARD_ERR_ARG, "invalid sizes: need tokens >= 0, rows >= 0, 1 <= width <= 2^24, stride >= width");
    if (tokens == 0) return GUARD_OK;
    if (!d_tokens || !d_out || (!d_table && rows > 0)) return call_error(GUARD_ERR_ARG, "d_tokens, d_table or d_out is NULL");
    const size_t b = dtype_bytes(dtype);
    if (!on(d_tokens, token_bits / 8) || !on(d_table, b) || !on(d_out, b)) return call_error(GUARD_ERR_ARG, "a pointer is not aligned to its elements");
    if (!good_word(d_status, "d_status")) return GUARD_ERR_ARG;
    const size_t nout = (size_t)tokens * width * b;
    if (overlap(d_out, nout, d_tokens, (size_t)tokens * token_bits / 8) || overlap(d_out, nout, d_table, rows ? ((size_t)(rows - 1) * stride + width) * b : 0))
        return call_error(GUARD_ERR_ARG, "d_out overlaps an input");
    EmbedArgs a{};
    a.tokens = d_tokens;
    a.token_bits = token_bits;
    a.n = tokens;
    a.rows = rows;
    a.width = width;
    a.stride = stride;
    a.table = d_table;
    a.scale = scale;
    a.out = d_out;
    a.status = d_status;
    return launched(launch_embed(a, dtype, (cudaStream_t)stream), "embedding");
}

size_t guard_embed_grad_workspace_bytes(int64_t tokens, int64_t rows, int64_t width) {
    if (tokens < 0 || tokens > (1LL << 30) || rows < 0 || rows >= 0x7FFFFFFFLL || !good_matrix(tokens, width, width) || !good_matrix(rows, width, width)) return 0;
    return embed_grad_workspace(tokens, rows, width);
}

int guard_embed_grad(const void *d_grad, int64_t stride, int dtype, const void *d_tokens, int token_bits, int64_t tokens,
                     int64_t rows, int64_t width, float scale, int64_t padding_idx, int accumulate, void *d_dtable,
                     void *d_workspace, size_t workspace_bytes, uint32_t *d_status, void *stream) {
    if (!good_dtype(dtype) || (token_bits != 32 && token_bits != 64)) return call_error(GUARD_ERR_ARG, "dtype must be GUARD_F32, _BF16 or _F16, token_bits 32 or 64");
    const size_t need = guard_embed_grad_workspace_bytes(tokens, rows, width);
    if (need == 0 || !good_matrix(tokens, width, stride))
        return call_error(GUARD_ERR_ARG, "invalid sizes: need 0 <= tokens <= 2^30, 0 <= rows < 2^31 - 1, 1 <= width <= 2^24, stride >= width");
    if (padding_idx < -1 || padding_idx >= rows) {
        if (rows > 0 || padding_idx != -1) return call_error(GUARD_ERR_ARG, "padding_idx must be -1 or a row");
    }
    if (rows == 0) return GUARD_OK;
    if (!d_dtable || (tokens > 0 && (!d_grad || !d_tokens))) return call_error(GUARD_ERR_ARG, "d_grad, d_tokens or d_dtable is NULL");
    const size_t b = dtype_bytes(dtype);
    if (!on(d_tokens, token_bits / 8) || !on(d_grad, b) || !on(d_dtable, b)) return call_error(GUARD_ERR_ARG, "a pointer is not aligned to its elements");
    if (!good_word(d_status, "d_status")) return GUARD_ERR_ARG;
    const size_t nout = (size_t)rows * width * b;
    if (overlap(d_dtable, nout, d_tokens, (size_t)tokens * token_bits / 8) || overlap(d_dtable, nout, d_grad, tokens ? ((size_t)(tokens - 1) * stride + width) * b : 0) ||
        overlap(d_dtable, nout, d_workspace, need))
        return call_error(GUARD_ERR_ARG, "d_dtable overlaps an input or the workspace");
    if (d_workspace && (overlap(d_workspace, need, d_tokens, (size_t)tokens * token_bits / 8) ||
                        overlap(d_workspace, need, d_grad, tokens ? ((size_t)(tokens - 1) * stride + width) * b : 0)))
        return call_error(GUARD_ERR_ARG, "an input overlaps the workspace");
    if (!d_workspace || !on(d_workspace, 256) || workspace_bytes < need)
        return call_error(GUARD_ERR_WORKSPACE, "workspace must be non-NULL, 256-byte aligned and at least %zu bytes", need);
    if (tokens == 0 && accumulate) return GUARD_OK;
    EmbedGradArgs a{};
    a.grad = d_grad;
    a.stride = stride;
    a.tokens = d_tokens;
    a.token_bits = token_bits;
    a.n = tokens;
    a.rows = rows;
    a.width = width;
    a.padding = padding_idx;
    a.scale = scale;
    a.accumulate = accumulate != 0;
    a.dtable = d_dtable;
    a.workspace = d_workspace;
    a.status = d_status;
    return launched(launch_embed_grad(a, dtype, (cudaStream_t)stream), "embedding gradient");
}

size_t guard_linear_xent_workspace_bytes(int64_t rows, int64_t width, int64_t vocab, int grads) {
    if (rows < 1 || rows > (1LL << 26) || width < 8 || width > (1 << 24) || width % 8 || vocab < 1 || vocab > (1LL << 30)) return 0;
    // tiles are counted in 32 bits (at most 148 splits of the depth)
    if (((rows + 127) / 128) * ((vocab + 255) / 256) > (1LL << 30) || ((rows + 127) / 128) * ((width + 255) / 256) > (1LL << 23) ||
        ((vocab + 127) / 128) * ((width + 255) / 256) > (1LL << 30))
        return 0;
    return xent_workspace(rows, width, vocab, grads != 0);
}

static std::atomic<long long> g_wait_limit{0};

int guard_debug_set_operator_wait_limit(long long cycles) {
    if (cycles < 0) return call_error(GUARD_ERR_ARG, "cycles must not be negative");
    g_wait_limit.store(cycles, std::memory_order_relaxed);
    return GUARD_OK;
}
static int xent_sizes() {
    return call_error(GUARD_ERR_ARG, "invalid sizes: need 1 <= vocab <= 2^30, rows <= 2^26, width a multiple of 8 up to 2^24, strides multiples of 8 and >= width, and a product that tiles");
}

// The checks that both directions share; 0 or an error.
static int xent_check(const XentArgs &a, size_t need, size_t given, const void *out0, size_t n0, const void *out1, size_t n1) {
    if ((a.dtype != GUARD_BF16 && a.dtype != GUARD_F16) || (a.target_bits != 32 && a.target_bits != 64))
        return call_error(GUARD_ERR_ARG, "dtype must be GUARD_BF16 or GUARD_F16, target_bits 32 or 64");
    if (need == 0 || a.x_stride < a.width || a.w_stride < a.width || a.x_stride % 8 || a.w_stride % 8 || a.x_stride >= (1LL << 36) || a.w_stride >= (1LL << 36))
        return xent_sizes();
    if (!a.x || !a.w || !a.targets) return call_error(GUARD_ERR_ARG, "d_x, d_w or d_targets is NULL");
    if (!good_word(a.status, "d_status")) return GUARD_ERR_ARG;
    if (!on(a.x, 16) || !on(a.w, 16) || !on(a.targets, a.target_bits / 8)) return call_error(GUARD_ERR_ARG, "d_x and d_w must be 16-byte aligned, d_targets to its elements");
    if (!a.workspace || !on(a.workspace, 256) || given < need)
        return call_error(GUARD_ERR_WORKSPACE, "workspace must be non-NULL, 256-byte aligned and at least %zu bytes", need);
    const struct { const void *p; size_t n; } ins[] = {{a.x, ((size_t)(a.rows - 1) * a.x_stride + a.width) * 2}, {a.w, ((size_t)(a.vocab - 1) * a.w_stride + a.width) * 2},
                                                       {a.targets, (size_t)a.rows * a.target_bits / 8}, {a.lse, (size_t)a.rows * 4},
                                                       {a.grad_loss, a.grad_stride ? (size_t)a.rows * 4 : 4}, {a.workspace, need}};
    for (const auto &in : ins) {
        if (in.p && (overlap(out0, out0 ? n0 : 0, in.p, in.n) || overlap(out1, out1 ? n1 : 0, in.p, in.n))) return call_error(GUARD_ERR_ARG, "an output overlaps an input or the workspace");
        if (in.p && &in != &ins[5] && overlap(a.workspace, need, in.p, in.n)) return call_error(GUARD_ERR_ARG, "an input overlaps the workspace");
    }
    if (out0 && out1 && overlap(out0, n0, out1, n1)) return call_error(GUARD_ERR_ARG, "the outputs overlap");
    return GUARD_OK;
}

int guard_linear_xent(const void *d_x, int64_t x_stride, const void *d_w, int64_t w_stride, int64_t rows, int64_t width,
                      int64_t vocab, int dtype, const void *d_targets, int target_bits, int64_t ignore_index,
                      float *d_loss, float *d_lse, void *d_workspace, size_t workspace_bytes, uint32_t *d_status,
                      void *stream) {
    if (rows == 0 && guard_linear_xent_workspace_bytes(1, width, vocab, 0) != 0) return GUARD_OK;
    XentArgs a{};
    a.x = d_x;
    a.w = d_w;
    a.rows = rows;
    a.width = width;
    a.vocab = vocab;
    a.x_stride = x_stride;
    a.w_stride = w_stride;
    a.dtype = dtype;
    a.targets = d_targets;
    a.target_bits = target_bits;
    a.ignore = ignore_index;
    a.loss = d_loss;
    a.lse_out = d_lse;
    a.workspace = d_workspace;
    a.status = d_status;
    a.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
    if (!d_loss || !d_lse || !on(d_loss, 4) || !on(d_lse, 4)) return call_error(GUARD_ERR_ARG, "d_loss and d_lse must be non-NULL and aligned to their elements");
    const int rc = xent_check(a, guard_linear_xent_workspace_bytes(rows, width, vocab, 0), workspace_bytes, d_loss, (size_t)rows * 4, d_lse, (size_t)rows * 4);
    if (rc != GUARD_OK) return rc;
    return launched(launch_xent(a, (cudaStream_t)stream), "cross entropy");
}

int guard_linear_xent_grad(const void *d_x, int64_t x_stride, const void *d_w, int64_t w_stride, int64_t rows, int64_t width,
                           int64_t vocab, int dtype, const void *d_targets, int target_bits, int64_t ignore_index,
                           const float *d_lse, const float *d_grad_loss, int grad_stride, void *d_dx, void *d_dw,
                           void *d_workspace, size_t workspace_bytes, uint32_t *d_status, void *stream) {
    if (grad_stride != 0 && grad_stride != 1) return call_error(GUARD_ERR_ARG, "grad_stride must be 0 or 1");
    if (!d_dx && !d_dw) return call_error(GUARD_ERR_ARG, "d_dx and d_dw are both NULL");
    if (!on(d_dx, 16) || !on(d_dw, 16)) return call_error(GUARD_ERR_ARG, "d_dx and d_dw must be 16-byte aligned");
    if (rows == 0 && (dtype == GUARD_BF16 || dtype == GUARD_F16)) {       // dw is all there is to write
        if (guard_linear_xent_workspace_bytes(1, width, vocab, 1) == 0 || w_stride < width || w_stride % 8 || w_stride >= (1LL << 36)) return xent_sizes();
        if (!d_dw) return GUARD_OK;
        const size_t ndw = (size_t)vocab * width * 2;
        if ((d_w && overlap(d_dw, ndw, d_w, ((size_t)(vocab - 1) * w_stride + width) * 2)) || overlap(d_dw, ndw, d_workspace, workspace_bytes))
            return call_error(GUARD_ERR_ARG, "an output overlaps an input or the workspace");
        const cudaError_t e = cudaMemsetAsync(d_dw, 0, ndw, (cudaStream_t)stream);
        if (e == cudaSuccess) return GUARD_OK;
        (void)cudaGetLastError();
        return call_error(GUARD_ERR_CUDA, "cudaMemsetAsync: %s", cudaGetErrorString(e));
    }
    XentArgs a{};
    a.x = d_x;
    a.w = d_w;
    a.rows = rows;
    a.width = width;
    a.vocab = vocab;
    a.x_stride = x_stride;
    a.w_stride = w_stride;
    a.dtype = dtype;
    a.targets = d_targets;
    a.target_bits = target_bits;
    a.ignore = ignore_index;
    a.lse = d_lse;
    a.grad_loss = d_grad_loss;
    a.grad_stride = grad_stride;
    a.dx = d_dx;
    a.dw = d_dw;
    a.workspace = d_workspace;
    a.status = d_status;
    a.wait_limit = g_wait_limit.load(std::memory_order_relaxed);
    if (!d_lse || !d_grad_loss || !on(d_lse, 4) || !on(d_grad_loss, 4)) return call_error(GUARD_ERR_ARG, "d_lse and d_grad_loss must be non-NULL and aligned to their elements");
    const int rc = xent_check(a, guard_linear_xent_workspace_bytes(rows, width, vocab, 1), workspace_bytes, d_dx, (size_t)rows * width * 2, d_dw, (size_t)vocab * width * 2);
    if (rc != GUARD_OK) return rc;
    return launched(launch_xent_grad(a, (cudaStream_t)stream), "cross entropy gradient");
}

int64_t guard_adamw_blocks(const guard_adamw_tensor *tensors, int n) {
    if (n < 0 || (n > 0 && !tensors)) return -1;
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) {
        if (tensors[i].count < 0 || tensors[i].count > (1LL << 44)) return -1;
        blocks += (tensors[i].count + kAdamwBlock - 1) / kAdamwBlock;
    }
    return blocks;
}

size_t guard_adamw_workspace_bytes(const guard_adamw_tensor *tensors, int n) {
    const int64_t blocks = guard_adamw_blocks(tensors, n);
    if (blocks < 0 || blocks > (1LL << 36)) return 0;
    const size_t table = 256 + ((size_t)n * sizeof(AdamwTensor) + 255) / 256 * 256;
    return table + (size_t)((blocks + kAdamwChunk - 1) / kAdamwChunk) * sizeof(uint32_t);
}

int guard_adamw_create(guard_adamw **out, const guard_adamw_tensor *tensors, int n, int grad_dtype, int copy_dtype,
                       int state_bits, double beta1, double beta2, double eps, void *d_m, void *d_v, float *d_m_scale,
                       float *d_v_scale, int64_t step, uint32_t seed, void *d_workspace, size_t workspace_bytes,
                       void *stream) {
    if (!out) return call_error(GUARD_ERR_ARG, "out is NULL");
    *out = nullptr;
    const size_t need = guard_adamw_workspace_bytes(tensors, n);
    if (n < 1 || need == 0) return call_error(GUARD_ERR_ARG, "need at least one tensor, counts >= 0");
    if (!good_dtype(grad_dtype) || !good_dtype(copy_dtype)) return call_error(GUARD_ERR_ARG, "grad_dtype and copy_dtype must be GUARD_F32, _BF16 or _F16");
    if (state_bits != 8 && state_bits != 32) return call_error(GUARD_ERR_ARG, "state_bits must be 8 or 32");
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 1e-30) || !std::isfinite((float)eps) || step < 0)
        return call_error(GUARD_ERR_ARG, "need 0 <= beta < 1, 1e-30 <= eps finite in float32, and step >= 0");
    const int64_t blocks = guard_adamw_blocks(tensors, n);
    if (blocks > 0 && (!d_m || !d_v || !on(d_m, 32) || !on(d_v, 32))) return call_error(GUARD_ERR_ARG, "d_m and d_v must be non-NULL and 32-byte aligned");
    if (blocks > 0 && state_bits == 8 && (!d_m_scale || !d_v_scale || !on(d_m_scale, 4) || !on(d_v_scale, 4)))
        return call_error(GUARD_ERR_ARG, "8-bit states need d_m_scale and d_v_scale");
    if (!d_workspace || !on(d_workspace, 256) || workspace_bytes < need)
        return call_error(GUARD_ERR_WORKSPACE, "workspace must be non-NULL, 256-byte aligned and at least %zu bytes", need);
    try {
        // what the update writes must be apart from all that it reads or writes elsewhere
        struct Range { uintptr_t from, to; bool writes; };
        std::vector<Range> ranges;
        auto add = [&](const void *p, size_t bytes, bool writes) { if (p && bytes) ranges.push_back({(uintptr_t)p, (uintptr_t)p + bytes, writes}); };
        const size_t gb = dtype_bytes(grad_dtype), cb = dtype_bytes(copy_dtype), sb = state_bits / 8;
        std::vector<char> host(need, 0);
        AdamwCounter *counter = (AdamwCounter *)host.data();
        AdamwTensor *table = (AdamwTensor *)(host.data() + 256);
        const size_t map_at = 256 + ((size_t)n * sizeof(AdamwTensor) + 255) / 256 * 256;
        uint32_t *map = (uint32_t *)(host.data() + map_at);
        counter->step = step;
        int64_t first = 0;
        for (int i = 0; i < n; ++i) {
            const guard_adamw_tensor &t = tensors[i];
            if (t.count > 0 && (!t.d_param || !t.d_grad)) return call_error(GUARD_ERR_ARG, "tensor %d: d_param or d_grad is NULL", i);
            if (!on(t.d_param, 4) || !on(t.d_grad, gb) || !on(t.d_copy, cb)) return call_error(GUARD_ERR_ARG, "tensor %d: a pointer is not aligned to its elements", i);
            if (!std::isfinite(t.weight_decay)) return call_error(GUARD_ERR_ARG, "tensor %d: weight_decay is not finite", i);
            AdamwTensor &d = table[i];
            d.param = t.d_param;
            d.grad = t.d_grad;
            d.copy = t.d_copy;
            d.count = t.count;
            d.first = first;
            d.decay = t.weight_decay;
            d.wide = on(t.d_param, 32) && on(t.d_grad, gb == 4 ? 32 : 16) && on(t.d_copy, cb == 4 ? 32 : 16);
            add(t.d_param, (size_t)t.count * 4, true);
            add(t.d_grad, (size_t)t.count * gb, false);
            add(t.d_copy, (size_t)t.count * cb, true);
            first += (t.count + kAdamwBlock - 1) / kAdamwBlock;
        }
        add(d_m, (size_t)blocks * kAdamwBlock * sb, true);
        add(d_v, (size_t)blocks * kAdamwBlock * sb, true);
        if (state_bits == 8) {
            add(d_m_scale, (size_t)blocks * 4, true);
            add(d_v_scale, (size_t)blocks * 4, true);
        }
        add(d_workspace, need, true);
        std::sort(ranges.begin(), ranges.end(), [](const Range &x, const Range &y) { return x.from < y.from; });
        uintptr_t end_all = 0, end_write = 0;
        for (const Range &r : ranges) {
            if (r.from < end_write || (r.writes && r.from < end_all)) return call_error(GUARD_ERR_ARG, "parameters, copies, states and the workspace must not overlap one another or a gradient");
            end_all = std::max(end_all, r.to);
            if (r.writes) end_write = std::max(end_write, r.to);
        }
        for (int64_t c = 0, i = 0; c * kAdamwChunk < blocks; ++c) {
            while (i + 1 < n && table[i + 1].first <= c * kAdamwChunk) ++i;
            map[c] = (uint32_t)i;
        }
        const int free = not_capturing(stream, "guard_adamw_create");
        if (free != GUARD_OK) return free;
        guard_adamw *o = new guard_adamw();
        o->grad_dtype = grad_dtype;
        o->copy_dtype = copy_dtype;
        o->bits = state_bits;
        AdamwArgs &a = o->a;
        a = AdamwArgs{};
        a.counter = (AdamwCounter *)d_workspace;
        a.tensors = (const AdamwTensor *)((char *)d_workspace + 256);
        a.tensor_of = (const uint32_t *)((char *)d_workspace + map_at);
        a.blocks = blocks;
        a.n = n;
        a.dbeta1 = beta1;
        a.dbeta2 = beta2;
        a.beta1 = (float)beta1;
        a.beta2 = (float)beta2;
        a.rest1 = (float)(1.0 - beta1);
        a.rest2 = (float)(1.0 - beta2);
        a.eps = (float)eps;
        a.m = d_m;
        a.v = d_v;
        a.m_scale = d_m_scale;
        a.v_scale = d_v_scale;
        a.seed = seed;
        // (a copy from pageable memory has left `host` when the call returns)
        const cudaError_t e = cudaMemcpyAsync(d_workspace, host.data(), need, cudaMemcpyHostToDevice, (cudaStream_t)stream);
        if (e != cudaSuccess) {
            delete o;
            (void)cudaGetLastError();
            return call_error(GUARD_ERR_CUDA, "copy of the tensor table: %s", cudaGetErrorString(e));
        }
        *out = o;
        return GUARD_OK;
    } catch (...) {
        return call_error(GUARD_ERR_ARG, "out of host memory");
    }
}

int guard_adamw_step(guard_adamw *opt, double lr, const float *d_lr, const float *d_grad_scale, void *stream) {
    if (!opt) return call_error(GUARD_ERR_ARG, "opt is NULL");
    if (!d_lr && !std::isfinite(lr)) return call_error(GUARD_ERR_ARG, "lr is not finite");
    if (!good_word(d_lr, "d_lr") || !good_word(d_grad_scale, "d_grad_scale")) return GUARD_ERR_ARG;
    AdamwArgs a = opt->a;
    a.lr = lr;
    a.d_lr = d_lr;
    a.grad_scale = d_grad_scale;
    return launched(launch_adamw(a, opt->grad_dtype, opt->copy_dtype, opt->bits, (cudaStream_t)stream), "AdamW");
}

int guard_adamw_steps(guard_adamw *opt, int64_t *steps, void *stream) {
    if (!opt || !steps) return call_error(GUARD_ERR_ARG, "opt or steps is NULL");
    const int free = not_capturing(stream, "guard_adamw_steps");
    if (free != GUARD_OK) return free;
    cudaError_t e = cudaMemcpyAsync(steps, &opt->a.counter->step, sizeof *steps, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e == cudaSuccess) return GUARD_OK;
    (void)cudaGetLastError();
    return call_error(GUARD_ERR_CUDA, "reading the step counter: %s", cudaGetErrorString(e));
}

void guard_adamw_destroy(guard_adamw *opt) { delete opt; }

}  // extern "C"
