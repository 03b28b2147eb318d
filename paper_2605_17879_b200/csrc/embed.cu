// Token embedding with scaling, and its gradient by sorted tokens.
//
// Lookup: out[i] = scale * table[token[i]].  Pure copying: bound by reading each different row and writing every output row.
//
// Gradient: dtable[v] = scale * sum of the gradient rows of the positions with token v.  Summing with atomics would make
// the order, and with it the result, a matter of chance, and would serialise on frequent tokens; so the positions are sorted
// by token first (a stable radix sort), then every row of the table has one writer.
//   1. embed_sort_*: least significant digit first, kDigitBits at a time; a CTA ranks a tile of keys with warp matches and
//      counters of its own, so equal keys keep their order.  One tile: all digits in one launch.  More: two launches per digit.
//   2. embed_window_kernel: the first and last position of every token, and the sums of those windows of 64 sorted positions
//      that belong to one token altogether, in float32, so that a token that occurs thousands of times is summed by many warps.
//   3. embed_rows_kernel: a warp per row of the table adds its windows and the positions at both ends, or writes zeros.  A
//      row of many windows is added by the whole CTA.
// The grouping of a sum depends on the positions alone.
#include "train_ops.h"

namespace guard {

namespace {

constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 512;            // one per digit in the scans
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 4;                // keys a thread ranks at a time
constexpr int kTile = kSortThreads * kSortItems;
constexpr int kWindow = 64;
constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kCols = 8;                     // columns a lane holds at a time

__device__ __forceinline__ int64_t token_at(const void *tokens, int bits, int64_t i) {
    return bits == 64 ? __ldg(reinterpret_cast<const long long *>(tokens) + i) : (int64_t)__ldg(reinterpret_cast<const int *>(tokens) + i);
}

// ---- lookup ----------------------------------------------------------------------------------------------------------

// Eight columns of a row, those behind `left` as they are.
template <typename T>
__device__ __forceinline__ void load_cols(const T *p, int left, bool wide, float (&x)[kCols]) {
    if (wide && left >= kCols) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 r = reinterpret_cast<const float4 *>(p)[h];
                x[4 * h] = r.x, x[4 * h + 1] = r.y, x[4 * h + 2] = r.z, x[4 * h + 3] = r.w;
            }
        } else {
            const uint4 r = *reinterpret_cast<const uint4 *>(p);
            const T *t = reinterpret_cast<const T *>(&r);
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = Conv<T>::up(t[j]);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < kCols; ++j) x[j] = j < left ? Conv<T>::up(p[j]) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_cols(T *p, int left, bool wide, const float (&x)[kCols]) {
    if (wide && left >= kCols) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                reinterpret_cast<float4 *>(p)[h] = make_float4(x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]);
        } else {
            Bytes16 r;
            T *t = reinterpret_cast<T *>(&r);
#pragma unroll
            for (int j = 0; j < kCols; ++j) t[j] = Conv<T>::down(x[j]);
            *reinterpret_cast<Bytes16 *>(p) = r;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < kCols; ++j)
        if (j < left) p[j] = Conv<T>::down(x[j]);
}

template <typename T>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a, int groups, bool wide) {
    pdl_wait();
    const int64_t work = a.n * groups;
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < work; w += (int64_t)gridDim.x * 256) {
        const int64_t i = w / groups;
        const int64_t col = (w - i * groups) * kCols;
        const int64_t tok = token_at(a.tokens, a.token_bits, i);
        const int left = (int)min((int64_t)kCols, a.width - col);
        float x[kCols];
        if (tok >= 0 && tok < a.rows) {
            load_cols(reinterpret_cast<const T *>(a.table) + tok * a.stride + col, left, wide, x);
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = __fmul_rn(x[j], a.scale);
        } else {
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = __uint_as_float(0x7FC00000u);
            if (col == 0 && a.status) atomicOr(a.status, kStatIndex);
        }
        store_cols(reinterpret_cast<T *>(a.out) + i * a.width + col, left, wide, x);
    }
}

// ---- sorting positions by token ---------------------------------------------------------------------------------------

struct SortShared {
    uint16_t count[kSortWarps][kDigits];   // keys of a digit per warp, then the number before that warp
    uint32_t base[kDigits];                // where a digit's keys of this tile go
    uint32_t scan[kSortWarps];
};

// A position's key: its token, or `rows` (behind all tokens) where it adds nothing.
__device__ __forceinline__ uint32_t key_at(const EmbedGradArgs &a, int64_t i) {
    const int64_t t = token_at(a.tokens, a.token_bits, i);
    if (t == a.padding) return (uint32_t)a.rows;
    if (t < 0 || t >= a.rows) {
        if (a.status) atomicOr(a.status, kStatIndex);
        return (uint32_t)a.rows;
    }
    return (uint32_t)t;
}

// Ranks the tile's keys by a digit.  Thread holds kSortItems keys, warp after warp and 32 at a time in order, so that rank
// order is position order.  rank[r]: number of keys of the same digit before this one in the warp; counts per warp in s.count.
__device__ __forceinline__ void rank_tile(SortShared &s, const uint32_t (&key)[kSortItems], const bool (&have)[kSortItems], int shift,
                                          uint32_t (&rank)[kSortItems]) {
    for (int d = threadIdx.x; d < kSortWarps * kDigits; d += kSortThreads) (&s.count[0][0])[d] = 0;
    __syncthreads();
    const int warp = warp_id(), lane = lane_id();
    for (int r = 0; r < kSortItems; ++r) {
        const uint32_t digit = have[r] ? (key[r] >> shift) & (kDigits - 1) : kDigits;
        const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
        const int first = __ffs(same) - 1;
        uint32_t before = 0;
        if (lane == first && have[r]) {
            before = s.count[warp][digit];
            s.count[warp][digit] = (uint16_t)(before + __popc(same));
        }
        before = __shfl_sync(0xFFFFFFFFu, before, first);
        rank[r] = before + __popc(same & ((1u << lane) - 1));
        __syncwarp();
    }
    __syncthreads();
}

// Turns s.count into the numbers before each warp; returns the tile's count of digit threadIdx.x.
__device__ __forceinline__ uint32_t warps_before(SortShared &s) {
    const int d = threadIdx.x;
    uint32_t sum = 0;
    for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = s.count[w][d];
        s.count[w][d] = (uint16_t)sum;
        sum += c;
    }
    return sum;
}

// Exclusive prefix over the digits (one a thread).
__device__ __forceinline__ uint32_t digits_before(SortShared &s, uint32_t mine) {
    uint32_t x = mine;
    const int lane = lane_id(), warp = warp_id();
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) s.scan[warp] = x;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < warp; ++w) before += s.scan[w];
    __syncthreads();
    return before + x - mine;
}

__device__ __forceinline__ void clear_bounds(uint2 *bounds, int64_t rows) {
    for (int64_t v = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; v < rows; v += (int64_t)gridDim.x * kSortThreads) bounds[v] = make_uint2(0, 0);
}

struct SortArgs {
    EmbedGradArgs a;
    const uint32_t *in_key, *in_pos;   // the previous digit's order (unused for the first digit)
    uint32_t *out_key, *out_pos;
    uint32_t *counts;                  // [tiles][kDigits]
    uint2 *bounds;
    int64_t tiles;
    int shift, digits, first;
};

__device__ __forceinline__ void load_tile(const SortArgs &s, int64_t tile, uint32_t (&key)[kSortItems], uint32_t (&pos)[kSortItems],
                                          bool (&have)[kSortItems]) {
    const int64_t at = tile * kTile + (int64_t)warp_id() * (32 * kSortItems) + lane_id();
#pragma unroll
    for (int r = 0; r < kSortItems; ++r) {
        const int64_t i = at + r * 32;
        have[r] = i < s.a.n;
        key[r] = 0;
        pos[r] = 0;
        if (have[r]) {
            key[r] = s.first ? key_at(s.a, i) : s.in_key[i];
            pos[r] = s.first ? (uint32_t)i : s.in_pos[i];
        }
    }
}

// Keys of every digit value in a tile.
__global__ void __launch_bounds__(kSortThreads) embed_sort_count_kernel(const SortArgs s) {
    __shared__ uint32_t count[kDigits];
    pdl_wait();
    count[threadIdx.x] = 0;
    __syncthreads();
    uint32_t key[kSortItems], pos[kSortItems];
    bool have[kSortItems];
    load_tile(s, blockIdx.x, key, pos, have);
#pragma unroll
    for (int r = 0; r < kSortItems; ++r)
        if (have[r]) atomicAdd(&count[(key[r] >> s.shift) & (kDigits - 1)], 1u);
    __syncthreads();
    s.counts[(int64_t)blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
    if (s.first) clear_bounds(s.bounds, s.a.rows);
}

// Moves a tile's keys to their places in the digit's order.
__global__ void __launch_bounds__(kSortThreads) embed_sort_move_kernel(const SortArgs s) {
    __shared__ SortShared sh;
    pdl_wait();
    uint32_t key[kSortItems], pos[kSortItems], rank[kSortItems];
    bool have[kSortItems];
    load_tile(s, blockIdx.x, key, pos, have);
    rank_tile(sh, key, have, s.shift, rank);
    warps_before(sh);
    uint32_t all = 0, mine = 0;
    for (int64_t t = 0; t < s.tiles; ++t) {
        const uint32_t c = s.counts[t * kDigits + threadIdx.x];
        if (t < blockIdx.x) mine += c;
        all += c;
    }
    sh.base[threadIdx.x] = digits_before(sh, all) + mine;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortItems; ++r)
        if (have[r]) {
            const uint32_t digit = (key[r] >> s.shift) & (kDigits - 1);
            const uint32_t to = sh.base[digit] + sh.count[warp_id()][digit] + rank[r];
            s.out_key[to] = key[r];
            s.out_pos[to] = pos[r];
        }
}

// One tile: every digit in turn by one CTA; the others clear the bounds.
__global__ void __launch_bounds__(kSortThreads) embed_sort_tile_kernel(const SortArgs s) {
    __shared__ SortShared sh;
    __shared__ uint32_t keys[kTile], places[kTile];
    pdl_wait();
    clear_bounds(s.bounds, s.a.rows);
    if (blockIdx.x != 0) return;
    uint32_t key[kSortItems], pos[kSortItems], rank[kSortItems];
    bool have[kSortItems];
    load_tile(s, 0, key, pos, have);
    for (int d = 0; d < s.digits; ++d) {
        const int shift = d * kDigitBits;
        rank_tile(sh, key, have, shift, rank);
        const uint32_t mine = warps_before(sh);
        sh.base[threadIdx.x] = digits_before(sh, mine);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSortItems; ++r)
            if (have[r]) {
                const uint32_t digit = (key[r] >> shift) & (kDigits - 1);
                const uint32_t to = sh.base[digit] + sh.count[warp_id()][digit] + rank[r];
                keys[to] = key[r];
                places[to] = pos[r];
            }
        __syncthreads();
        const int at = warp_id() * (32 * kSortItems) + lane_id();
#pragma unroll
        for (int r = 0; r < kSortItems; ++r)
            if (have[r]) {
                key[r] = keys[at + r * 32];
                pos[r] = places[at + r * 32];
            }
        __syncthreads();
    }
    const int at = warp_id() * (32 * kSortItems) + lane_id();
#pragma unroll
    for (int r = 0; r < kSortItems; ++r)
        if (have[r]) {
            s.out_key[at + r * 32] = key[r];
            s.out_pos[at + r * 32] = pos[r];
        }
}

// ---- sums ------------------------------------------------------------------------------------------------------------

struct SumArgs {
    EmbedGradArgs a;
    const uint32_t *key, *pos;   // sorted
    uint2 *bounds;               // [rows] first and end of a token's sorted positions
    float *windows;              // [n / kWindow][width] sums of windows of one token
    bool wide;
};

// Adds the gradient rows of sorted positions [from, to) to x, columns col .. col + 7, in order.
template <typename T>
__device__ __forceinline__ void add_rows(const SumArgs &s, uint32_t from, uint32_t to, int64_t col, int left, float (&x)[kCols]) {
    const T *g = reinterpret_cast<const T *>(s.a.grad) + col;
    uint32_t i = from;
    for (; i + 4 <= to; i += 4) {
        float y[4][kCols];
#pragma unroll
        for (int u = 0; u < 4; ++u) load_cols(g + (int64_t)s.pos[i + u] * s.a.stride, left, s.wide, y[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = __fadd_rn(x[j], y[u][j]);
    }
    for (; i < to; ++i) {
        float y[kCols];
        load_cols(g + (int64_t)s.pos[i] * s.a.stride, left, s.wide, y);
#pragma unroll
        for (int j = 0; j < kCols; ++j) x[j] = __fadd_rn(x[j], y[j]);
    }
}

// A warp per window of sorted positions: notes where tokens begin and end, and sums the window if it is one token's.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) embed_window_kernel(const SumArgs s) {
    pdl_wait();
    const int64_t windows = (s.a.n + kWindow - 1) / kWindow;
    const uint32_t n = (uint32_t)s.a.n, rows = (uint32_t)s.a.rows;
    for (int64_t w = (int64_t)blockIdx.x * kRowWarps + warp_id(); w < windows; w += (int64_t)gridDim.x * kRowWarps) {
        const uint32_t from = (uint32_t)w * kWindow;
#pragma unroll
        for (int h = 0; h < kWindow; h += 32) {
            const uint32_t i = from + h + lane_id();
            if (i < n) {
                const uint32_t k = s.key[i];
                if (k < rows) {
                    if (i == 0 || s.key[i - 1] != k) s.bounds[k].x = i;
                    if (i == n - 1 || s.key[i + 1] != k) s.bounds[k].y = i + 1;
                }
            }
        }
        if (from + kWindow > n) continue;
        const uint32_t k = s.key[from];
        if (k >= rows || s.key[from + kWindow - 1] != k) continue;
        for (int64_t col = lane_id() * kCols; col < s.a.width; col += 32 * kCols) {
            const int left = (int)min((int64_t)kCols, s.a.width - col);
            float x[kCols] = {};
            add_rows<T>(s, from, from + kWindow, col, left, x);
            store_cols(s.windows + w * s.a.width + col, left, s.a.width % 4 == 0, x);
        }
    }
}

// Adds window sums [w0, w1) to x.
__device__ __forceinline__ void add_windows(const SumArgs &s, uint32_t w0, uint32_t w1, int64_t col, int left, float (&x)[kCols]) {
    const bool wide = s.a.width % 4 == 0;
    uint32_t w = w0;
    for (; w + 4 <= w1; w += 4) {
        float y[4][kCols];
#pragma unroll
        for (int u = 0; u < 4; ++u) load_cols(s.windows + (int64_t)(w + u) * s.a.width + col, left, wide, y[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = __fadd_rn(x[j], y[u][j]);
    }
    for (; w < w1; ++w) {
        float y[kCols];
        load_cols(s.windows + (int64_t)w * s.a.width + col, left, wide, y);
#pragma unroll
        for (int j = 0; j < kCols; ++j) x[j] = __fadd_rn(x[j], y[j]);
    }
}

// One row, columns from the lane's first on, `step` columns apart.
template <typename T>
__device__ __forceinline__ void sum_row(const SumArgs &s, int64_t v, uint2 b, int64_t col0, int64_t step) {
    T *out = reinterpret_cast<T *>(s.a.dtable) + v * s.a.width;
    // whole windows of this token: [w0, w1); the positions outside them at both ends
    uint32_t w0 = (b.x + kWindow - 1) / kWindow, w1 = b.y / kWindow;
    if (w1 <= w0) w0 = w1 = 0;
    for (int64_t col = col0; col < s.a.width; col += step) {
        const int left = (int)min((int64_t)kCols, s.a.width - col);
        float x[kCols] = {};
        if (w1 > w0) {
            add_rows<T>(s, b.x, w0 * kWindow, col, left, x);
            add_windows(s, w0, w1, col, left, x);
            add_rows<T>(s, w1 * kWindow, b.y, col, left, x);
        } else {
            add_rows<T>(s, b.x, b.y, col, left, x);
        }
#pragma unroll
        for (int j = 0; j < kCols; ++j) x[j] = __fmul_rn(x[j], s.a.scale);
        if (s.a.accumulate) {
            float y[kCols];
            load_cols(out + col, left, s.wide, y);
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = __fadd_rn(y[j], x[j]);
        }
        store_cols(out + col, left, s.wide, x);
    }
}

constexpr uint32_t kHeavy = 8 * kWindow;   // positions from which on a whole CTA adds a row

template <typename T>
__global__ void __launch_bounds__(kRowThreads) embed_rows_kernel(const SumArgs s) {
    __shared__ uint2 s_bounds[kRowWarps];
    pdl_wait();
    const int64_t groups = (s.a.rows + kRowWarps - 1) / kRowWarps;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t v = g * kRowWarps + warp_id();
        const uint2 b = v < s.a.rows ? s.bounds[v] : make_uint2(0, 0);
        const bool heavy = b.y - b.x >= kHeavy;
        if (v < s.a.rows && !heavy && (b.y > b.x || !s.a.accumulate)) sum_row<T>(s, v, b, lane_id() * kCols, 32 * kCols);
        if (__syncthreads_or(heavy)) {
            if (lane_id() == 0) s_bounds[warp_id()] = b;
            __syncthreads();
            for (int r = 0; r < kRowWarps; ++r)
                if (s_bounds[r].y - s_bounds[r].x >= kHeavy)
                    sum_row<T>(s, g * kRowWarps + r, s_bounds[r], (int64_t)threadIdx.x * kCols, kRowThreads * kCols);
            __syncthreads();
        }
    }
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct GradLayout {
    size_t key[2], pos[2], counts, bounds, windows, total;
    int64_t tiles;
};
GradLayout grad_layout(int64_t n, int64_t rows, int64_t width) {
    GradLayout L{};
    size_t off = 0;
    L.tiles = (n + kTile - 1) / kTile;
    for (int i = 0; i < 2; ++i) {
        L.key[i] = off, off = up256(off + (size_t)n * 4);
        L.pos[i] = off, off = up256(off + (size_t)n * 4);
    }
    L.counts = off, off = up256(off + (size_t)L.tiles * kDigits * 4);
    L.bounds = off, off = up256(off + (size_t)rows * sizeof(uint2));
    L.windows = off, off = up256(off + (size_t)(n / kWindow) * width * 4);
    L.total = off ? off : 256;
    return L;
}

template <typename T>
cudaError_t launch_sums(const SumArgs &s, cudaStream_t st) {
    const int64_t sms = sm_count();
    const int64_t windows = (s.a.n + kWindow - 1) / kWindow;
    int64_t grid = (windows + kRowWarps - 1) / kRowWarps;
    if (grid > sms * 8) grid = sms * 8;
    if (grid < 1) grid = 1;
    cudaError_t e = launch_after(embed_window_kernel<T>, dim3((unsigned)grid), dim3(kRowThreads), st, s);
    if (e != cudaSuccess) return e;
    grid = (s.a.rows + kRowWarps - 1) / kRowWarps;
    if (grid > sms * 8) grid = sms * 8;
    return launch_after(embed_rows_kernel<T>, dim3((unsigned)grid), dim3(kRowThreads), st, s);
}

bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }

}  // namespace

size_t embed_grad_workspace(int64_t n, int64_t rows, int64_t width) { return grad_layout(n, rows, width).total; }

cudaError_t launch_embed(const EmbedArgs &a, int dtype, cudaStream_t st) {
    const int64_t groups = (a.width + kCols - 1) / kCols;
    const size_t b = dtype_bytes(dtype);
    const bool wide = aligned(a.table, 16) && aligned(a.out, 16) && (a.width * b) % 16 == 0 && (a.stride * b) % 16 == 0;
    int64_t grid = (a.n * groups + 255) / 256;
    const int64_t most = (int64_t)sm_count() * 16;
    if (grid > most) grid = most;
    if (dtype == 0) return launch_after(embed_kernel<float>, dim3((unsigned)grid), dim3(256), st, a, (int)groups, wide);
    if (dtype == 1) return launch_after(embed_kernel<__nv_bfloat16>, dim3((unsigned)grid), dim3(256), st, a, (int)groups, wide);
    return launch_after(embed_kernel<__half>, dim3((unsigned)grid), dim3(256), st, a, (int)groups, wide);
}

cudaError_t launch_embed_grad(const EmbedGradArgs &a, int dtype, cudaStream_t st) {
    const GradLayout L = grad_layout(a.n, a.rows, a.width);
    char *ws = (char *)a.workspace;
    SortArgs s{};
    s.a = a;
    s.counts = (uint32_t *)(ws + L.counts);
    s.bounds = (uint2 *)(ws + L.bounds);
    s.tiles = L.tiles;
    int bits = 1;
    while (bits < 32 && (a.rows >> bits) != 0) ++bits;      // keys 0 .. rows
    s.digits = (bits + kDigitBits - 1) / kDigitBits;
    int at = 0;      // which of the two orders holds the result
    cudaError_t e;
    if (L.tiles <= 1) {
        s.first = 1;
        s.out_key = (uint32_t *)(ws + L.key[0]);
        s.out_pos = (uint32_t *)(ws + L.pos[0]);
        const int64_t clear = (a.rows + kSortThreads * 4 - 1) / (kSortThreads * 4);
        const int64_t most = sm_count();
        e = launch_after(embed_sort_tile_kernel, dim3((unsigned)(clear < 1 ? 1 : clear > most ? most : clear)), dim3(kSortThreads), st, s);
        if (e != cudaSuccess) return e;
    } else {
        for (int d = 0; d < s.digits; ++d) {
            s.first = d == 0;
            s.shift = d * kDigitBits;
            s.in_key = (const uint32_t *)(ws + L.key[at]);
            s.in_pos = (const uint32_t *)(ws + L.pos[at]);
            if (d > 0) at ^= 1;
            s.out_key = (uint32_t *)(ws + L.key[at]);
            s.out_pos = (uint32_t *)(ws + L.pos[at]);
            e = launch_after(embed_sort_count_kernel, dim3((unsigned)L.tiles), dim3(kSortThreads), st, s);
            if (e != cudaSuccess) return e;
            e = launch_after(embed_sort_move_kernel, dim3((unsigned)L.tiles), dim3(kSortThreads), st, s);
            if (e != cudaSuccess) return e;
        }
    }
    SumArgs u{};
    u.a = a;
    u.key = (const uint32_t *)(ws + L.key[at]);
    u.pos = (const uint32_t *)(ws + L.pos[at]);
    u.bounds = s.bounds;
    u.windows = (float *)(ws + L.windows);
    const size_t b = dtype_bytes(dtype);
    u.wide = aligned(a.grad, 16) && aligned(a.dtable, 16) && (a.width * b) % 16 == 0 && (a.stride * b) % 16 == 0;
    return dtype == 0 ? launch_sums<float>(u, st) : dtype == 1 ? launch_sums<__nv_bfloat16>(u, st) : launch_sums<__half>(u, st);
}

}  // namespace guard
