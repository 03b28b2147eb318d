// Token embedding with scaling, and its gradient by sorted tokens.
//
// Lookup: out[i] = scale * table[token[i]].  Pure copying: bound by reading each different row and writing every output row
// (16 384 rows of 2 048 bfloat16: 16.9 us for 93 MB, 5.5 TB/s; 23.5 with a thread per 16 bytes of the output, one load each).
//
// Gradient: dtable[v] = scale * sum of the gradient rows of the positions with token v.  Summing with atomics would make
// the order, and with it the result, a matter of chance, and would serialise on frequent tokens; so the positions are sorted
// by token first (a stable radix sort), and runs of one token are summed.
//   1. embed_sort_*: least significant digit first, kDigitBits at a time; a CTA ranks a tile of keys with warp matches and
//      counters of its own, so equal keys keep their order; two launches per digit.  Short lists: every key's place counted directly.
//   2. embed_sum_kernel: a warp takes a window of 32 sorted positions and a strip of columns, loads eight rows' vectors at a
//      time and adds them run by run.  A run inside the window is a finished row.  One that crosses its borders leaves a
//      partial sum: two places a window, in order, so the partial sums are again a sorted list, a sixteenth as long, to which
//      the same is applied until the list is short; embed_finish_kernel then adds each token's places.  So a token that occurs once costs one read and one write, one that
//      fills the batch is summed by as many warps as there are windows, and nothing depends on how frequent tokens are.
//      The first of these launches also writes zeros to the rows whose token is not in the list (but for those that the SMs
//      which had nothing to sort have cleared).
// The grouping of a sum depends on the positions alone.
// Bound: memory, and above all writing the table (3.9 TB/s at best where it does not fit the second-level cache, as a memset of
// it does: 139 us for 537 MB).  65 536 rows of 2 048 bfloat16 into 131 072: 177 us, of
// which 136 are step 2's first launch (650 MB) and 25 the sort.
#include "train_ops.h"

namespace guard {

namespace {

constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 512;            // one per digit in the scans
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 4;                // keys a thread ranks at a time
constexpr int kTile = kSortThreads * kSortItems;
constexpr int kWindow = 32;
constexpr int kSumThreads = 256;
constexpr int kSumWarps = kSumThreads / 32;
constexpr uint32_t kHole = 0x80000000u;      // a place without a partial sum; its key keeps the list sorted

__device__ __forceinline__ int64_t token_at(const void *tokens, int bits, int64_t i) {
    return bits == 64 ? __ldg(reinterpret_cast<const long long *>(tokens) + i) : (int64_t)__ldg(reinterpret_cast<const int *>(tokens) + i);
}

// ---- lookup ----------------------------------------------------------------------------------------------------------

// A warp takes a token and a strip of its row; where rows are whole vectors of 16 bytes, all of a lane's loads (up to eight)
// are in flight before the first is scaled and stored.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a, int strips) {
    constexpr int V = 16 / sizeof(T), kVectors = 8;
    constexpr int kStrip = WIDE ? 32 * V * kVectors : 256;      // columns
    pdl_wait();
    const int lane = lane_id();
    const int64_t work = a.n * strips, warps = (int64_t)gridDim.x * 8;
    for (int64_t u = (int64_t)blockIdx.x * 8 + warp_id(); u < work; u += warps) {
        int64_t i = u, strip = 0;
        if (strips > 1) {
            i = (u >> 31) ? u / strips : (int64_t)((uint32_t)u / (uint32_t)strips);
            strip = u - i * strips;
        }
        const int64_t tok = token_at(a.tokens, a.token_bits, i);
        const bool good = tok >= 0 && tok < a.rows;
        if (!good && strip == 0 && lane == 0 && a.status) atomicOr(a.status, kStatIndex);
        const T *from = reinterpret_cast<const T *>(a.table) + (good ? tok : 0) * a.stride;
        T *to = reinterpret_cast<T *>(a.out) + i * a.width;
        const float nan = __uint_as_float(0x7FC00000u);
        const int64_t c0 = strip * kStrip + (WIDE ? lane * V : lane);
        if constexpr (WIDE) {
            Bytes16 r[kVectors];
#pragma unroll
            for (int q = 0; q < kVectors; ++q)
                if (good && c0 + q * 32 * V < a.width) r[q] = *reinterpret_cast<const Bytes16 *>(from + c0 + q * 32 * V);
#pragma unroll
            for (int q = 0; q < kVectors; ++q) {
                const int64_t c = c0 + q * 32 * V;
                if (c >= a.width) break;
                T *t = reinterpret_cast<T *>(&r[q]);
#pragma unroll
                for (int j = 0; j < V; ++j) t[j] = Conv<T>::down(good ? __fmul_rn(Conv<T>::up(t[j]), a.scale) : nan);
                store16_once(to + c, r[q]);
            }
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int64_t c = c0 + q * 32;
                if (c < a.width) to[c] = Conv<T>::down(good ? __fmul_rn(Conv<T>::up(from[c]), a.scale) : nan);
            }
        }
    }
}

// ---- sorting positions by token ---------------------------------------------------------------------------------------

struct SortShared {
    alignas(16) uint16_t count[kSortWarps][kDigits];   // keys of a digit per warp, then the number before that warp
    uint32_t base[kDigits];                // where a digit's keys of this tile go
    uint32_t scan[kSortWarps];
};

// A token's key: the token, or `rows` (behind all tokens) where it adds nothing.
__device__ __forceinline__ uint32_t key_of(const EmbedGradArgs &a, int64_t t) {
    if (t < 0 || t >= a.rows) {
        if (a.status) atomicOr(a.status, kStatIndex);
        return (uint32_t)a.rows;
    }
    return t == a.padding ? (uint32_t)a.rows : (uint32_t)t;
}
__device__ __forceinline__ uint32_t key_at(const EmbedGradArgs &a, int64_t i) { return key_of(a, token_at(a.tokens, a.token_bits, i)); }

// Ranks the tile's keys by a digit.  Thread holds kSortItems keys, warp after warp and 32 at a time in order, so that rank
// order is position order.  rank[r]: number of keys of the same digit before this one in the warp; counts per warp in s.count.
__device__ __forceinline__ void rank_tile(SortShared &s, const uint32_t (&key)[kSortItems], const bool (&have)[kSortItems], int shift,
                                          uint32_t (&rank)[kSortItems]) {
    for (int d = threadIdx.x; d < kSortWarps * kDigits / 8; d += kSortThreads) reinterpret_cast<uint4 *>(&s.count[0][0])[d] = make_uint4(0, 0, 0, 0);
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

struct SortArgs {
    EmbedGradArgs a;
    const uint32_t *in_key, *in_pos;   // the previous digit's order (unused for the first digit)
    uint32_t *out_key, *out_pos;
    uint32_t *counts;                  // [tiles][kDigits], then [kDigits] totals
    bool scanned;                      // counts hold the numbers before each tile, totals theirs
    int64_t tiles;
    int shift, digits, first;
    // CTAs behind the sorting ones write zeros meanwhile: a piece of the table's last rows, see launch_embed_grad
    unsigned sorters;
    uint8_t *clear;
    int64_t clear_bytes;
};

// Zero bytes from p on (a whole number of 2-byte units, aligned to one); `threads` threads together, this one the i-th.
__device__ __forceinline__ void clear_by(uint8_t *p, int64_t bytes, int64_t i, int64_t threads) {
    const int64_t head = min(bytes, (int64_t)((16 - ((uintptr_t)p & 15)) & 15));
    const int64_t vectors = (bytes - head) / 16, done = head + vectors * 16;
    uint16_t *ends = reinterpret_cast<uint16_t *>(p);
    uint4 *mid = reinterpret_cast<uint4 *>(p + head);
    for (int64_t k = i; k < vectors; k += threads) mid[k] = make_uint4(0, 0, 0, 0);
    for (int64_t k = i; k * 2 < head; k += threads) ends[k] = 0;
    for (int64_t k = done / 2 + i; k * 2 < bytes; k += threads) ends[k] = 0;
}
__device__ __forceinline__ bool clears(const SortArgs &s) {
    if (blockIdx.x < s.sorters) return false;
    clear_by(s.clear, s.clear_bytes, (int64_t)(blockIdx.x - s.sorters) * blockDim.x + threadIdx.x, (int64_t)(gridDim.x - s.sorters) * blockDim.x);
    return true;
}

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
    if (clears(s)) return;
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
}

// Many tiles: turns the counts into the numbers before each tile, 32 digits a CTA, a part of the tiles a warp.
__global__ void __launch_bounds__(1024) embed_sort_scan_kernel(uint32_t *counts, int64_t tiles) {
    __shared__ uint32_t part[32][32];
    pdl_wait();
    const int lane = lane_id(), warp = warp_id();
    const int64_t each = (tiles + 31) / 32, begin = min(tiles, warp * each), end = min(tiles, begin + each);
    uint32_t *c = counts + blockIdx.x * 32 + lane;
    uint32_t sum = 0;
#pragma unroll 8
    for (int64_t t = begin; t < end; ++t) sum += c[t * kDigits];
    part[warp][lane] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < warp; ++w) before += part[w][lane];
    for (int64_t t = begin; t < end; ++t) {
        const uint32_t x = c[t * kDigits];
        c[t * kDigits] = before;
        before += x;
    }
    if (warp == 31) c[tiles * kDigits] = before;
}

// Moves a tile's keys to their places in the digit's order.
__global__ void __launch_bounds__(kSortThreads) embed_sort_move_kernel(const SortArgs s) {
    __shared__ SortShared sh;
    pdl_wait();
    if (clears(s)) return;
    uint32_t key[kSortItems], pos[kSortItems], rank[kSortItems];
    bool have[kSortItems];
    load_tile(s, blockIdx.x, key, pos, have);
    uint32_t all = 0, mine = 0;
    if (s.scanned) {
        mine = s.counts[(int64_t)blockIdx.x * kDigits + threadIdx.x];
        all = s.counts[s.tiles * kDigits + threadIdx.x];
    } else {
#pragma unroll 8
        for (int64_t t = 0; t < s.tiles; ++t) {
            const uint32_t c = s.counts[t * kDigits + threadIdx.x];
            if (t < blockIdx.x) mine += c;
            all += c;
        }
    }
    rank_tile(sh, key, have, s.shift, rank);
    warps_before(sh);
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

// Short lists: a key's place is the number of keys that come before it, and counting them all is quick: a CTA holds the list
// in shared memory and counts for 64 of its keys, four a warp, 128 comparisons with each at a time.  5 003 keys: 12 us, where
// one CTA took 18 for the digits in turn.
constexpr int kShort = 8192, kRankThreads = 512, kRankEach = 64;
__global__ void __launch_bounds__(kRankThreads) embed_sort_short_kernel(const SortArgs s) {
    __shared__ alignas(16) uint32_t keys[kShort];
    pdl_wait();
    if (clears(s)) return;
    const int n = (int)s.a.n, blocks = (n + 127) / 128, lane = lane_id();
    for (int j0 = threadIdx.x; j0 < blocks * 128; j0 += kRankThreads * 8) {
        int64_t t[8];                    // (all on their way before the first is looked at)
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = j0 + k * kRankThreads < n ? token_at(s.a.tokens, s.a.token_bits, j0 + k * kRankThreads) : 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int j = j0 + k * kRankThreads;
            if (j < blocks * 128) keys[j] = j < n ? key_of(s.a, t[k]) : 0xFFFFFFFFu;
        }
    }
    __syncthreads();
    constexpr int kMine = kRankEach / (kRankThreads / 32);
    const int i0 = blockIdx.x * kRankEach + warp_id() * kMine;
    if (i0 >= n) return;
    uint32_t key[kMine], count[kMine] = {};
#pragma unroll
    for (int m = 0; m < kMine; ++m) key[m] = keys[min(i0 + m, n - 1)];
    for (int b = 0; b < blocks; ++b) {
        const uint4 k = reinterpret_cast<const uint4 *>(keys)[b * 32 + lane];
        const uint32_t other[4] = {k.x, k.y, k.z, k.w};
        // before: smaller, or equal and further ahead in the list
        if (b * 128 + 128 <= i0) {
#pragma unroll
            for (int m = 0; m < kMine; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) count[m] += other[e] <= key[m];
        } else if (b * 128 >= i0 + kMine) {
#pragma unroll
            for (int m = 0; m < kMine; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) count[m] += other[e] < key[m];
        } else {
#pragma unroll
            for (int m = 0; m < kMine; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) count[m] += other[e] < key[m] || (other[e] == key[m] && b * 128 + lane * 4 + e < i0 + m);
        }
    }
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        const uint32_t to = __reduce_add_sync(0xFFFFFFFFu, count[m]);
        if (lane == 0 && i0 + m < n) {
            s.out_key[to] = key[m];
            s.out_pos[to] = (uint32_t)(i0 + m);
        }
    }
}

// ---- sums ------------------------------------------------------------------------------------------------------------

// A sorted list and where its sums go.
struct List {
    int64_t n;
    const uint32_t *key, *pos;   // pos: NULL where rows lie in the list's order
    const void *from;
    int64_t stride;
    uint32_t *next_key;          // or NULL
    float *next;
};

struct SumArgs {
    List list;                   // sorted keys (kHole: nothing there)
    int64_t rows, width, clear_to;   // rows from clear_to on are zero already
    float scale;
    int accumulate;
    void *dtable;
    const uint32_t *all_key;     // the first list, for the CTAs that write zeros to the rows without tokens
    int64_t all_n;
    bool clear_late;             // those are in the last launch, not in the first
    int clear_each;
    unsigned sum_blocks, clear_blocks;
    int strips;
};

// The lane's columns of a strip of 32 * V columns: V consecutive ones (WIDE: one vector of 16 bytes of the rows' type), or
// every 32nd.
template <bool WIDE, int V> __device__ __forceinline__ int64_t column(int64_t strip, int j) {
    return WIDE ? (strip * 32 + lane_id()) * V + j : strip * 32 * V + j * 32 + lane_id();
}
template <typename T, bool WIDE, int V>
__device__ __forceinline__ void load_strip(const T *row, int64_t strip, int64_t width, T (&x)[V]) {
    if constexpr (WIDE) {
        static_assert(sizeof(T) * V == 16, "");
        const int64_t c = column<true, V>(strip, 0);
        if (c < width) *reinterpret_cast<uint4 *>(x) = *reinterpret_cast<const uint4 *>(row + c);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int64_t c = column<false, V>(strip, j);
            if (c < width) x[j] = row[c];
        }
    }
}
template <typename O, bool WIDE, int V>
__device__ __forceinline__ void store_strip(O *row, int64_t strip, int64_t width, const float (&x)[V]) {
    if constexpr (WIDE) {
        const int64_t c = column<true, V>(strip, 0);
        if (c >= width) return;
        O y[V];
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = Conv<O>::down(x[j]);
        constexpr int B = sizeof(O) * V;          // 8, 16 or 32 bytes
        if constexpr (B == 8) *reinterpret_cast<uint2 *>(row + c) = *reinterpret_cast<const uint2 *>(y);
        else
#pragma unroll
            for (int h = 0; h < B / 16; ++h) reinterpret_cast<uint4 *>(row + c)[h] = reinterpret_cast<const uint4 *>(y)[h];
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int64_t c = column<false, V>(strip, j);
            if (c < width) row[c] = Conv<O>::down(x[j]);
        }
    }
}

// First place of the sorted list whose key is not below k; the warp together, 32 probes at a time.
__device__ __forceinline__ int64_t warp_lower_bound(const uint32_t *key, int64_t n, uint32_t k) {
    int64_t lo = 0, hi = n;
    while (hi - lo > 0) {
        const int64_t step = (hi - lo + 31) / 32;
        const int64_t i = lo + (lane_id() + 1) * step - 1;        // the last place of the lane's part
        const bool below = i < hi && key[i] < k;
        const int parts = __popc(__ballot_sync(0xFFFFFFFFu, below));   // parts that lie below k altogether
        lo += parts * step;
        hi = min(hi, lo + step - 1);
        if (step == 1) break;
    }
    return lo;
}

// Zeros for the rows of the table without tokens, clear_each rows a warp (at most 32): the sorted keys say which those are.
template <typename O>
__device__ __forceinline__ void clear_rows(const SumArgs &s, int64_t warp, int64_t warps) {
    O *table = reinterpret_cast<O *>(s.dtable);
    const uint32_t *key = s.all_key;
    const int64_t n = s.all_n;
    for (int64_t first = warp * s.clear_each; first < s.clear_to; first += warps * s.clear_each) {
        const int64_t last = min(first + s.clear_each, s.clear_to);
        int64_t lo = warp_lower_bound(key, n, (uint32_t)first);
        const int64_t end = lo + warp_lower_bound(key + lo, n - lo, (uint32_t)last);
        const int64_t mine = first + lane_id();
        int64_t hi = end;
        while (lo < hi) {                             // the lane's own row among those
            const int64_t mid = (lo + hi) / 2;
            if (key[mid] < (uint32_t)mine) lo = mid + 1;
            else hi = mid;
        }
        const bool empty = mine < last && !(lo < end && key[lo] == (uint32_t)mine);
        uint32_t rows = __ballot_sync(0xFFFFFFFFu, empty);
        while (rows) {                                // runs of them are one stretch of memory each
            const int at = __ffs(rows) - 1;
            const int run = __ffs(~(rows >> at) | (at ? 1u << (32 - at) : 0u)) - 1;      // (ends at row 32)
            const int count = run < 0 ? 32 : run;
            clear_by(reinterpret_cast<uint8_t *>(table + (first + at) * s.width), (int64_t)count * s.width * sizeof(O), lane_id(), 32);
            rows = at + count >= 32 ? 0u : rows & ~((1u << (at + count)) - 1);
        }
    }
}

// A row's sum is complete: scaled, added to what the table holds where that is wanted, and stored.
template <typename O, bool WIDE, int V>
__device__ __forceinline__ void finish_row(const SumArgs &s, uint32_t row, int64_t strip, float (&sum)[V]) {
    O *out = reinterpret_cast<O *>(s.dtable) + (int64_t)row * s.width;
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = __fmul_rn(sum[e], s.scale);
    if (s.accumulate) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int64_t c = column<WIDE, V>(strip, e);
            if (c < s.width) sum[e] = __fadd_rn(Conv<O>::up(out[c]), sum[e]);
        }
    }
    store_strip<O, WIDE, V>(out, strip, s.width, sum);
}

// One warp, one window of the list, one strip of columns.  T: the list's rows (the gradient's type, or float32 for partial
// sums); O: the table's.
template <typename T, typename O, bool WIDE>
__device__ __forceinline__ void sum_window(const SumArgs &s, const List &l, int64_t w, int64_t strip) {
    constexpr int V = 16 / sizeof(T);
    constexpr int kBatch = V == 4 ? 16 : 8;      // rows whose vectors are loaded together
    const int lane = lane_id();
    const int64_t i = w * kWindow + lane;
    const uint32_t raw = i < l.n ? l.key[i] : 0x7FFFFFFFu;
    const uint32_t key = raw & ~kHole;
    const uint32_t pos = l.pos && i < l.n ? l.pos[i] : (uint32_t)i;
    const uint32_t used = __ballot_sync(0xFFFFFFFFu, raw == key && key < (uint32_t)s.rows);
    // the keys around the window: its first and its last run may be parts of longer ones
    const uint32_t before = w > 0 ? l.key[w * kWindow - 1] & ~kHole : 0x7FFFFFFFu;
    const uint32_t after = (w + 1) * kWindow < l.n ? l.key[(w + 1) * kWindow] & ~kHole : 0x7FFFFFFFu;
    const uint32_t next = __shfl_down_sync(0xFFFFFFFFu, key, 1);
    const uint32_t ends = __ballot_sync(0xFFFFFFFFu, lane == 31 || next != key);
    const uint32_t first = __shfl_sync(0xFFFFFFFFu, key, 0), last = __shfl_sync(0xFFFFFFFFu, key, 31);
    const bool enters = first == before, leaves = last == after;
    float sum[V] = {};
    bool any = false, head = true;            // the run holds something; it is the window's first
    bool full0 = false, full1 = false;        // places of the next list that get a partial sum
#pragma unroll 1
    for (int b = 0; b < kWindow; b += kBatch) {
        T x[kBatch][V];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const uint32_t p = __shfl_sync(0xFFFFFFFFu, pos, b + j);
            if ((used >> (b + j)) & 1) load_strip<T, WIDE, V>(reinterpret_cast<const T *>(l.from) + (int64_t)p * l.stride, strip, s.width, x[j]);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if ((used >> (b + j)) & 1) {
                any = true;
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = __fadd_rn(sum[e], Conv<T>::up(x[j][e]));
            }
            if ((ends >> (b + j)) & 1) {
                const bool tail = b + j == 31 && leaves, from_before = head && enters;
                if (any) {
                    if (tail || from_before) {
                        full0 |= from_before;
                        full1 |= !from_before;
                        store_strip<float, WIDE, V>(l.next + (2 * w + (from_before ? 0 : 1)) * s.width, strip, s.width, sum);
                    } else {
                        finish_row<O, WIDE, V>(s, __shfl_sync(0xFFFFFFFFu, key, b + j), strip, sum);
                    }
                }
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = 0.0f;
                any = head = false;
            }
        }
    }
    if (lane < 2 && l.next_key) l.next_key[2 * w + lane] = (lane == 0 ? first : last) | ((lane == 0 ? full0 : full1) ? 0u : kHole);
}

template <typename T, typename O, bool WIDE>
__global__ void __launch_bounds__(kSumThreads, sizeof(T) == 4 ? 2 : 3) embed_sum_kernel(const SumArgs s) {
    pdl_wait();
    // the clearing CTAs lie evenly among the others, so that reading and writing go on side by side
    const int64_t all = gridDim.x, b = blockIdx.x;
    const int64_t cleared = b * s.clear_blocks / all;
    if ((b + 1) * s.clear_blocks / all > cleared) {
        clear_rows<O>(s, cleared * kSumWarps + warp_id(), (int64_t)s.clear_blocks * kSumWarps);
        return;
    }
    const int64_t work = (s.list.n + kWindow - 1) / kWindow * s.strips;
    for (int64_t u = (b - cleared) * kSumWarps + warp_id(); u < work; u += (int64_t)s.sum_blocks * kSumWarps) {
        const int64_t w = u / s.strips, strip = u - w * s.strips;
        List l = s.list;
        if (strip != 0) l.next_key = nullptr;     // (every strip finds the same)
        sum_window<T, O, WIDE>(s, l, w, strip);
    }
}

// The last list of partial sums, a CTA per strip of 128 columns: a warp per token adds its places in order.
constexpr int kFinish = 512, kFinishThreads = 512;
template <typename O, bool WIDE>
__global__ void __launch_bounds__(kFinishThreads) embed_finish_kernel(const SumArgs s) {
    constexpr int V = 4, kBatch = 8;
    __shared__ uint32_t keys[kFinish];
    __shared__ uint16_t runs[kFinish];
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    pdl_wait();
    if (blockIdx.x >= s.strips) {
        constexpr int kWarps = kFinishThreads / 32;
        clear_rows<O>(s, (int64_t)(blockIdx.x - s.strips) * kWarps + warp_id(), (int64_t)(gridDim.x - s.strips) * kWarps);
        return;
    }
    const int n = (int)s.list.n, i = threadIdx.x;
    keys[i] = i < n ? s.list.key[i] : 0xFFFFFFFFu;
    __syncthreads();
    // a token's first place that holds something (in any order: every token is added by itself)
    const uint32_t key = keys[i];
    if (!(key & kHole) && key < (uint32_t)s.rows) {
        int j = i - 1;
        while (j >= 0 && keys[j] == (key | kHole)) --j;
        if (j < 0 || keys[j] != key) runs[atomicAdd(&count, 1)] = (uint16_t)i;
    }
    __syncthreads();
    const int64_t strip = blockIdx.x;
    const float *from = reinterpret_cast<const float *>(s.list.from);
    for (int r = warp_id(); r < count; r += kFinishThreads / 32) {
        int at = runs[r];
        const uint32_t row = keys[at];
        float sum[V] = {};
        while (at < n && (keys[at] & ~kHole) == row) {
            float x[kBatch][V];
            uint32_t have = 0;
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (at + j < n && keys[at + j] == row) {
                    have |= 1u << j;
                    load_strip<float, WIDE, V>(from + (int64_t)(at + j) * s.list.stride, strip, s.width, x[j]);
                }
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if ((have >> j) & 1) {
#pragma unroll
                    for (int e = 0; e < V; ++e) sum[e] = __fadd_rn(sum[e], x[j][e]);
                }
            at += kBatch;
        }
        finish_row<O, WIDE, V>(s, row, strip, sum);
    }
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct GradLayout {
    size_t key[2], pos[2], counts, next_key[2], next[2], total;
    int64_t tiles;
};
// Places of the list that a list of n leaves (0: none).
inline int64_t next_length(int64_t n) { return n > kWindow ? 2 * ((n + kWindow - 1) / kWindow) : 0; }
GradLayout grad_layout(int64_t n, int64_t rows, int64_t width) {
    GradLayout L{};
    size_t off = 0;
    L.tiles = (n + kTile - 1) / kTile;
    for (int i = 0; i < 2; ++i) {
        L.key[i] = off, off = up256(off + (size_t)n * 4);
        L.pos[i] = off, off = up256(off + (size_t)n * 4);
    }
    L.counts = off, off = up256(off + (size_t)(L.tiles + 1) * kDigits * 4);
    // two lists of partial sums, used in turn
    int64_t m = next_length(n);
    for (int i = 0; i < 2; ++i) {
        L.next_key[i] = off, off = up256(off + (size_t)m * 4);
        L.next[i] = off, off = up256(off + (size_t)m * width * 4);
        m = next_length(m);
    }
    L.total = off ? off : 256;
    return L;
}

template <typename T, typename O>
cudaError_t launch_sum(SumArgs s, bool first, bool wide, cudaStream_t st) {
    const int64_t most = (int64_t)sm_count() * 8;
    constexpr int V = 16 / sizeof(T);
    s.strips = (int)((s.width + 32 * V - 1) / (32 * V));
    const int64_t work = (s.list.n + kWindow - 1) / kWindow * s.strips;
    int64_t blocks = (work + kSumWarps - 1) / kSumWarps;
    if (blocks > most * 16) blocks = most * 16;
    s.sum_blocks = (unsigned)blocks;
    int64_t clear = first && !s.accumulate && !s.clear_late ? (s.clear_to + s.clear_each * kSumWarps - 1) / (s.clear_each * kSumWarps) : 0;
    if (clear > most * 4) clear = most * 4;
    s.clear_blocks = (unsigned)clear;
    if (blocks + clear == 0) return cudaSuccess;
    const dim3 grid((unsigned)(blocks + clear)), block(kSumThreads);
    return wide ? launch_after(embed_sum_kernel<T, O, true>, grid, block, st, s) : launch_after(embed_sum_kernel<T, O, false>, grid, block, st, s);
}

// Sums the sorted list, then the lists of partial sums.
template <typename T>
cudaError_t launch_sums(SumArgs s, const GradLayout &L, char *ws, bool wide, cudaStream_t st) {
    for (int level = 0;; ++level) {
        const int to = level & 1;
        const int64_t next = next_length(s.list.n);
        s.list.next_key = next ? (uint32_t *)(ws + L.next_key[to]) : nullptr;
        s.list.next = next ? (float *)(ws + L.next[to]) : nullptr;
        cudaError_t e;
        if (level > 0 && s.list.n <= kFinish) {
            s.strips = (int)((s.width + 127) / 128);
            int64_t clear = s.clear_late && !s.accumulate ? (s.clear_to * 32 + kFinishThreads * s.clear_each - 1) / (kFinishThreads * s.clear_each) : 0;
            if (clear > sm_count() * 4) clear = sm_count() * 4;
            const dim3 grid((unsigned)(s.strips + clear)), block(kFinishThreads);
            return wide ? launch_after(embed_finish_kernel<T, true>, grid, block, st, s) : launch_after(embed_finish_kernel<T, false>, grid, block, st, s);
        }
        e = level == 0 ? launch_sum<T, T>(s, true, wide, st) : launch_sum<float, T>(s, false, wide, st);
        if (e != cudaSuccess || !next) return e;
        s.list = List{next, s.list.next_key, nullptr, s.list.next, s.width, nullptr, nullptr};
    }
}

// Bytes that are cleared beside the sort of up to kFew keys, of a short list, and in each launch of longer sorts.
constexpr int kFew = 1024;
constexpr int64_t kTinyClear = 16 << 20, kShortClear = 64 << 20, kLaunchClear = 20 << 20;

bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }

}  // namespace

size_t embed_grad_workspace(int64_t n, int64_t rows, int64_t width) { return grad_layout(n, rows, width).total; }

template <typename T>
static cudaError_t launch_embed_as(const EmbedArgs &a, cudaStream_t st) {
    const size_t b = sizeof(T);
    const bool wide = aligned(a.table, 16) && aligned(a.out, 16) && (a.width * b) % 16 == 0 && (a.stride * b) % 16 == 0;
    const int64_t strip = wide ? 32 * 16 / b * 8 : 256;
    const int64_t strips = (a.width + strip - 1) / strip;
    int64_t grid = (a.n * strips + 7) / 8;
    const int64_t most = (int64_t)sm_count() * 32;
    if (grid > most) grid = most;
    return wide ? launch_after(embed_kernel<T, true>, dim3((unsigned)grid), dim3(256), st, a, (int)strips)
                : launch_after(embed_kernel<T, false>, dim3((unsigned)grid), dim3(256), st, a, (int)strips);
}
cudaError_t launch_embed(const EmbedArgs &a, int dtype, cudaStream_t st) {
    return dtype == 0 ? launch_embed_as<float>(a, st) : dtype == 1 ? launch_embed_as<__nv_bfloat16>(a, st) : launch_embed_as<__half>(a, st);
}

cudaError_t launch_embed_grad(const EmbedGradArgs &a, int dtype, cudaStream_t st) {
    const GradLayout L = grad_layout(a.n, a.rows, a.width);
    char *ws = (char *)a.workspace;
    SortArgs s{};
    s.a = a;
    s.counts = (uint32_t *)(ws + L.counts);
    s.tiles = L.tiles;
    int bits = 1;
    while (bits < 32 && (a.rows >> bits) != 0) ++bits;      // keys 0 .. rows
    s.digits = (bits + kDigitBits - 1) / kDigitBits;
    int at = 0;      // which of the two orders holds the result
    cudaError_t e;
    // Writing the table is what bounds the whole (a memset writes 537 MB at 3.9 TB/s; 128 MB, which the second-level cache takes
    // up in part, at 6.2), and sorting does not use memory.  So other CTAs write zeros to the last rows meanwhile; rows whose
    // token occurs are written again later.  What is left is cleared beside the first sums, or, for short lists, whose few reads
    // would wait behind the writes, beside the last ones.  5 003 x 1 001 into 32 001 rows of float32: 45 us (with another sort:
    // 48 so, 52 with the rest beside the first sums, 62 without a head start).  The head start does not pay everywhere; with
    // and without it (us, by tokens): 8 000 x 2 048 bfloat16: 16: 10.2, 8.8; 1 100: 21.3, 24.8; 8 000: 40, 37.
    // 32 001 x 1 001 float32: 16: 22.6, 23.2; 1 100: 43, 40; 8 000: 52, 56; 65 536: 127, 131.  131 072 x 2 048 bfloat16:
    // 1 100: 118, 106; 8 000: 124, 119; 8 200: 132, 137; 65 536: 177, 183.  Bytes in proportion to the tokens (8 KB each) win 10 %
    // in the last table for 1 100 to 3 000 tokens and lose 20 % in the first and 10 % for 5 003 in the second.
    const int64_t sms = sm_count(), row_bytes = a.width * (int64_t)dtype_bytes(dtype);
    const bool is_short = a.n <= kShort;
    const int64_t spare = is_short ? sms : sms - L.tiles, launches = is_short ? 1 : 2 * s.digits;
    int64_t early = 0;                   // rows
    if (!a.accumulate && spare > sms / 4) {
        const int64_t bytes = (!is_short ? kLaunchClear * launches : a.n > kFew ? kShortClear : kTinyClear) * spare / sms;
        early = bytes / row_bytes < a.rows ? bytes / row_bytes : a.rows;
    }
    uint8_t *const early_from = (uint8_t *)a.dtable + (a.rows - early) * row_bytes;
    int64_t given = 0;
    auto share = [&](int64_t launch) {   // of the launch-th: whole rows
        const int64_t to = early * (launch + 1) / launches;
        s.clear = early_from + given * row_bytes;
        s.clear_bytes = (to - given) * row_bytes;
        given = to;
    };
    if (is_short) {
        s.sorters = (unsigned)((a.n + kRankEach - 1) / kRankEach);
        share(0);
        s.out_key = (uint32_t *)(ws + L.key[0]);
        s.out_pos = (uint32_t *)(ws + L.pos[0]);
        const int64_t grid = s.sorters + (early ? sms : 0);
        e = grid ? launch_after(embed_sort_short_kernel, dim3((unsigned)grid), dim3(kRankThreads), st, s) : cudaSuccess;
        if (e != cudaSuccess) return e;
    } else {
        s.sorters = (unsigned)L.tiles;
        const unsigned grid = (unsigned)(L.tiles + (early ? spare : 0));
        for (int d = 0; d < s.digits; ++d) {
            s.first = d == 0;
            s.shift = d * kDigitBits;
            s.in_key = (const uint32_t *)(ws + L.key[at]);
            s.in_pos = (const uint32_t *)(ws + L.pos[at]);
            if (d > 0) at ^= 1;
            s.out_key = (uint32_t *)(ws + L.key[at]);
            s.out_pos = (uint32_t *)(ws + L.pos[at]);
            share(2 * d);
            e = launch_after(embed_sort_count_kernel, dim3(grid), dim3(kSortThreads), st, s);
            if (e != cudaSuccess) return e;
            // (each CTA of the move adds the counts of all tiles up itself where they are few)
            s.scanned = L.tiles > 64;
            if (s.scanned) e = launch_after(embed_sort_scan_kernel, dim3(kDigits / 32), dim3(1024), st, s.counts, L.tiles);
            if (e != cudaSuccess) return e;
            share(2 * d + 1);
            e = launch_after(embed_sort_move_kernel, dim3(grid), dim3(kSortThreads), st, s);
            if (e != cudaSuccess) return e;
        }
    }
    SumArgs u{};
    u.list = List{a.n, (const uint32_t *)(ws + L.key[at]), (const uint32_t *)(ws + L.pos[at]), a.grad, a.stride, nullptr, nullptr};
    u.clear_to = a.rows - early;
    u.all_key = u.list.key;
    u.all_n = a.n;
    u.clear_late = is_short && a.n > kFew;
    u.clear_each = u.clear_to > sms * 16 * 32 ? 32 : 8;      // enough warps to use every SM
    u.rows = a.rows;
    u.width = a.width;
    u.scale = a.scale;
    u.accumulate = a.accumulate;
    u.dtable = a.dtable;
    const size_t b = dtype_bytes(dtype);
    const bool wide = aligned(a.grad, 16) && aligned(a.dtable, 16) && (a.width * b) % 16 == 0 && (a.stride * b) % 16 == 0;
    return dtype == 0   ? launch_sums<float>(u, L, ws, wide, st)
           : dtype == 1 ? launch_sums<__nv_bfloat16>(u, L, ws, wide, st)
                        : launch_sums<__half>(u, L, ws, wide, st);
}

}  // namespace guard
