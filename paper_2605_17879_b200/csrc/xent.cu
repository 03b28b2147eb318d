// Softmax cross entropy of a vocabulary product, and its gradients, without keeping the logits.
//
//   z = x w^T;  lse_n = log sum_v exp z_nv;  loss_n = lse_n - z_n,target(n)
//   G_nv = g_n (exp(z_nv - lse_n) - [v = target(n)]);  dx = G w;  dw = G^T x
//
// All four products run on the tensor cores in one kernel frame (product_kernel): pairs of CTAs take tiles of 256 x 256, each
// CTA loads its half of either operand by TMA, one thread issues tcgen05.mma into the TMEM of both, and eight warps a CTA
// read the finished accumulator while the next one is filled.  Single CTAs with tiles of 128 x 256 load half as much again
// per product and were bound by that (4 096 x 1 024 x 65 536 forward 565 us a pass, 512 with pairs, before later steps).  What
// differs is the last step on an accumulator: the logits' largest value and sum of exponentials per row (the forward pass), G
// in 16 bits (the backward pass computes the logits again, a piece of the vocabulary at a time), or a gradient.
//
// Bound: the tensor cores, 2 N V D operations per product, but for few rows, where reading w once is what takes the time.
// The forward product of 4 096 x 1 024 x 65 536 alone takes 328 us, 1 677 TFLOP/s (tensor cores busy 89 % of the cycles); pass
// after pass 414 to 434 us, since the power limit lowers the clock, as it does for all large sizes (8 192 x 4 096 x 131 072
// with gradients, four products: 28 to 30 ms, 1 170 to 1 250 TFLOP/s).  The reading warps share the shared-memory pipe with
// the operands, so what they do to memory counts: an array that the compiler put there, and rows of results stored 16 bytes a
// lane instead of by TMA, cost 70 us.
//
// Rounding: G is held in the inputs' type, since the tensor cores take both operands in one type; each value is off by at
// most half a step (relative), as independent of its neighbours as the outputs' own rounding.  It is held relative to the
// largest finite |g_n|: where all rows weigh the same, as in a mean, the large value of a row, exp(z - lse) - 1 at its target,
// then rounds from near -1 and not from -g_n, whose rounding error all rows would share.  In float16 it is scaled by 2^15
// on top, or exp(z - lse) would lie among the subnormals; below 2^-39 it is lost.  Sums are float32, in passes of 1 024 (see
// LONG).  Against float64 dx and dw are off by 1.7e-3 (bfloat16) and 2.1e-4 (float16) of their norm from their own rounding;
// G's adds up to 2 % to that under a vocabulary of 32 001, 5 to 15 % under 1 000 and 20 to 25 % under 100.
//
// Rows that are ignored take no part: where there are any, the others are gathered first, and whatever the ignored ones
// hold (NaN among it) reaches nothing.
#include <cudaTypedefs.h>

#include <atomic>
#include <type_traits>

#include "tcgen05.cuh"
#include "train_ops.h"

namespace guard {

namespace {

constexpr int kM = 256, kN = 256, kK = 64;    // a tile: rows, columns, depth of a stage
constexpr int kHalf = 128;                    // rows of either operand that each CTA of the pair holds
constexpr int kStages = 6;
constexpr int kOperand = kHalf * kK * 2;      // bytes
constexpr int kStage = 2 * kOperand;
constexpr int kPass = 1024 / kK;              // stages that one accumulator takes
constexpr int kEpilogueWarps = 8;
constexpr int kProductThreads = 32 * (4 + kEpilogueWarps);
constexpr int kBox = 32 * 128;                // bytes of what a warp stores at a time: 32 rows of 64 values
constexpr int kProductSmem = kStages * kStage + kEpilogueWarps * kBox + 1024;
constexpr float kLog2e = 1.4426950408889634f;

enum Mode { kStats, kGrad, kBack };      // kBack: dx and dw in one launch

struct Header {         // at the start of the workspace, written by xent_rows_kernel
    int32_t count;      // rows that take part
    int32_t whole;      // they are all rows: x is read where it is
    float unit, scale;  // G holds g / unit * scale
    float inverse;      // what a gradient from G is multiplied by: unit / scale
};

struct Maps { CUtensorMap a, a2, b, b2, b3, out, out2; };   // of the operands and results (see where each is used)

struct ProductArgs {
    const Header *head;    // or NULL: all rows
    int rows;              // N
    int64_t vocab, width;
    int m_tiles, n_tiles, k_blocks;   // kStats, kGrad: of the logits; kBack: of dx (m_tiles 0: not wanted)
    int group;             // row tiles that share column tiles while those are in the second-level cache
    int dw_tiles, dw_group;           // row tiles of dw (0: not wanted)
    int64_t v0;            // first vocabulary entry of the piece
    const int32_t *target; // [rows] vocabulary index or -1, by (gathered) row
    const void *raw_target;   // without a header: int32 or int64 as the caller gave them
    int target_bits;
    const float *lse, *grad;  // [rows], by gathered row: log sums and row gradients
    float2 *parts;         // [rows][n_parts] largest value and sum
    int n_parts;
    float *picked;         // [rows] logit of the target
    void *dx;              // where gathered rows are scattered
    int64_t dx_stride;
    const int32_t *row_of; // gathered row -> row
    float4 *partial;       // or NULL: partial sums of dx by tile and split, as threads hold them (see partial_at)
    int max_units, max_splits;        // places in it, and splits that the depth allows
    int add;               // add to partial
    long long wait_limit;  // cycles, or 0
    uint32_t *status;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// What exponents are taken relative to: the largest value, or 0 where that is infinite.
__device__ __forceinline__ float finite_or_zero(float m) { return fabsf(m) == INFINITY ? 0.0f : m; }

struct alignas(8) ProductShared {
    uint64_t full[kStages], empty[kStages], done[2], free_[2], drain;
    uint32_t tmem;
    uint32_t abort;        // a wait ran out in this CTA; in either of the pair, once they have met
    uint32_t issued[2];    // in the first CTA: stages that each CTA of the pair has issued copies for
};

// Bounded wait; false when the time ran out here or in another warp.  POLL: with a test's short limit (a waiting instruction
// may sleep beyond it); an instance of its own, since a limit that is looked up costs the forward pass 2 %.
template <bool POLL>
__device__ __forceinline__ bool wait_for(ProductShared &s, uint64_t *bar, uint32_t parity, long long limit) {
    const long long t0 = clock64();
    while (!(POLL ? mbar_test_wait(bar, parity) : mbar_try_wait(bar, parity))) {
        if (*(volatile uint32_t *)&s.abort) return false;
        if (clock64() - t0 > (POLL ? limit : kWaitLimitCycles)) {
            *(volatile uint32_t *)&s.abort = 1;
            return false;
        }
    }
    return true;
}
// What a wait that ran out leaves in flight, once nobody of the pair issues any more: copies into the memory of either CTA,
// counted on the first one's barriers, and products.  Waits for them, a second at most.
__device__ __forceinline__ void land_copies(ProductShared &s) {      // one thread of the first CTA
    const long long t0 = clock64();
    const uint32_t armed = s.issued[0], other = s.issued[1], most = max(armed, other);
    for (uint32_t i = most > kStages ? most - kStages : 0; i < most; ++i) {
        uint64_t *bar = &s.full[i % kStages];
        // a barrier is armed by the first CTA, for the bytes of both
        if (i >= armed) mbar_arrive_expect_tx(bar, kStage);
        else if (i >= other) mbar_complete_tx(bar, kStage);
        while (!mbar_try_wait(bar, (i / kStages) & 1) && clock64() - t0 < kWaitLimitCycles) {}
    }
}
__device__ __forceinline__ void land_products(ProductShared &s) {
    const long long t0 = clock64();
    while (!mbar_try_wait(&s.drain, 0) && clock64() - t0 < kWaitLimitCycles) {}
}

// Parts into which the depth of dx is split: as many as keep every pair of CTAs busy and have a place.
__device__ __forceinline__ int dx_splits(int tiles, int max_units, int max_splits) { return tiles > 0 ? max(1, min(max_units / tiles, max_splits)) : 1; }

// One accumulation: a tile and the stages of depth that it takes.
struct Unit {
    bool dw;
    int m, n, k0, k1;
    int64_t place;         // of its partial sum
};

// The units of one pair of CTAs, in order; every warp that has a part in them goes through the same ones.
struct Work {
    int pairs, pair, m_tiles, n_tiles, k_blocks, group, splits, units;
    int dw_m, dw_group, dw_k, dw_units, early, early_each, rest;     // kBack
    int i, phase;

    template <int MODE>
    __device__ __forceinline__ void begin(const ProductArgs &a, int rows) {
        pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;
        n_tiles = a.n_tiles, k_blocks = a.k_blocks, group = a.group;
        m_tiles = MODE == kBack && a.m_tiles == 0 ? 0 : (rows + kM - 1) / kM;
        splits = MODE == kBack && a.partial ? dx_splits(m_tiles * n_tiles, a.max_units, a.max_splits) : 1;
        units = m_tiles * n_tiles * splits;
        dw_units = 0;
        i = phase = 0;
        if constexpr (MODE == kBack) {
            dw_m = a.dw_tiles, dw_group = a.dw_group;
            dw_k = (rows + kK - 1) / kK;
            dw_units = dw_m * n_tiles;
            // units of dx are few and long: pairs that got one less than others take tiles of dw for it first
            rest = units % pairs;
            early_each = rest ? k_blocks / splits / max(dw_k, 1) : 0;
            early = (int)min((int64_t)dw_units, (int64_t)(pairs - rest) * early_each);
        }
    }
    // The t-th tile: groups of row tiles, column tile after column tile within a group.
    static __device__ __forceinline__ void tile(int t, int m_tiles, int n_tiles, int group, int &m, int &n) {
        const int per = group * n_tiles;
        const int g = t / per, first = g * group;
        const int high = min(group, m_tiles - first), in = t - g * per;
        m = first + in % high;
        n = in / high;
    }
    template <int MODE>
    __device__ __forceinline__ bool next(Unit &u) {
        if (phase == 0) {
            const int t = pair + i * pairs;
            if (t < units) {
                ++i;
                const int split = t % splits;
                u.dw = false;
                tile(t / splits, m_tiles, n_tiles, group, u.m, u.n);
                u.k0 = (int)((int64_t)k_blocks * split / splits);
                u.k1 = (int)((int64_t)k_blocks * (split + 1) / splits);
                u.place = ((int64_t)u.m * n_tiles + u.n) * splits + split;
                return true;
            }
            phase = 1, i = 0;
        }
        if constexpr (MODE == kBack) {
            int t = -1;
            if (phase == 1) {
                t = pair - rest + i * (pairs - rest);
                if (pair < rest || i >= early_each || t >= early) phase = 2, i = 0;
            }
            if (phase == 2) t = early + pair + i * pairs;
            if (t >= dw_units) return false;
            ++i;
            u.dw = true;
            tile(t, dw_m, n_tiles, dw_group, u.m, u.n);
            u.k0 = 0, u.k1 = dw_k;
            return true;
        }
        return false;
    }
};

template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// N values of a thread's row to 16-bit memory, those before `left` (a multiple of eight).
template <typename T, int N>
__device__ __forceinline__ void store_row(T *p, int left, const float (&x)[N]) {
#pragma unroll
    for (int q = 0; q < N / 8; ++q)
        if (8 * q < left)
            reinterpret_cast<uint4 *>(p)[q] = make_uint4(pack2<T>(x[8 * q], x[8 * q + 1]), pack2<T>(x[8 * q + 2], x[8 * q + 3]),
                                                         pack2<T>(x[8 * q + 4], x[8 * q + 5]), pack2<T>(x[8 * q + 6], x[8 * q + 7]));
}
// N values of a thread's row to the h-th place for so many in the warp's box in shared memory (32 rows of 128 bytes, swizzled
// as TMA wants).
template <typename T, int N>
__device__ __forceinline__ void box_row(uint8_t *box, int h, const float (&x)[N]) {
    const int row = lane_id();
#pragma unroll
    for (int q = 0; q < N / 8; ++q)
        *reinterpret_cast<uint4 *>(box + row * 128 + (((h * (N / 8) + q) ^ (row & 7)) << 4)) =
            make_uint4(pack2<T>(x[8 * q], x[8 * q + 1]), pack2<T>(x[8 * q + 2], x[8 * q + 3]), pack2<T>(x[8 * q + 4], x[8 * q + 5]),
                       pack2<T>(x[8 * q + 6], x[8 * q + 7]));
}

// Partial sums of dx lie as the threads hold them: per tile and split 16 warps (rank, half, quarter), per warp 32 groups of
// four columns, per group the 32 rows: every access of a warp is 512 bytes in a row.
constexpr int64_t kPartialTile = (int64_t)kM * kN / 4;    // float4 of a tile
__device__ __forceinline__ int64_t partial_at(int64_t unit, int rank, int half, int quarter, int group, int lane) {
    return unit * kPartialTile + ((((rank * 2 + half) * 4 + quarter) * 32 + group) << 5) + lane;
}

// What a thread of the forward pass knows of its row: largest value so far, and the sum of exponentials relative to it.
struct RowSum {
    float top, sum;
    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N]) {
        float most = top;
#pragma unroll
        for (int j = 0; j < N; ++j) most = fmaxf(most, z[j]);
        const float base = finite_or_zero(most);
        const float shift = -__fmul_rn(base, kLog2e);
        if (sum != 0.0f) sum = __fmul_rn(sum, exp2_fast(__fmul_rn(__fsub_rn(finite_or_zero(top), base), kLog2e)));
        float part[4] = {};
#pragma unroll
        for (int j = 0; j < N; ++j) part[j & 3] = __fadd_rn(part[j & 3], exp2_fast(__fmaf_rn(z[j], kLog2e, shift)));
        sum = __fadd_rn(sum, __fadd_rn(__fadd_rn(part[0], part[1]), __fadd_rn(part[2], part[3])));
        top = most;
    }
};
// y where j == at, else z; kept in registers (an indexed array would go to memory, tile by tile).
__device__ __forceinline__ float pick(int j, int at, float y, float z) {
    asm("{\n\t.reg .pred p;\n\tsetp.eq.s32 p, %1, %2;\n\tselp.f32 %0, %3, %0, p;\n\t}" : "+f"(z) : "r"(j), "r"(at), "f"(y));
    return z;
}

// LONG: the depth takes more than one pass.  The tensor cores cut off what an accumulator's last bit cannot hold, product
// step by product step, which shrinks a sum of one sign by some 1.5 x 2^-24 of itself per 16 of depth; so every product starts
// a new accumulator every kPass stages and adds them in registers, rounded to nearest.  Logits: the losses of 4 096 deep ones
// are off by 3.4e-7 of themselves so, as those of 1 024 deep ones are, and by over 1e-6 without.  The backward pass takes the
// same steps, so that its logits are the forward pass's to the last bit: where a target has all the probability, G is
// exp(z - lse) - 1 = 0 only if lse was made of this z.  Gradients, as deep as there are rows or vocabulary entries: dw of
// 2^21 rows is off by 1.3 % without, by 7e-6 with it (and its rounding).  Passes four and sixteen times as long save up to 1 %
// of the time and lose 2.5e-5 and 1e-4.
template <int MODE, bool LONG, bool POLL, typename T>
__global__ void __launch_bounds__(kProductThreads, 1) __cluster_dims__(2, 1, 1)
product_kernel(const __grid_constant__ Maps maps, const __grid_constant__ ProductArgs a) {
    extern __shared__ uint8_t raw[];
    __shared__ ProductShared s;
    uint8_t *tiles = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const int warp = warp_id(), lane = lane_id();
    const uint32_t rank = cluster_rank();
    pdl_wait();

    const int rows = a.head ? a.head->count : a.rows;
    const bool whole = a.head ? a.head->whole != 0 : true;
    Work work;
    work.begin<MODE>(a, rows);
    const int pass = LONG ? kPass : INT32_MAX / 2;      // stages an accumulator takes

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&s.full[i], 1);
            mbar_init(&s.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.done[i], 1);
            mbar_init(&s.free_[i], 2 * kEpilogueWarps);
        }
        mbar_init(&s.drain, 1);
        s.abort = 0;
        s.issued[0] = s.issued[1] = 0;
    }
    if (warp == 2) tmem_alloc(&s.tmem, 512);
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem = s.tmem;

    if (warp == 0 && lane == 0) {
        // ---- loads: this CTA's half of the rows of either operand
        // (x is read where it is when every row takes part, else from the gathered copy)
        uint32_t it = 0;
        bool ok = true;
        Unit u;
        while (ok && work.next<MODE>(u)) {
            const CUtensorMap *pa, *pb;
            if constexpr (MODE == kBack) {
                pa = u.dw ? &maps.a2 : &maps.a;                                   // G, by either of its sides
                pb = u.dw ? (whole ? &maps.b2 : &maps.b3) : &maps.b;              // x or w
            } else {
                pa = whole ? &maps.a : &maps.a2;                                  // x
                pb = &maps.b;                                                     // w
            }
            const int m0 = u.m * kM + rank * kHalf, n0 = u.n * kN + rank * kHalf;
            for (int k = u.k0; k < u.k1; ++k, ++it) {
                const int st = it % kStages;
                if (!(ok = wait_for<POLL>(s, &s.empty[st], ((it / kStages) & 1) ^ 1, a.wait_limit))) break;
                uint8_t *sa = tiles + st * kStage, *sb = sa + kOperand;
                const uint32_t full = in_first(&s.full[st]);
                if (rank == 0) mbar_arrive_expect_tx(&s.full[st], 2 * kStage);      // of both CTAs
                if (MODE == kBack && u.dw) {          // A: G, tokens by vocabulary; the vocabulary (rows of dw) is contiguous
                    for (int h = 0; h < kHalf / 64; ++h) tma_load(sa + h * 8192, pa, m0 + h * 64, k * kK, full);
                } else {
                    tma_load(sa, pa, k * kK, m0, full);
                }
                if (MODE != kBack) {
                    tma_load(sb, pb, k * kK, (int)a.v0 + n0, full);
                } else {                    // B: w or x, whose columns (of the result) are contiguous
                    const int y = u.dw ? k * kK : (int)a.v0 + k * kK;
                    for (int h = 0; h < kHalf / 64; ++h) tma_load(sb + h * 8192, pb, n0 + h * 64, y, full);
                }
            }
        }
        store_in_pair(&s.issued[rank], 0, it);
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---- products
        constexpr uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
        // operand rows: contiguous (1) or strided, by operand; bits 15 and 16 of the instruction's descriptor
        constexpr uint32_t common = (1u << 4) | (type << 7) | (type << 10) | ((kN / 8) << 17) | ((kM / 16) << 24) | (MODE == kBack ? 1u << 16 : 0u);
        uint32_t it = 0, nth = 0;
        bool ok = true;
        Unit u;
        while (ok && work.next<MODE>(u)) {
            const int k0 = u.k0, k1 = u.k1;
            const bool dw = MODE == kBack && u.dw;
            const uint32_t idesc = common | (dw ? 1u << 15 : 0u);
            // 16 deeper: 16 elements on in a row of 128 bytes, or, where the operand's rows are contiguous, 16 such rows on
            const uint32_t a_step = dw ? 2048 : 32, b_step = MODE == kBack ? 2048 : 32;
            for (int p0 = k0; ok; p0 += pass, ++nth) {          // (once even where there is no depth)
                const uint32_t acc = nth & 1;
                const int p1 = min(k1, LONG ? p0 + pass : k1);
                if (!(ok = wait_for<POLL>(s, &s.free_[acc], ((nth >> 1) & 1) ^ 1, a.wait_limit))) break;
                tc_fence_after();
                for (int k = p0; k < p1; ++k, ++it) {
                    const int st = it % kStages;
                    if (!(ok = wait_for<POLL>(s, &s.full[st], (it / kStages) & 1, a.wait_limit))) break;
                    tc_fence_after();
                    const uint8_t *sa = tiles + st * kStage, *sb = sa + kOperand;
#pragma unroll
                    for (int j = 0; j < kK / 16; ++j) {
                        const uint64_t da = smem_desc(sa + j * a_step, 8192, 1024), db = smem_desc(sb + j * b_step, 8192, 1024);
                        tc_mma(tmem + acc * kN, da, db, idesc, k > p0 || j > 0);
                    }
                    tc_commit(&s.empty[st]);
                }
                if (!ok) break;
                tc_commit(&s.done[acc]);
                if (p1 >= k1) {
                    ++nth;
                    break;
                }
            }
        }
    } else if (warp >= 4) {
        // ---- what becomes of an accumulator: a thread has a row, and half of its columns
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t mine = tmem + ((uint32_t)(quarter * 32) << 16) + half * 128;
        uint8_t *box = tiles + kStages * kStage + (warp - 4) * kBox;
        const float inverse = a.head ? a.head->inverse : 1.0f, unit = a.head ? a.head->unit : 1.0f, scale = a.head ? a.head->scale : 1.0f;
        const uint32_t free0 = in_first(&s.free_[0]), free1 = in_first(&s.free_[1]);
        uint32_t nth = 0;
        Unit u;
        while (work.next<MODE>(u)) {
            const int row = u.m * kM + rank * kHalf + quarter * 32 + lane;
            const bool empty = u.k0 == u.k1;       // no depth at all: the accumulator was not written
            int64_t target = -1;
            float lse = 0.0f, lse2 = 0.0f, g = 0.0f;
            if (MODE == kStats || MODE == kGrad) {
                if (row < rows) {
                    if (a.target) target = a.target[row];
                    else target = a.target_bits == 64 ? reinterpret_cast<const long long *>(a.raw_target)[row] : reinterpret_cast<const int *>(a.raw_target)[row];
                    if (MODE == kGrad) {
                        lse = a.lse[row];
                        lse2 = __fmul_rn(lse, kLog2e);
                        g = __fmul_rn(__fdiv_rn(a.grad[row], unit), scale);
                    }
                }
            }
            float held[LONG ? 128 : 1];
            bool ok = true;
            if constexpr (LONG) {     // all passes but the last are added up in registers
                if (MODE == kBack) {  // (there may be none)
#pragma unroll
                    for (int j = 0; j < 128; ++j) held[j] = 0.0f;
                }
                for (int p = u.k0; p + kPass < u.k1; p += kPass, ++nth) {
                    const uint32_t acc = nth & 1;
                    ok = __all_sync(0xFFFFFFFFu, wait_for<POLL>(s, &s.done[acc], (nth >> 1) & 1, a.wait_limit));   // (the warp stays together)
                    if (!ok) break;
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint32_t r[16];
                        tmem_load16(mine + acc * kN + c * 16, r);
                        tmem_load_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) held[c * 16 + j] = MODE != kBack && p == 0 ? __uint_as_float(r[j]) : __fadd_rn(held[c * 16 + j], __uint_as_float(r[j]));
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_at(acc ? free1 : free0);
                }
                if (!ok) break;
            }
            const uint32_t acc = nth & 1;
            if (!__all_sync(0xFFFFFFFFu, wait_for<POLL>(s, &s.done[acc], (nth >> 1) & 1, a.wait_limit))) break;
            ++nth;
            tc_fence_after();
            const uint32_t from = mine + acc * kN, freed = acc ? free1 : free0;
            const int64_t col0 = (int64_t)u.n * kN + half * 128;
            if constexpr (MODE == kStats) {
                RowSum sums{-INFINITY, 0.0f};
                constexpr int N = LONG ? 16 : 32;
                constexpr int kUnroll = LONG ? 128 / N : 1;
                const int64_t left = a.vocab - col0;                     // columns that are there
                const int at = (int)max((int64_t)-1, min((int64_t)128, target - col0));
#pragma unroll kUnroll
                for (int c = 0; c < 128 / N; ++c) {
                    uint32_t r[N];
                    float z[N];
                    if constexpr (LONG) tmem_load16(from + c * N, r);
                    else tmem_load32(from + c * N, r);
                    tmem_load_wait();
                    if (c == 128 / N - 1) {         // the accumulator is free once every warp has read its part
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_at(freed);
                    }
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        z[j] = __uint_as_float(r[j]);
                        if constexpr (LONG) z[j] = __fadd_rn(held[c * N + j], z[j]);
                    }
                    if (left < (c + 1) * N) {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (c * N + j >= left) z[j] = -INFINITY;
                    }
                    const bool here = at >= c * N && at < (c + 1) * N;
                    if (__any_sync(0xFFFFFFFFu, here)) {
                        float y = 0.0f;
#pragma unroll
                        for (int j = 0; j < N; ++j) y = pick(c * N + j, at, z[j], y);
                        if (here) a.picked[row] = y;
                    }
                    sums.add(z);
                }
                if (row < rows) a.parts[(int64_t)row * a.n_parts + u.n * 2 + half] = make_float2(sums.top, sums.sum);
            } else {
                const bool dw = MODE == kBack && u.dw, dx = MODE == kBack && !u.dw, partly = dx && a.partial;
                // (dx of gathered rows goes to the rows they come from; everything else is stored box by box)
                const bool boxes = !partly && (!dx || whole);
                const int64_t most = MODE == kGrad ? INT64_MAX : dx ? rows : a.vocab - a.v0;      // rows that are there
                const int64_t left = MODE == kGrad ? a.vocab - a.v0 - col0 : a.width - col0;     // columns that are there
                const int at = (int)max((int64_t)-1, min((int64_t)128, target - a.v0 - col0));
                constexpr int N = LONG ? 16 : 32, kSteps = 128 / N, kBoxSteps = 64 / N;
                constexpr int kUnroll = LONG ? kSteps : 1;
#pragma unroll kUnroll
                for (int c = 0; c < kSteps; ++c) {
                    uint32_t r[N];
                    float x[N];
                    if constexpr (LONG) tmem_load16(from + c * N, r);
                    else tmem_load32(from + c * N, r);
                    tmem_load_wait();
                    if (c == kSteps - 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_at(freed);
                    }
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        x[j] = __uint_as_float(r[j]);
                        if constexpr (LONG) x[j] = __fadd_rn(held[c * N + j], x[j]);
                        if (MODE == kBack && empty) x[j] = 0.0f;
                    }
                    if constexpr (MODE == kGrad) {
                        const bool here = at >= c * N && at < (c + 1) * N;
                        float y = 0.0f;                                  // the target's logit
                        if (__any_sync(0xFFFFFFFFu, here)) {
#pragma unroll
                            for (int j = 0; j < N; ++j) y = pick(c * N + j, at, x[j], y);
                        }
#pragma unroll
                        for (int j = 0; j < N; ++j) x[j] = __fmul_rn(exp2_fast(__fmaf_rn(x[j], kLog2e, -lse2)), g);
                        if (__any_sync(0xFFFFFFFFu, here)) {             // the target: less one, which may leave little
                            y = __fmul_rn(expm1f(__fsub_rn(y, lse)), g);
#pragma unroll
                            for (int j = 0; j < N; ++j) x[j] = pick(c * N + j, at, y, x[j]);
                        }
                        // (G has whole tiles: its padding is written as zeros)
                        if (left < (c + 1) * N || row >= rows) {
#pragma unroll
                            for (int j = 0; j < N; ++j)
                                if (c * N + j >= left || row >= rows) x[j] = 0.0f;
                        }
                    } else if (partly) {
#pragma unroll
                        for (int q = 0; q < N / 4; ++q) {
                            float4 *p = a.partial + partial_at(u.place, rank, half, quarter, c * (N / 4) + q, lane);
                            float4 y = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
                            if (a.add) {
                                const float4 z = *p;
                                y = make_float4(__fadd_rn(z.x, y.x), __fadd_rn(z.y, y.y), __fadd_rn(z.z, y.z), __fadd_rn(z.w, y.w));
                            }
                            *p = y;
                        }
                        continue;
                    } else {
#pragma unroll
                        for (int j = 0; j < N; ++j) x[j] = __fmul_rn(x[j], inverse);
                    }
                    if (boxes) {
                        if (c % kBoxSteps == 0) {    // the box's memory, once the last store has read it
                            if (lane == 0) tma_store_wait_read();
                            __syncwarp();
                        }
                        box_row<T>(box, c % kBoxSteps, x);
                        if (c % kBoxSteps == kBoxSteps - 1) {
                            const int c0 = (c - kBoxSteps + 1) * N;      // the box's first column
                            fence_to_tma();
                            __syncwarp();
                            // (row: of lane 0, the box's first; a box that starts outside the result is not stored)
                            if (lane == 0 && (MODE == kGrad || c0 < left) && row < most) {
                                tma_store(dw ? &maps.out2 : &maps.out, box, (int)(col0 + c0), (int)(dw ? a.v0 + row : row));
                                tma_store_commit();
                            }
                        }
                    } else if (row < rows) {
                        store_row(reinterpret_cast<T *>(a.dx) + (int64_t)a.row_of[row] * a.dx_stride + col0 + c * N, (int)min((int64_t)N, left - c * N), x);
                    }
                }
            }
        }
        if (MODE != kStats && lane == 0) tma_store_wait();
    }
    tc_fence_before();
    if (*(volatile uint32_t *)&s.abort) store_in_pair(&s.abort, rank ^ 1, 1);      // (whoever set it comes here after that)
    __syncwarp();
    cluster_sync();              // the pair's memory and barriers are used by both until here
    tc_fence_after();
    if (s.abort) {
        if (warp == 0 && lane == 0 && rank == 0) land_copies(s);
        if (warp == 1 && lane == 0) {
            if (rank == 0) tc_commit(&s.drain);      // (of this thread's products)
            land_products(s);
        }
        if (threadIdx.x == 0 && a.status) atomicOr(a.status, kStatTimeout);
        __syncwarp();
        cluster_sync();
        tc_fence_after();
    }
    if (warp == 2) tmem_free(tmem, 512);
}

// ---- rows that take part ----------------------------------------------------------------------------------------------

struct RowsArgs {
    const void *targets;
    int bits;
    int rows;
    int64_t vocab, ignore;
    Header *head;
    int32_t *target;       // [padded] by gathered row
    int32_t *row_of;       // [padded] gathered row -> row
    int32_t *place;        // [rows] row -> gathered row, or -1
    const float *lse, *grad;   // backward: by row
    int64_t grad_stride;       // 0: one value for all rows
    float *lse_to, *grad_to;   // by gathered row
    bool grads, half;      // backward; float16
    float *loss, *lse_out; // forward: by row, written for those that take no part
    uint32_t *status;
};

__device__ __forceinline__ int64_t target_at(const void *t, int bits, int64_t i) {
    return bits == 64 ? reinterpret_cast<const long long *>(t)[i] : (int64_t) reinterpret_cast<const int *>(t)[i];
}

struct GatherArgs {
    const Header *head;
    const int32_t *place;
    int rows;
    const void *x;
    int64_t stride;
    int vectors;           // 16-byte vectors of a row
    void *to;              // [padded][vectors]
    void *dx;              // or NULL: rows that take no part become zero
};

// A warp copies a row that takes part to its place, or clears its gradient.
__device__ __forceinline__ void gather_row(const GatherArgs &a, int64_t r, int at) {
    const uint4 *from = reinterpret_cast<const uint4 *>((const char *)a.x + r * a.stride * 2);
    uint4 *to = at >= 0 ? reinterpret_cast<uint4 *>(a.to) + (int64_t)at * a.vectors : a.dx ? reinterpret_cast<uint4 *>(a.dx) + r * a.vectors : nullptr;
    if (!to) return;
#pragma unroll 4
    for (int v = lane_id(); v < a.vectors; v += 32) to[v] = at >= 0 ? from[v] : make_uint4(0, 0, 0, 0);
}
// Rows of the gathered copy behind the last one, up to a whole tile: zeros.
__device__ __forceinline__ void pad_rows(const GatherArgs &a, int count, int warp, int warps) {
    const int padded = (count + kM - 1) / kM * kM;
    for (int64_t p = count + warp; p < padded; p += warps)
        for (int v = lane_id(); v < a.vectors; v += 32) reinterpret_cast<uint4 *>(a.to)[p * a.vectors + v] = make_uint4(0, 0, 0, 0);
}

// Finds the rows that take part: a CTA walks over all rows in order, eight a thread at a time.  GATHER (up to kWalk rows):
// every CTA of the grid does so for itself and gathers a slice of the rows, which saves a launch; the first one writes what
// the products read.
constexpr int kEach = 8, kWalk = 1024 * kEach, kSlice = 256;
template <bool GATHER>
__global__ void __launch_bounds__(1024) xent_rows_kernel(const RowsArgs a, const GatherArgs ga, int slice) {
    __shared__ int s_count[32];
    __shared__ float s_top[32];
    __shared__ int s_place[kSlice];
    pdl_wait();
    const int lane = lane_id(), warp = warp_id();
    const bool writes = blockIdx.x == 0;
    const int64_t slice0 = (int64_t)blockIdx.x * slice;
    int before = 0;
    float top = 0.0f;
    for (int64_t base = 0; base < a.rows; base += kWalk) {
        const int64_t first = base + threadIdx.x * kEach;
        int64_t t[kEach];
        float g[kEach];
        uint32_t in = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            t[j] = first + j < a.rows ? target_at(a.targets, a.bits, first + j) : a.ignore;
            g[j] = writes && a.grads && first + j < a.rows ? a.grad[(first + j) * a.grad_stride] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const bool bad = t[j] != a.ignore && (t[j] < 0 || t[j] >= a.vocab);
            if (t[j] != a.ignore && !bad) {
                in |= 1u << j;
                if (fabsf(g[j]) < INFINITY) top = fmaxf(top, fabsf(g[j]));      // (others spoil their own rows alone)
            } else if (writes && first + j < a.rows) {
                if (bad && a.status) atomicOr(a.status, kStatIndex);
                if (a.loss) {
                    a.loss[first + j] = bad ? __uint_as_float(0x7FC00000u) : 0.0f;
                    a.lse_out[first + j] = 0.0f;
                }
            }
        }
        const int mine = __popc(in);
        int upto = mine;
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= d) upto += y;
        }
        if (lane == 31) s_count[warp] = upto;
        __syncthreads();
        const int other = s_count[lane];
        const int all = __reduce_add_sync(0xFFFFFFFFu, other);
        int at = before + upto - mine + __reduce_add_sync(0xFFFFFFFFu, lane < warp ? other : 0);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (first + j >= a.rows) continue;
            const bool takes = (in >> j) & 1;
            if (takes && writes) {
                a.target[at] = (int32_t)t[j];
                a.row_of[at] = (int32_t)(first + j);
                if (a.grads) {
                    a.lse_to[at] = a.lse[first + j];
                    a.grad_to[at] = g[j];
                }
            }
            if (GATHER) {
                if (first + j >= slice0 && first + j < slice0 + slice) s_place[first + j - slice0] = takes ? at : -1;
            } else {
                a.place[first + j] = takes ? at : -1;
            }
            at += takes;
        }
        before += all;
        __syncthreads();
    }
    if (GATHER && before != a.rows) {
        for (int64_t r = warp; r < slice && slice0 + r < a.rows; r += 32) gather_row(ga, slice0 + r, s_place[r]);
        pad_rows(ga, before, blockIdx.x * 32 + warp, gridDim.x * 32);
    }
    if (!writes) return;
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 0; w < 32; ++w) top = fmaxf(top, s_top[w]);
        const bool plain = !(top >= 1e-30f);     // (the products could leave float32's range)
        a.head->count = before;
        a.head->whole = before == a.rows;
        a.head->unit = plain ? 1.0f : top;
        a.head->scale = a.half && !plain ? 32768.0f : 1.0f;
        a.head->inverse = __fdiv_rn(a.head->unit, a.head->scale);
    }
}

// Gathers the rows that take part, where the walk has not done so; a warp per row.
__global__ void __launch_bounds__(256) xent_gather_kernel(const GatherArgs a) {
    pdl_wait();
    if (a.head->whole) return;
    const int warp = blockIdx.x * 8 + warp_id(), warps = gridDim.x * 8;
    for (int64_t r = warp; r < a.rows; r += warps) gather_row(a, r, a.place[r]);
    pad_rows(a, a.head->count, warp, warps);
}

struct CombineArgs {
    const Header *head;    // or NULL: all rows, targets as the caller gave them
    int rows;
    const void *targets;
    int bits;
    int64_t vocab, ignore;
    const int32_t *row_of;
    const float2 *parts;
    int n_parts;
    const float *picked;
    float *loss, *lse;
    uint32_t *status;
};

// A warp per row joins its partial results.
__global__ void __launch_bounds__(256) xent_combine_kernel(const CombineArgs a) {
    pdl_wait();
    const int rows = a.head ? a.head->count : a.rows;
    for (int64_t r = (int64_t)blockIdx.x * 8 + warp_id(); r < rows; r += (int64_t)gridDim.x * 8) {
        const int64_t to = a.head ? a.row_of[r] : r;
        if (!a.head) {
            const int64_t t = target_at(a.targets, a.bits, r);
            const bool bad = t != a.ignore && (t < 0 || t >= a.vocab);
            if (t == a.ignore || bad) {
                if (lane_id() == 0) {
                    if (bad && a.status) atomicOr(a.status, kStatIndex);
                    a.loss[to] = bad ? __uint_as_float(0x7FC00000u) : 0.0f;
                    a.lse[to] = 0.0f;
                }
                continue;
            }
        }
        const float2 *p = a.parts + r * a.n_parts;
        float top = -INFINITY, sum = 0.0f;
        for (int i = lane_id(); i < a.n_parts; i += 128) {
            float2 q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) q[k] = i + 32 * k < a.n_parts ? p[i + 32 * k] : make_float2(-INFINITY, 0.0f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float most = fmaxf(top, q[k].x), base = finite_or_zero(most);
                // (nothing summed yet, or an empty part: its exponent says nothing)
                const float x = sum != 0.0f ? __fmul_rn(sum, exp2_fast(__fmul_rn(__fsub_rn(finite_or_zero(top), base), kLog2e))) : 0.0f;
                const float y = q[k].y != 0.0f ? __fmul_rn(q[k].y, exp2_fast(__fmul_rn(__fsub_rn(finite_or_zero(q[k].x), base), kLog2e))) : 0.0f;
                sum = __fadd_rn(x, y);
                top = most;
            }
        }
        for (int d = 16; d > 0; d >>= 1) {
            const float t2 = __shfl_xor_sync(0xFFFFFFFFu, top, d), s2 = __shfl_xor_sync(0xFFFFFFFFu, sum, d);
            const float most = fmaxf(top, t2), base = finite_or_zero(most);
            const float x = sum != 0.0f ? __fmul_rn(sum, exp2_fast(__fmul_rn(__fsub_rn(finite_or_zero(top), base), kLog2e))) : 0.0f;
            const float y = s2 != 0.0f ? __fmul_rn(s2, exp2_fast(__fmul_rn(__fsub_rn(finite_or_zero(t2), base), kLog2e))) : 0.0f;
            sum = __fadd_rn(x, y);
            top = most;
        }
        if (lane_id() == 0) {
            const float lse = __fadd_rn(finite_or_zero(top), logf(sum));
            a.loss[to] = __fsub_rn(lse, a.picked[r]);
            a.lse[to] = lse;
        }
    }
}

struct JoinArgs {
    const Header *head;
    const int32_t *row_of;
    int64_t width;
    const float4 *partial;
    int n_tiles, max_units, max_splits;
    void *dx;
};

// dx from its partial sums, in order: a warp takes eight columns of 32 rows, in the products' layout.
template <typename T>
__global__ void __launch_bounds__(256) xent_join_kernel(const JoinArgs a) {
    pdl_wait();
    const int rows = a.head->count;
    const int tiles = (rows + kM - 1) / kM * a.n_tiles, splits = dx_splits(tiles, a.max_units, a.max_splits);
    const int64_t work = (int64_t)tiles * 256;       // (16 warps of a tile, 16 pairs of groups)
    const float inverse = a.head->inverse;
    const bool whole = a.head->whole != 0;
    for (int64_t i = (int64_t)blockIdx.x * 8 + warp_id(); i < work; i += (int64_t)gridDim.x * 8) {
        const int64_t tile = i >> 8;
        const int part = (int)(i >> 4) & 15, pair = (int)i & 15;
        const int rank = part >> 3, half = (part >> 2) & 1, quarter = part & 3;
        const int64_t row = tile / a.n_tiles * kM + rank * kHalf + quarter * 32 + lane_id();
        const int64_t col = tile % a.n_tiles * kN + half * 128 + pair * 8;
        if (col >= a.width) continue;
        float x[8] = {};
#pragma unroll 4
        for (int k = 0; k < splits; ++k) {
            const float4 *p = a.partial + partial_at(tile * splits + k, rank, half, quarter, pair * 2, lane_id());
            const float4 u = p[0], v = p[32];
            const float y[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __fadd_rn(x[j], y[j]);
        }
        if (row >= rows) continue;
        *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.dx) + (whole ? row : a.row_of[row]) * a.width + col) =
            make_uint4(pack2<T>(__fmul_rn(x[0], inverse), __fmul_rn(x[1], inverse)), pack2<T>(__fmul_rn(x[2], inverse), __fmul_rn(x[3], inverse)),
                       pack2<T>(__fmul_rn(x[4], inverse), __fmul_rn(x[5], inverse)), pack2<T>(__fmul_rn(x[6], inverse), __fmul_rn(x[7], inverse)));
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Allows a kernel its shared memory, once per device.
struct SmemAttribute {
    std::atomic<uint64_t> done{0};
    cudaError_t set(const void *kernel, int bytes) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = dev < 64 ? 1ull << dev : 0;
        if (bit & done.load(std::memory_order_relaxed)) return cudaSuccess;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
        return e;
    }
};

PFN_cuTensorMapEncodeTiled encoder() {
    static PFN_cuTensorMapEncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return (PFN_cuTensorMapEncodeTiled)p;
    }();
    return fn;
}

// A row-major matrix of 16-bit elements in boxes of 64 columns (128 bytes, swizzled) by `box` rows; outside it reads zeros.
bool make_map(CUtensorMap *map, bool bf16, const void *p, int64_t width, int64_t rows, int64_t stride, int box) {
    const PFN_cuTensorMapEncodeTiled encode = encoder();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)(rows < 1 ? 1 : rows)};
    const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)box};
    const cuuint32_t steps[2] = {1, 1};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(p), dims, strides, boxes, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kDirectRows = kHalf;     // up to here the forward pass takes the rows as they are: there is no tile to save

struct XentLayout {
    size_t head, target, row_of, place, lse, grad, picked, parts, x, g, partial, total;
    int64_t padded, piece;
    int n_parts, max_units, max_splits;     // max_units 0: dx is written directly
};

// What G of one piece of the vocabulary may take, unless the narrowest piece, a tile of 256 entries, takes more: 512 bytes a
// row, which is more from 2^20 rows on (2^26 rows, the most there may be: 34 GB).  More pieces cost more passes over dx's
// partial sums (0.3 GB a piece for 8 192 x 4 096, some 50 us beside 7 ms of products); this is a quarter of the 16-bit logits
// of 8 192 rows and 131 072 entries.
constexpr int64_t kPieceBytes = 512ll << 20;

XentLayout layout(int64_t rows, int64_t width, int64_t vocab, bool grads) {
    XentLayout L{};
    L.padded = (rows + kM - 1) / kM * kM;
    const int64_t n_tiles = (vocab + kN - 1) / kN;
    size_t off = 0;
    auto take = [&](size_t &at, size_t bytes) { at = off, off = up256(off + bytes); };
    take(L.head, sizeof(Header));
    take(L.target, L.padded * 4);
    take(L.row_of, L.padded * 4);
    take(L.place, rows * 4);
    take(L.x, grads || rows > kDirectRows ? L.padded * width * 2 : 0);
    if (!grads) {
        L.n_parts = (int)(n_tiles * 2);
        take(L.picked, L.padded * 4);
        take(L.parts, (size_t)L.padded * L.n_parts * sizeof(float2));
    } else {
        take(L.lse, L.padded * 4);
        take(L.grad, L.padded * 4);
        int64_t piece = kPieceBytes / (L.padded * 2) / kN * kN;
        if (piece < kN) piece = kN;
        const int64_t pieces = (n_tiles * kN + piece - 1) / piece;
        piece = ((n_tiles + pieces - 1) / pieces) * kN;
        L.piece = piece;
        take(L.g, (size_t)L.padded * piece * 2);
        const int64_t tiles = L.padded / kM * ((width + kN - 1) / kN);
        const int64_t pairs = sm_count() / 2;
        L.max_splits = (int)(piece / kK / 4 > 1 ? piece / kK / 4 : 1);
        const bool split = tiles * 2 <= pairs && L.max_splits > 1;
        L.max_units = (int)(!split && pieces == 1 ? 0 : tiles > pairs ? tiles : pairs);
        take(L.partial, (size_t)(L.max_units * kPartialTile) * sizeof(float4));
    }
    L.total = off;
    return L;
}

template <int MODE, bool LONG, bool POLL, typename T>
cudaError_t launch_product_as(const Maps &maps, const ProductArgs &a, int64_t units, cudaStream_t st) {
    static SmemAttribute wide;
    const cudaError_t e = wide.set((const void *)product_kernel<MODE, LONG, POLL, T>, kProductSmem);
    if (e != cudaSuccess) return e;
    const int64_t pairs = sm_count() / 2;
    return launch_after_smem(product_kernel<MODE, LONG, POLL, T>, dim3((unsigned)(2 * (units < pairs ? units : pairs))), dim3(kProductThreads), kProductSmem, st, maps, a);
}
template <int MODE, typename T>
cudaError_t launch_product(const Maps &maps, const ProductArgs &a, int64_t units, cudaStream_t st) {
    const int dw_k = MODE == kBack && a.dw_tiles > 0 ? (a.rows + kK - 1) / kK : 0;
    const bool deep = a.k_blocks > kPass || dw_k > kPass;
    if (a.wait_limit > 0) return deep ? launch_product_as<MODE, true, true, T>(maps, a, units, st) : launch_product_as<MODE, false, true, T>(maps, a, units, st);
    return deep ? launch_product_as<MODE, true, false, T>(maps, a, units, st) : launch_product_as<MODE, false, false, T>(maps, a, units, st);
}

// Row tiles that share a column tile: as many as fit in about a third of the second-level cache.
int group_of(int64_t depth_bytes, int m_tiles) {
    int64_t g = (40ll << 20) / (depth_bytes * kM);
    if (g < 8) g = 8;
    return (int)(g < m_tiles ? g : m_tiles);
}

cudaError_t launch_rows(const XentArgs &x, const XentLayout &L, bool grads, cudaStream_t st) {
    char *ws = (char *)x.workspace;
    RowsArgs r{};
    r.targets = x.targets;
    r.bits = x.target_bits;
    r.rows = (int)x.rows;
    r.vocab = x.vocab;
    r.ignore = x.ignore;
    r.head = (Header *)(ws + L.head);
    r.target = (int32_t *)(ws + L.target);
    r.row_of = (int32_t *)(ws + L.row_of);
    r.place = (int32_t *)(ws + L.place);
    r.status = x.status;
    if (grads) {
        r.lse = x.lse;
        r.grad = x.grad_loss;
        r.grad_stride = x.grad_stride;
        r.lse_to = (float *)(ws + L.lse);
        r.grad_to = (float *)(ws + L.grad);
        r.grads = true;
        r.half = x.dtype == 2;
    } else {
        r.loss = x.loss;
        r.lse_out = x.lse_out;
    }
    GatherArgs g{};
    g.head = r.head;
    g.place = r.place;
    g.rows = r.rows;
    g.x = x.x;
    g.stride = x.x_stride;
    g.vectors = (int)(x.width / 8);
    g.to = ws + L.x;
    g.dx = grads ? x.dx : nullptr;
    const int64_t sms = sm_count();
    if (x.rows <= kWalk) {
        int64_t grid = (x.rows + 7) / 8;
        if (grid > sms) grid = sms;
        const int64_t slice = (x.rows + grid - 1) / grid;
        if (slice <= kSlice) return launch_after(xent_rows_kernel<true>, dim3((unsigned)grid), dim3(1024), st, r, g, (int)slice);
    }
    const cudaError_t e = launch_after(xent_rows_kernel<false>, dim3(1), dim3(1024), st, r, g, 0);
    if (e != cudaSuccess) return e;
    int64_t grid = (x.rows + 7) / 8;
    if (grid > sms * 8) grid = sms * 8;
    return launch_after(xent_gather_kernel, dim3((unsigned)grid), dim3(256), st, g);
}

template <typename T>
cudaError_t forward(const XentArgs &x, cudaStream_t st) {
    const XentLayout L = layout(x.rows, x.width, x.vocab, false);
    char *ws = (char *)x.workspace;
    const bool direct = x.rows <= kDirectRows, bf16 = x.dtype == 1;
    cudaError_t e;
    Maps maps{};
    if (!make_map(&maps.a, bf16, x.x, x.width, x.rows, x.x_stride, kHalf) || !make_map(&maps.b, bf16, x.w, x.width, x.vocab, x.w_stride, kHalf)) return cudaErrorInvalidValue;
    maps.a2 = maps.a;
    if (!direct) {
        if (!make_map(&maps.a2, bf16, ws + L.x, x.width, L.padded, x.width, kHalf)) return cudaErrorInvalidValue;
        e = launch_rows(x, L, false, st);
        if (e != cudaSuccess) return e;
    }
    ProductArgs a{};
    a.head = direct ? nullptr : (const Header *)(ws + L.head);
    a.rows = (int)x.rows;
    a.vocab = x.vocab;
    a.width = x.width;
    a.m_tiles = (int)(L.padded / kM);
    a.n_tiles = (int)((x.vocab + kN - 1) / kN);
    a.k_blocks = (int)((x.width + kK - 1) / kK);
    a.group = group_of(x.width * 2, a.m_tiles);
    a.target = direct ? nullptr : (const int32_t *)(ws + L.target);
    a.raw_target = x.targets;
    a.target_bits = x.target_bits;
    a.parts = (float2 *)(ws + L.parts);
    a.n_parts = L.n_parts;
    a.picked = (float *)(ws + L.picked);
    a.status = x.status;
    a.wait_limit = x.wait_limit;
    e = launch_product<kStats, T>(maps, a, (int64_t)a.m_tiles * a.n_tiles, st);
    if (e != cudaSuccess) return e;
    CombineArgs c{};
    c.head = a.head;
    c.rows = (int)x.rows;
    c.targets = x.targets;
    c.bits = x.target_bits;
    c.vocab = x.vocab;
    c.ignore = x.ignore;
    c.row_of = (const int32_t *)(ws + L.row_of);
    c.parts = a.parts;
    c.n_parts = a.n_parts;
    c.picked = a.picked;
    c.loss = x.loss;
    c.lse = x.lse_out;
    c.status = x.status;
    int64_t grid = (x.rows + 7) / 8;
    if (grid > sm_count() * 8) grid = sm_count() * 8;
    return launch_after(xent_combine_kernel, dim3((unsigned)grid), dim3(256), st, c);
}

template <typename T>
cudaError_t backward(const XentArgs &x, cudaStream_t st) {
    const XentLayout L = layout(x.rows, x.width, x.vocab, true);
    char *ws = (char *)x.workspace;
    const bool bf16 = x.dtype == 1;
    cudaError_t e = launch_rows(x, L, true, st);
    if (e != cudaSuccess) return e;
    Maps logits{}, back{};
    // logits: x, gathered x, w, G.  back: G by its rows (the depth of dx is the vocabulary) and by its columns (the rows of
    // dw), w and x with the result's columns contiguous, dx, dw
    if (!make_map(&logits.a, bf16, x.x, x.width, x.rows, x.x_stride, kHalf) || !make_map(&logits.a2, bf16, ws + L.x, x.width, L.padded, x.width, kHalf) ||
        !make_map(&logits.b, bf16, x.w, x.width, x.vocab, x.w_stride, kHalf) || !make_map(&logits.out, bf16, ws + L.g, L.piece, L.padded, L.piece, 32) ||
        !make_map(&back.a, bf16, ws + L.g, L.piece, L.padded, L.piece, kHalf) || !make_map(&back.a2, bf16, ws + L.g, L.piece, L.padded, L.piece, kK) ||
        !make_map(&back.b, bf16, x.w, x.width, x.vocab, x.w_stride, kK) || !make_map(&back.b2, bf16, x.x, x.width, x.rows, x.x_stride, kK) ||
        !make_map(&back.b3, bf16, ws + L.x, x.width, L.padded, x.width, kK) || (x.dx && !make_map(&back.out, bf16, x.dx, x.width, x.rows, x.width, 32)) ||
        (x.dw && !make_map(&back.out2, bf16, x.dw, x.width, x.vocab, x.width, 32)))
        return cudaErrorInvalidValue;
    const int64_t pieces = (x.vocab + L.piece - 1) / L.piece;
    ProductArgs a{};
    a.head = (const Header *)(ws + L.head);
    a.rows = (int)x.rows;
    a.vocab = x.vocab;
    a.width = x.width;
    a.target = (const int32_t *)(ws + L.target);
    a.lse = (const float *)(ws + L.lse);
    a.grad = (const float *)(ws + L.grad);
    a.row_of = (const int32_t *)(ws + L.row_of);
    a.status = x.status;
    a.wait_limit = x.wait_limit;
    const int row_tiles = (int)(L.padded / kM), width_tiles = (int)((x.width + kN - 1) / kN);
    for (int64_t p = 0; p < pieces; ++p) {
        a.v0 = p * L.piece;
        const int64_t here = x.vocab - a.v0 < L.piece ? x.vocab - a.v0 : L.piece;
        ProductArgs g = a;
        g.m_tiles = row_tiles;
        g.n_tiles = (int)((here + kN - 1) / kN);
        g.k_blocks = (int)((x.width + kK - 1) / kK);
        g.group = group_of(x.width * 2, g.m_tiles);
        e = launch_product<kGrad, T>(logits, g, (int64_t)g.m_tiles * g.n_tiles, st);
        if (e != cudaSuccess) return e;
        ProductArgs d = a;
        d.n_tiles = width_tiles;
        d.k_blocks = (int)((here + kK - 1) / kK);
        d.m_tiles = x.dx ? row_tiles : 0;
        d.group = row_tiles < 8 ? row_tiles : 8;
        d.dw_tiles = x.dw ? (int)((here + kM - 1) / kM) : 0;
        d.dw_group = d.dw_tiles < 8 ? d.dw_tiles : 8;
        d.dx = x.dx;
        d.dx_stride = x.width;
        d.partial = L.max_units ? (float4 *)(ws + L.partial) : nullptr;
        d.max_units = L.max_units;
        d.max_splits = L.max_splits;
        d.add = p > 0;
        // (one launch for both: tiles of dw fill the pairs that a last round of dx leaves idle)
        const int64_t dx_units = !x.dx ? 0 : L.max_units ? L.max_units : (int64_t)row_tiles * width_tiles;
        e = launch_product<kBack, T>(back, d, dx_units + (int64_t)d.dw_tiles * width_tiles, st);
        if (e != cudaSuccess) return e;
    }
    if (x.dx && L.max_units) {
        JoinArgs j{};
        j.head = a.head;
        j.row_of = a.row_of;
        j.width = x.width;
        j.partial = (const float4 *)(ws + L.partial);
        j.n_tiles = width_tiles;
        j.max_units = L.max_units;
        j.max_splits = L.max_splits;
        j.dx = x.dx;
        int64_t grid = (int64_t)row_tiles * width_tiles * 32;
        if (grid > sm_count() * 8) grid = sm_count() * 8;
        return launch_after(xent_join_kernel<T>, dim3((unsigned)grid), dim3(256), st, j);
    }
    return cudaSuccess;
}

}  // namespace

size_t xent_workspace(int64_t rows, int64_t width, int64_t vocab, bool grads) { return layout(rows, width, vocab, grads).total; }
cudaError_t launch_xent(const XentArgs &x, cudaStream_t st) { return x.dtype == 1 ? forward<__nv_bfloat16>(x, st) : forward<__half>(x, st); }
cudaError_t launch_xent_grad(const XentArgs &x, cudaStream_t st) { return x.dtype == 1 ? backward<__nv_bfloat16>(x, st) : backward<__half>(x, st); }

}  // namespace guard
