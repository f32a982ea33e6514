// Attention over a 4-bit cache with many query rows a KV head: tcgen05 (cb_attend).
//
// A block takes up to 256 query rows (token, head of the group) of one KV head over a part of the
// positions, in tiles of 128 positions.  20 warps:
//   0..7    softmax, four a stream (TMEM lane quarter = warp % 4): a thread is a query row
//   8..11   K: four-bit rows from global memory, as bf16 into shared memory (K-major, 128-byte swizzle)
//   12..15  V: the same, transposed, as fp16
//   16      issues tcgen05.mma; 17 finds the next segment, 18 what the join has to (19 fills the warp group)
// Two streams alternate on the tensor core, so that one's softmax runs beside the other's products: with
// more than 128 rows a stream is a half of the rows and both take every tile; with fewer the streams take
// alternate tiles of the same rows, each with its own maximum and sums, and join at the end.
//   S [128 rows][128 positions] = Q K^T            (bf16; fp32 in tensor memory)
//   P = exp2(S - M), fp16, back into tensor memory as the next product's A operand
//   O [128 rows][D] += P V                          (fp16)
// Tensor memory (512 columns): two S of 128, two O of D.  P has 64 columns: its own for D = 64, the lower
// half of S for D = 128, where the next S waits for the product that reads P to end.
// O is scaled in place when a row's maximum has grown by more than 8 (log2 domain) since M was set: seldom
// after the first tiles; until then weights are up to 2^15, in fp16's range.
//
// Measured (32 query heads, 8 KV heads of 128): 1024 tokens over 16384 positions 266 us, 1001 TFLOP/s, 253 of it before
// the join; 64 tokens over 12352 positions 41 us, 34 before it. Bound by the chain of waits of a stream (weights, their
// product, the next scores, its maximum), by fetching the roles' code and by the shared memory that the products read.
// 256 rows a block, because each unpacking of a tile serves all of them.  Other forms, when this one (with a slower
// join) took 286 to 292 us: 128 rows 367; two warps that issue 335; 16 softmax warps of 72 registers 408; registers not
// moved between the roles and 8 + 8 + 1 warps 317; scores in two halves of 64 positions 293 to 299; the products alone,
// without softmax and unpacking, 249.
#include <atomic>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_attend.cuh"
#include "cb_receiver.cuh"
#include "cb_sm100_attend.cuh"

namespace cbk {
namespace {
using namespace sm100;

constexpr int kTile = 128;                  // positions a tile, rows a stream
constexpr int kRowTile = 2 * kTile;         // query rows a block takes at a time
constexpr int kWarpsAt = 20;
constexpr int kThreadsAt = kWarpsAt * 32;
// Registers a thread is launched with, and those of a softmax thread, of one that unpacks and of the last
// four warps.
constexpr int kRegs = 96, kRegsSoftmax = 128, kRegsUnpack = 72, kRegsIssue = 72;
static_assert(256 * kRegsSoftmax + 256 * kRegsUnpack + 128 * kRegsIssue <= kThreadsAt * kRegs, "more registers than at launch");
constexpr int kStages = 2;
constexpr int kJoinBlocks = 32;             // blocks that join one item
constexpr float kBits = 7.f;                // weights are exp2(z - M'), M' = M - 7
constexpr float kGrow = 8.f;                // growth of a row's maximum that M follows
constexpr uint32_t kPollNs = 1000000u;
constexpr uint64_t kDrainNs = 1000000000ull;

struct Ctl {
    uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
    uint64_t s_full[2], p_full[2], pv_done[2], done;
    uint64_t stall;         // failure-detection test: a barrier nothing arrives on
    uint64_t wait_ns;
    uint32_t tmem;
    int abort;
    // the run (registers are for the roles): its next unit, its ends, all units, and what the segments before had
    int unit, run0, run1, segment, tiles, items[2];
};

// Bytes: the control block and the units before each pair, Q of two streams, K and V stages, the packed rows
// on their way, 1 KB of alignment.
constexpr int kCtlBytes = 1024 + (kMaxPairs + 1) * 4;
template <int D>
constexpr int smem_bytes() {
    return 2 * kTile * D * 2 + kStages * 2 * kTile * D * 2 + 8 * (32 * D / 2 + 256) + kCtlBytes + 1024;
}

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Bounded wait: false when it gave up or another role did (bits 8 + tag of the error word name the wait).
// (Inline: a call would have to do with the registers of every role.)
__device__ __forceinline__ bool poll(uint64_t* bar, uint32_t parity, Ctl* c, uint32_t* err, int tag) {
    const uint64_t t0 = now_ns();
    do {
        if (mbar_try_wait_hint(bar, parity, kPollNs)) return true;
        if (*reinterpret_cast<volatile int*>(&c->abort)) return false;
    } while (now_ns() - t0 <= c->wait_ns);
    *reinterpret_cast<volatile int*>(&c->abort) = 1;
    atomicOr(err, kErrTimeout | (1u << (8 + tag)));
    return false;
}
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, Ctl* c, uint32_t* err, int tag) {
    return mbar_try_wait(bar, parity) || poll(bar, parity, c, err, tag);
}
// The same for a whole warp, which stays together whatever its lanes saw.
__device__ __forceinline__ bool wait_warp(uint64_t* bar, uint32_t parity, Ctl* c, uint32_t* err, int tag) {
    return __all_sync(0xFFFFFFFFu, wait(bar, parity, c, err, tag));
}
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity) {
    const uint64_t t0 = now_ns();
    while (!mbar_try_wait(bar, parity))
        if (now_ns() - t0 > kDrainNs) return;
}

__device__ __forceinline__ uint64_t desc(uint32_t lo, uint32_t hi) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
    return d;
}

// A 16-byte piece of a K-major operand with 128-byte rows (64 elements a block): row, piece 0..7 of block.
__device__ __forceinline__ uint32_t piece(int block, int rows, int row, int p) {
    return (uint32_t)(block * rows * 128 + row * 128 + ((p ^ (row & 7)) << 4));
}

__device__ __forceinline__ void st_piece(uint8_t* base, uint32_t at, const uint32_t (&w)[4]) {
    *reinterpret_cast<uint4*>(base + at) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Codes and scales of a tile on their way: each of the eight warps that unpack copies its own share of the
// next tile into shared memory (cp.async) while it unpacks this one.
//   K, warp w: rows 32 w .. 32 w + 31.  Lane: rows 8 y + lane % 8, the quarter lane / 8 of each.
//   V, warp w: rows 64 (w % 2) .., the half w / 2 of each.  Lane: the eight rows 8 (lane % 8) .., of each an
//     eighth of the row (lane / 8 of that half), so that eight neighbouring lanes write eight pieces of one
//     row of V^T.
// Places of the 16-byte pieces keep both reads free of bank conflicts.
template <int D>
struct Share {
    static constexpr int kCodes = 32 * D / 2, kBytes = kCodes + 256;   // (64 rows of V, 4 bytes of scales each)
    static __device__ __forceinline__ uint32_t k_at(int row, int p) {
        return row * (D / 2) + ((p ^ (D == 128 ? (row >> 1) & 3 : (row >> 2) & 1)) << 4);
    }
    static __device__ __forceinline__ uint32_t v_at(int row, int p) {
        return ((row & 7) * 8 + (row >> 3)) * (D / 4) + (D == 128 ? (p ^ (row >> 5)) << 4 : 0);
    }
};

// mine: the row of position t0 + 32 w + lane.
template <int D>
__device__ __forceinline__ void copy_k(uint32_t to, const Segment& x, int mine) {
    constexpr int P = D / 32;                       // pieces a row
    const int lane = threadIdx.x & 31, p = lane % P;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int row = lane / P + i * (32 / P), r = __shfl_sync(0xFFFFFFFFu, mine, row);
        copy16(to + Share<D>::k_at(row, p), x.code[0] + (int64_t)max(r, 0) * (D / 2) + p * 16);
    }
    copy_small<D / 16>(to + Share<D>::kCodes + lane * (D / 16), x.scale[0] + (int64_t)max(mine, 0) * (D / 32), mine >= 0);
    copy_commit();
}
// lo, hi: the rows of positions t0 + 64 (w % 2) + lane and 32 more.
template <int D>
__device__ __forceinline__ void copy_v(uint32_t to, const Segment& x, int lo, int hi, int half) {
    constexpr int P = D / 64;                       // pieces of half a row
    const int lane = threadIdx.x & 31, p = lane % P;
#pragma unroll
    for (int i = 0; i < 2 * P; ++i) {
        const int at = lane / P + (i % P) * (32 / P), row = at + (i / P) * 32;
        const int r = __shfl_sync(0xFFFFFFFFu, i / P ? hi : lo, at);
        copy16(to + Share<D>::v_at(row, p), x.code[1] + (int64_t)max(r, 0) * (D / 2) + half * (D / 4) + p * 16);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {                   // four bytes a row: D = 128 two groups of four, D = 64 both
        const int r = i ? hi : lo;
        copy_small<4>(to + Share<D>::kCodes + (lane + 32 * i) * 4,
                      x.scale[1] + (int64_t)max(r, 0) * (D / 32) + (D == 128 ? half * 2 : 0), r >= 0);
    }
    copy_commit();
}

// A thread's row of one tile: S at ts becomes weights at tp, M and l follow; where M rises by much the sums at
// `to` (if there are any) are scaled.  EDGE: columns [c0, c1) alone are seen; without it no column is looked at.
template <int D, bool EDGE>
__device__ __forceinline__ void softmax_tile(uint32_t ts, uint32_t tp, uint32_t to, bool sums, int c0, int c1, float scale,
                                             float& M, float& l) {
    // 32 columns at a time, first for the maximum, then for the weights, each read from tensor memory when its
    // turn comes.  (Rolled up: the roles share the instruction cache.  With the four steps written out and all
    // columns in registers, read once, 1024 tokens over 16384 positions took 353 us for 292.)
    float z[32];
    float high = -INFINITY;
    auto seen = [&](float (&x)[32], int first) {
        if (EDGE) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
                if (first + k < c0 || first + k >= c1) x[k] = -INFINITY;
        }
    };
#pragma unroll 1
    for (int c = 0; c < kTile; c += 32) {
        tmem_ld32(ts + c, z);
        tmem_wait_ld(z);
        seen(z, c);
        high = fmaxf(high, max_tree1(z));
    }
    const float top = high * scale;
    const bool grow = top > M + kGrow || (M == -INFINITY && top > -INFINITY);
    if (__any_sync(0xFFFFFFFFu, grow)) {
        const float f = grow ? exp2f(M - top) : 1.f;         // (0 for the first)
        if (grow) M = top;
        l *= f;
        if (sums) {
#pragma unroll 1
            for (int c = 0; c < D; c += 8) {                 // (few registers: seldom run)
                float o[8];
                tmem_ld8(to + c, o);
                tmem_wait_ld(o);
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] *= f;
                tmem_st8(to + c, o);
            }
        }
    }
    const float m = M == -INFINITY ? 0.f : M - kBits;
    const uint64_t nm = pack2(-m, -m), cc = pack2(scale, scale);
    uint64_t l0 = 0, l1 = 0;
    auto weigh = [&](const float (&x)[32], int first) {
        uint32_t p[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            float y0, y1;
            unpack2(ffma2(pack2(x[2 * k], x[2 * k + 1]), cc, nm), y0, y1);
            y0 = ex2(y0);
            y1 = ex2(y1);
            if (k & 1) l1 = fadd2(l1, pack2(y0, y1));
            else l0 = fadd2(l0, pack2(y0, y1));
            const __half2 e = __floats2half2_rn(y0, y1);
            p[k] = reinterpret_cast<const uint32_t&>(e);
        }
        tmem_st16(tp + first / 2, p);
    };
#pragma unroll 1
    for (int c = 0; c < kTile; c += 32) {
        tmem_ld32(ts + c, z);
        tmem_wait_ld(z);
        seen(z, c);
        weigh(z, c);
    }
    float a, e;
    unpack2(fadd2(l0, l1), a, e);
    l += a + e;
}

// Items no more than blocks: record i is item i's.  Otherwise it is that of the item that goes on behind the run of
// block i, if one begins in the run and does.
__host__ __device__ __forceinline__ bool cuts_by_item(const AttendBatch& b, int blocks) { return b.pairs * b.n_kv_heads <= blocks; }

__device__ __forceinline__ AttendCut cut_of(const AttendBatch& b, const int* pre, int block, int blocks) {
    const Runs runs = attend_runs(pre[b.pairs] * b.n_kv_heads, blocks);
    const bool by_item = cuts_by_item(b, blocks);
    AttendCut cut{};
    int u = -1;
    if (by_item) {
        const int p = block / b.n_kv_heads;
        if (p < b.pairs) u = pre[p] * b.n_kv_heads + block % b.n_kv_heads * (pre[p + 1] - pre[p]);
    } else if (block + 1 < runs.blocks) {
        u = attend_run(runs, block + 1) - 1;
    }
    if (u < 0) return cut;
    const Item item = attend_item(b, pre, b.n_kv_heads, u);
    const int b0 = attend_block(runs, item.first), b1 = attend_block(runs, item.first + item.units - 1);
    if (b0 == b1 || (!by_item && b0 != block)) return cut;
    cut.seq = item.seq;
    cut.g = item.g;
    cut.row0 = item.tile * kRowTile;
    cut.rows = min(kRowTile, b.span[item.seq].m * b.G - cut.row0);
    cut.parts = b1 - b0 + 1;
    cut.block = b0;
    cut.skip = attend_run(runs, b0) == item.first ? 0 : 1;
    return cut;
}

template <int D>
__global__ void __launch_bounds__(kThreadsAt, 1) k_attend_tc(const __grid_constant__ AttendBatch b) {
    constexpr int kOp = kTile * D * 2;              // bytes of an operand tile
    constexpr bool kOver = D == 128;                // P in S's columns
    extern __shared__ uint8_t raw[];
    __shared__ Segment seg;
    Ctl* ctl = reinterpret_cast<Ctl*>(raw);
    int* pre = reinterpret_cast<int*>(raw + 1024);
    uint8_t* sq = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + kCtlBytes + 1023) & ~uintptr_t(1023));
    uint8_t* sk = sq + 2 * kOp;
    uint8_t* sv = sk + kStages * kOp;
    uint8_t* raw_rows = sv + kStages * kOp;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    attend_units(b, kRowTile, pre);
    if (threadIdx.x == 0) {
        const Runs runs = attend_runs(pre[b.pairs] * b.n_kv_heads, gridDim.x);
        const int at = min((int)blockIdx.x, runs.blocks);            // (blocks without a unit have an empty run)
        ctl->unit = ctl->run0 = attend_run(runs, at);
        ctl->run1 = attend_run(runs, min(at + 1, runs.blocks));
        ctl->segment = ctl->tiles = ctl->items[0] = ctl->items[1] = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&ctl->k_full[i], 4);
            mbar_init(&ctl->k_empty[i], 1);
            mbar_init(&ctl->v_full[i], 4);
            mbar_init(&ctl->v_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&ctl->s_full[i], 1);
            mbar_init(&ctl->p_full[i], 4);
            mbar_init(&ctl->pv_done[i], 1);
        }
        mbar_init(&ctl->done, 1);
        mbar_init(&ctl->stall, 1);
        ctl->wait_ns = b.wait_ns;
        ctl->abort = 0;
        fence_barrier_init();
    }
    if (warp == 16) {
        tmem_alloc(&ctl->tmem, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = ctl->tmem;
    static_assert(kTile * (D + 4) * 4 + 1024 + 8 * 32 * 36 * 4 <= 6 * kOp, "the results' way through the operands' memory");
    // Every role walks the run's segments by itself, in a branch of its own, whose registers are its own; all of
    // the block meets at a segment's beginning (the segment, then Q, are in shared memory) and end.
    const int log2g = b.G >> 1;                     // (G is 1, 2 or 4)
    auto begin = [&]() {
        if (ctl->unit >= ctl->run1 || *reinterpret_cast<volatile int*>(&ctl->abort)) return false;
        __syncthreads();
        const AttendSeq& s = b.s[seg.seq];
        // Q: row 128 h + r of the segment, zeros behind the last
        for (int e = threadIdx.x; e < 2 * kTile * (D / 8); e += kThreadsAt) {
            const int r = e / (D / 8), c = e % (D / 8), row = seg.row0 + r;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (r < seg.rows)
                v = __ldg(reinterpret_cast<const uint4*>(s.q + (int64_t)(row >> log2g) * s.s_tok +
                                                         (int64_t)((seg.g << log2g) + (row & (b.G - 1))) * s.s_head + c * 8));
            *reinterpret_cast<uint4*>(sq + (r / kTile) * kOp + piece(c / 8, kTile, r % kTile, c % 8)) = v;
        }
        fence_async_smem();
        __syncthreads();
        tc_fence_after();
        return true;
    };
    auto finish = [&](int n_tiles, int items) {
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (threadIdx.x == 0) {
            ctl->tiles += n_tiles;
            ctl->items[0] += (items + 1) / 2;
            ctl->items[1] += items / 2;
            ctl->unit += seg.n;
            ++ctl->segment;
        }
        __syncthreads();
    };
    // A stream is a half of the rows, not every other tile; tiles; items (item i: stream i % 2, tile i / 2 or i).
#define SEGMENT()                                             \
    const bool both = seg.rows > kTile;                       \
    const int n_tiles = (seg.len + kTile - 1) / kTile;        \
    const int items = both ? 2 * n_tiles : n_tiles

    if (warp >= 16) {
        // ---------------- products ----------------
        regs_down<kRegsIssue>();
        if (threadIdx.x == 18 * 32) b.cuts[blockIdx.x] = cut_of(b, pre, blockIdx.x, gridDim.x);
        __syncwarp();
        while (true) {
            if (threadIdx.x == 17 * 32 && ctl->unit < ctl->run1)
                attend_segment(b, pre, b.n_kv_heads, 0, ctl->unit, ctl->run1, D, kRowTile, &seg);
            __syncwarp();
            if (!begin()) break;
            SEGMENT();
            if (warp == 16 && elect_one()) {
                const uint32_t hi = (uint32_t)(smem_desc_sw128(0) >> 32), lo = (uint32_t)smem_desc_sw128(0);
                const uint32_t q0 = (smem_u32(sq) >> 4) + lo, k0 = (smem_u32(sk) >> 4) + lo, v0 = (smem_u32(sv) >> 4) + lo;
                const int tiles0 = ctl->tiles;
                bool ok = !b.stall || blockIdx.x || wait(&ctl->stall, 0, ctl, b.err, 8);
                auto score = [&](int i) {               // S of item i
                    const int h = i & 1, j = tiles0 + (both ? i >> 1 : i);
                    if (!wait(&ctl->k_full[j % kStages], (j / kStages) & 1, ctl, b.err, 0)) return false;
                    tc_fence_after();
                    const uint32_t q = q0 + (both ? h : 0) * (kOp >> 4), k = k0 + (j % kStages) * (kOp >> 4);
#pragma unroll 4
                    for (int x = 0; x < D / 16; ++x) {
                        const uint32_t off = (x / 4) * (kTile * 128 >> 4) + (x % 4) * 2;
                        umma_bf16(tmem + h * 128, desc(q + off, hi), desc(k + off, hi), idesc_bf16_f32(128, 128), x > 0);
                    }
                    umma_commit(&ctl->s_full[h]);
                    if (!both || h) umma_commit(&ctl->k_empty[j % kStages]);
                    return true;
                };
                for (int i = 0; i < 2 && i < items && ok; ++i) ok = score(i);
                for (int i = 0; i < items && ok; ++i) {
                    const int h = i & 1, j = tiles0 + (both ? i >> 1 : i), n = ctl->items[h] + (i >> 1);   // n-th item of its stream
                    if (!(ok = wait(&ctl->v_full[j % kStages], (j / kStages) & 1, ctl, b.err, 1))) break;
                    if (!(ok = wait(&ctl->p_full[h], n & 1, ctl, b.err, 2))) break;
                    tc_fence_after();
                    const uint32_t v = v0 + (j % kStages) * (kOp >> 4);
#pragma unroll 4
                    for (int x = 0; x < kTile / 16; ++x)
                        umma_f16_ts(tmem + 256 + h * D, (kOver ? tmem + h * 128 : tmem + 384 + h * 64) + x * 8, desc(v + (x / 4) * (D * 128 >> 4) + (x % 4) * 2, hi),
                                    idesc_f16_f32(128, D), i > 1 || x > 0);
                    umma_commit(&ctl->pv_done[h]);
                    if (!both || h) umma_commit(&ctl->v_empty[j % kStages]);
                    if (i + 2 < items) {
                        if (kOver) {
                            if (!(ok = wait(&ctl->pv_done[h], n & 1, ctl, b.err, 3))) break;
                            tc_fence_after();
                        }
                        ok = score(i + 2);
                    }
                }
                umma_commit(&ctl->done);
                drain(&ctl->done, ctl->segment & 1);
            }
            __syncwarp();
            if (!both) {
                __syncthreads();
                __syncthreads();
            }
            finish(n_tiles, items);
        }
    } else if (warp >= 12) {
        // ---------------- V ----------------
        regs_down<kRegsUnpack>();
        while (begin()) {
            SEGMENT();
            const int w = warp - 12, half = w / 2, q = lane / 8;
            const int word0 = (D / 64) * (4 * half + q), block = 8 * (w % 2) + lane % 8;    // words of eight elements, positions
            uint8_t* share = raw_rows + (warp - 8) * Share<D>::kBytes;
            const uint32_t share32 = smem_u32(share);
            uint32_t bad = 0;
            int t = 64 * (w % 2) + lane;                // of the next tile to copy
            if (n_tiles)
                copy_v<D>(share32, seg, segment_row(seg, t, segment_page(seg, t), b.err),
                          segment_row(seg, t + 32, segment_page(seg, t + 32), b.err), half);
            t += kTile;
            uint32_t lo = segment_page(seg, t), hi = segment_page(seg, t + 32);
            for (int i = 0; i < n_tiles; ++i) {
                const int j = ctl->tiles + i;
                copy_wait<0>();
                __syncwarp();
                const uint16_t* scales = reinterpret_cast<const uint16_t*>(share + Share<D>::kCodes) + (D == 128 ? q / 2 : half);
                uint32_t x[8], later[8] = {};                    // the first word of every row, and the second (D = 128)
                __half2 s2[4];
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const uint8_t* c = share + Share<D>::v_at(8 * (lane % 8) + y, q / 2) + (D == 128 ? (q % 2) * 8 : q * 4);
                    if (D == 128) {
                        const uint2 v = *reinterpret_cast<const uint2*>(c);
                        x[y] = v.x; later[y] = v.y;
                    } else {
                        x[y] = *reinterpret_cast<const uint32_t*>(c);
                    }
                }
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int row = 8 * (lane % 8) + 2 * y;
                    const uint32_t w2 = f16_scales(checked_scale(scales[2 * row], bad), checked_scale(scales[2 * row + 2], bad));
                    s2[y] = reinterpret_cast<const __half2&>(w2);
                }
                __syncwarp();
                if (i + 1 < n_tiles)
                    copy_v<D>(share32, seg, segment_row(seg, t, lo, b.err), segment_row(seg, t + 32, hi, b.err), half);
                t += kTile;
                lo = segment_page(seg, t), hi = segment_page(seg, t + 32);
                if (j >= kStages && !wait_warp(&ctl->v_empty[j % kStages], (j / kStages - 1) & 1, ctl, b.err, 4)) break;
                uint8_t* to = sv + (j % kStages) * kOp;
                // pairs of positions: low halves hold the nibbles of elements 0, 2, 4, 6, high ones those of 1, 3, 5, 7
#pragma unroll 1
                for (int k = 0; k < D / 64; ++k) {
#pragma unroll
                    for (int odd = 0; odd < 2; ++odd) {
                        uint32_t pair[4];
#pragma unroll
                        for (int y = 0; y < 4; ++y) pair[y] = __byte_perm(x[2 * y], x[2 * y + 1], odd ? 0x7632 : 0x5410);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t v[4];
#pragma unroll
                            for (int y = 0; y < 4; ++y) v[y] = value_f16(pair[y], e, s2[y]);
                            st_piece(to, piece(block / 8, D, (word0 + k) * 8 + 2 * e + odd, block % 8), v);
                        }
                    }
#pragma unroll
                    for (int y = 0; y < 8; ++y) x[y] = later[y];
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->v_full[j % kStages]);
            }
            copy_wait<0>();
            if (bad) atomicOr(b.err, kErrPackScale);
            if (!both) {
                __syncthreads();
                __syncthreads();
            }
            finish(n_tiles, items);
        }
    } else if (warp >= 8) {
        // ---------------- K ----------------
        regs_down<kRegsUnpack>();
        while (begin()) {
            SEGMENT();
            const int w = warp - 8, q = lane / 8;
            // pieces q (D / 32) + k of rows 32 w + 8 y + lane % 8 (whose last three bits the swizzle takes: lane % 8)
            const uint32_t at = piece(q * (D / 32) / 8, kTile, 32 * w, 0) + (lane % 8) * 128;
            const uint32_t col = ((q * (D / 32) % 8) ^ (lane % 8)) << 4;
            uint8_t* share = raw_rows + w * Share<D>::kBytes;
            const uint32_t share32 = smem_u32(share);
            uint32_t bad = 0;
            int t = 32 * w + lane;                      // of the next tile to copy
            if (n_tiles) copy_k<D>(share32, seg, segment_row(seg, t, segment_page(seg, t), b.err));
            t += kTile;
            uint32_t page = segment_page(seg, t);
            for (int i = 0; i < n_tiles; ++i) {
                const int j = ctl->tiles + i;
                copy_wait<0>();
                __syncwarp();
                uint32_t x[4][D / 32], sc[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int row = 8 * y + lane % 8;
                    const uint8_t* c = share + Share<D>::k_at(row, D == 128 ? q : q / 2) + (D == 128 ? 0 : (q % 2) * 8);
                    if (D == 128) {
                        const uint4 v = *reinterpret_cast<const uint4*>(c);
                        x[y][0] = v.x; x[y][1] = v.y; x[y][D / 32 - 2] = v.z; x[y][D / 32 - 1] = v.w;
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2*>(c);
                        x[y][0] = v.x; x[y][1] = v.y;
                    }
                    sc[y] = reinterpret_cast<const uint16_t*>(share + Share<D>::kCodes)[row * (D / 32) + q * (D / 32) / 4];
                }
                __syncwarp();
                if (i + 1 < n_tiles) copy_k<D>(share32, seg, segment_row(seg, t, page, b.err));
                t += kTile;
                page = segment_page(seg, t);
                if (j >= kStages && !wait_warp(&ctl->k_empty[j % kStages], (j / kStages - 1) & 1, ctl, b.err, 5)) break;
                uint8_t* to = sk + (j % kStages) * kOp + at;
#pragma unroll 1
                for (int y = 0; y < 4; ++y, to += 8 * 128) {
                    const uint32_t s2 = checked_scale(sc[0], bad) * 0x10001u;
#pragma unroll
                    for (int k = 0; k < D / 32; ++k) {
                        uint32_t v[4];
                        values_bf16(x[0][k], s2, v);
                        st_piece(to, col ^ (k << 4), v);
                    }
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        sc[k] = sc[k + 1];
#pragma unroll
                        for (int e = 0; e < D / 32; ++e) x[k][e] = x[k + 1][e];
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->k_full[j % kStages]);
            }
            copy_wait<0>();
            if (bad) atomicOr(b.err, kErrPackScale);
            if (!both) {
                __syncthreads();
                __syncthreads();
            }
            finish(n_tiles, items);
        }
    } else {
        // ---------------- softmax ----------------
        regs_up<kRegsSoftmax>();
        while (begin()) {
            SEGMENT();
            float M = -INFINITY, l = 0.f;           // the row's maximum, and its sum of weights
            const int h = warp >> 2, r0 = (both ? h * kTile : 0) + (warp & 3) * 32;
            const uint32_t lanes = (uint32_t)(warp & 3) << 21;               // 32 (warp % 4) << 16
            const uint32_t ts = tmem + lanes + h * 128, to = tmem + lanes + 256 + h * D;
            const uint32_t tp = kOver ? ts : tmem + lanes + 384 + h * 64;
            const bool any = r0 < seg.rows;                                  // a row of the warp exists
            const int mine = items > h ? (items - h + 1) / 2 : 0;            // items of the stream
            for (int n = 0; n < mine; ++n) {
                const int t0 = (both ? n : 2 * n + h) * kTile;
                if (!wait_warp(&ctl->s_full[h], (ctl->items[h] + n) & 1, ctl, b.err, 6)) break;
                tc_fence_after();
                if (any) {
                    // columns [c0, c1) of the row are seen
                    const bool edge = t0 + kTile > seg.all_from || t0 < seg.all_to;
                    int c0 = 0, c1 = kTile;
                    if (edge) {
                        int64_t hi = seg.len - t0, lo = 0;
                        if (b.causal) {
                            const int64_t at = seg.at + (seg.row0 + min(r0 + lane, seg.rows - 1)) / b.G - t0;   // of the row's token
                            hi = min(hi, at + 1);
                            if (b.window) lo = at - b.window + 1;
                        }
                        c0 = (int)max((int64_t)0, min(lo, (int64_t)kTile));
                        c1 = (int)max((int64_t)0, min(hi, (int64_t)kTile));
                    }
                    if (edge) softmax_tile<D, true>(ts, tp, to, n > 0, c0, c1, b.scale_log2e, M, l);
                    else softmax_tile<D, false>(ts, tp, to, n > 0, 0, kTile, b.scale_log2e, M, l);
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->p_full[h]);
            }
            wait_warp(&ctl->done, ctl->segment & 1, ctl, b.err, 7);        // (returns at once where another role gave up)
            tc_fence_after();

            // The rows' results.  Alternate tiles: the second stream's go to the first through the operands' memory,
            // free by now (the products have ended).
            float* so = reinterpret_cast<float*>(sq);           // [128 rows][D + 4]
            float2* sml = reinterpret_cast<float2*>(sq + kTile * (D + 4) * 4);
            const int lr = (warp & 3) * 32 + lane;
            const float m = M - kBits;
            if (!both) {
                __syncthreads();
                if (h == 1) {
                    sml[lr] = make_float2(m, l);
                    if (items > 1) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            float o[32];
                            tmem_ld32(to + c, o);
                            tmem_wait_ld(o);
#pragma unroll
                            for (int k = 0; k < 32; k += 4)
                                *reinterpret_cast<float4*>(so + lr * (D + 4) + c + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                        }
                    }
                }
                __syncthreads();
            }
            if (both || h == 0) {
                const AttendSeq& s = b.s[seg.seq];
                const int r = (both ? h * kTile : 0) + lr;
                float f0 = 1.f, f1 = 0.f, mm = m, ll = l;
                if (!both) {
                    const float2 x = sml[lr];
                    mm = fmaxf(m, x.x);
                    f0 = m == -INFINITY ? 0.f : exp2f(m - mm);
                    f1 = x.x == -INFINITY ? 0.f : exp2f(x.x - mm);
                    ll = l * f0 + x.y * f1;
                }
                const bool whole = seg.n == seg.units;
                const int64_t slot = 2 * (int64_t)blockIdx.x + (ctl->unit == ctl->run0 ? 0 : 1);
                // 32 columns at a time through shared memory, so that eight lanes write a row's 128 bytes
                float* stage = reinterpret_cast<float*>(sq + kTile * (D + 4) * 4 + 1024) + warp * 32 * 36;
                const int r0w = r - lane;                               // the warp's first row
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    if (mine > 0) {
                        tmem_ld32(to + c, o);
                        tmem_wait_ld(o);
                    }
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (mine > 0 && f0 > 0.f) y = make_float4(o[k] * f0, o[k + 1] * f0, o[k + 2] * f0, o[k + 3] * f0);
                        if (!both && items > 1 && f1 > 0.f) {
                            const float4 z = *reinterpret_cast<const float4*>(so + lr * (D + 4) + c + k);
                            y.x += z.x * f1; y.y += z.y * f1; y.z += z.z * f1; y.w += z.w * f1;
                        }
                        *reinterpret_cast<float4*>(stage + lane * 36 + k) = y;
                    }
                    __syncwarp();
#pragma unroll 1
                    for (int i = 0; i < 32; i += 4) {
                        const int at = i + lane / 8, rr = r0w + at, d = c + (lane % 8) * 4;
                        const float4 y = *reinterpret_cast<const float4*>(stage + at * 36 + (lane % 8) * 4);
                        const float my = __shfl_sync(0xFFFFFFFFu, mm, at), ly = __shfl_sync(0xFFFFFFFFu, ll, at);
                        if (rr >= seg.rows) continue;
                        if (whole) attend_write<D>(b, s, seg.g, seg.row0 + rr, d, y, my, ly);
                        else *reinterpret_cast<float4*>(b.part + (slot * kRowTile + rr) * D + d) = y;
                    }
                    __syncwarp();
                }
                if (!whole && r < seg.rows) b.part_ml[slot * kRowTile + r] = make_float2(mm, ll);
            }
            finish(n_tiles, items);
        }
    }
#undef SEGMENT
    __syncthreads();
    if (warp == 16) tmem_dealloc(tmem, 512);
}

// Joins the parts of the items that runs' ends cut, one record's each (x).  A thread takes four elements of a row.
// Launched while the products are still running (griddepcontrol): nothing may be read, nor a block leave, before
// their end.  (With every block counting the units for itself, launched behind the products, 1024 tokens over 16384
// positions took 285 us for 270.)
template <int D>
__global__ void __launch_bounds__(256) k_attend_join(const __grid_constant__ AttendBatch b) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const AttendCut cut = b.cuts[blockIdx.x];
    if (cut.parts == 0) return;
    for (int e = blockIdx.y * 256 + threadIdx.x; e < cut.rows * (D / 4); e += kJoinBlocks * 256) {
        const int r = e / (D / 4), d = (e % (D / 4)) * 4;
        // (a prompt's items have two or three parts: with eight places each it took 270 us, with four 266)
        const Joined j = cut.parts <= 4 ? attend_join_row<D, 4>(b, 2 * cut.block, cut.skip, 2, cut.parts, kRowTile, r, d)
                                        : attend_join_row<D, 8>(b, 2 * cut.block, cut.skip, 2, cut.parts, kRowTile, r, d);
        attend_write<D>(b, b.s[cut.seq], cut.g, cut.row0 + r, d, j.y, j.M, j.l);
    }
}

template <int D>
cudaError_t launch(const AttendBatch& b, int blocks, cudaStream_t st) {
    static std::atomic<bool> set[64];     // (the attribute belongs to the device's function)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !set[dev]) {
        cudaFuncAttributes a;
        if ((e = cudaFuncGetAttributes(&a, k_attend_tc<D>)) != cudaSuccess) return e;
        if (a.numRegs < kRegs) return cudaErrorInvalidKernelImage;      // (the warp groups' shares need them all)
        e = cudaFuncSetAttribute(k_attend_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D>());
        if (e != cudaSuccess) return e;
        if (dev < 64) set[dev] = true;
    }
    k_attend_tc<D><<<blocks, kThreadsAt, smem_bytes<D>(), st>>>(b);
    e = cudaGetLastError();
    if (e != cudaSuccess || blocks == 1) return e;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(cuts_by_item(b, blocks) ? b.pairs * b.n_kv_heads : blocks - 1, kJoinBlocks);
    config.blockDim = dim3(256);
    config.stream = st;
    config.attrs = &early;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, k_attend_join<D>, b);
}

}  // namespace

cudaError_t launch_attend_tc(AttendBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    const int64_t units = attend_pairs(b, kRowTile);
    const int blocks = (int)(units < num_sms ? units : num_sms);
    const cudaError_t e = head_dim == 128 ? launch<128>(b, blocks, st) : launch<64>(b, blocks, st);
    b.stall = 0;
    return e;
}

}  // namespace cbk
