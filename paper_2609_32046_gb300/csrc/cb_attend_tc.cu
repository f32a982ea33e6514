// Attention over a 4-bit cache with many query rows a KV head: tcgen05 (cb_attend).
//
// A block takes up to 256 query rows (token, head of the group) of one KV head over a part of the
// positions, in tiles of 128 positions.  17 warps:
//   0..7    softmax, four a stream (TMEM lane quarter = warp % 4): a thread is a query row
//   8..11   K: four-bit rows from global memory, as bf16 into shared memory (K-major, 128-byte swizzle)
//   12..15  V: the same, transposed, as fp16
//   16      issues tcgen05.mma
// Two streams alternate on the tensor core, so that one's softmax runs beside the other's products: with
// more than 128 rows a stream is a half of the rows and both take every tile; with fewer the streams take
// alternate tiles of the same rows, each with its own maximum and sums, and join at the end.
//   S [128 rows][128 positions] = Q K^T            (bf16; fp32 in tensor memory)
//   P = exp2(S - M), fp16, back into tensor memory as the next product's A operand
//   O [128 rows][D] += P V                          (fp16)
// Tensor memory (512 columns): two S of 128, two O of D.  P has 64 columns: its own for D = 64, the lower
// half of S for D = 128.  There the next S's upper half is written first, by products that need no P,
// while the product that reads P ends; the lower half only once that has ended.
// O is scaled in place when a row's maximum has grown by more than 8 (log2 domain) since M was set: seldom
// after the first tiles; until then weights are up to 2^15, in fp16's range.
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "cb_attend.cuh"
#include "cb_internal.cuh"
#include "cb_sm100.cuh"

namespace cbk {
namespace {
using namespace sm100;

constexpr int kTile = 128;                  // positions a tile, rows a stream
constexpr int kWarpsAt = 17;
constexpr int kThreadsAt = kWarpsAt * 32;
constexpr int kStages = 2;
constexpr float kBits = 7.f;                // weights are exp2(z - M'), M' = M - 7
constexpr float kGrow = 8.f;                // growth of a row's maximum that M follows
constexpr uint32_t kPollNs = 1000000u;
constexpr uint64_t kDrainNs = 1000000000ull;

struct Ctl {
    uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
    uint64_t s_full[2], p_full[2], pv_done[2], done;
    uint64_t wait_ns;
    uint32_t tmem;
    int abort;
};

// Bytes: Q of two streams, K and V stages, 1 KB for the control block and 1 KB of alignment.
template <int D>
constexpr int smem_bytes() { return 2 * kTile * D * 2 + kStages * 2 * kTile * D * 2 + 2048; }

__device__ __forceinline__ uint64_t now_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Bounded wait: false when it gave up or another role did (bits 8 + tag of the error word name the wait).
static __device__ __noinline__ bool poll(uint64_t* bar, uint32_t parity, Ctl* c, uint32_t* err, int tag) {
    const uint64_t t0 = now_ns();
    for (uint32_t i = 1; i < (1u << 30); ++i) {
        if (mbar_try_wait_hint(bar, parity, kPollNs)) return true;
        if ((i & 63) == 0) {
            if (*reinterpret_cast<volatile int*>(&c->abort)) return false;
            if (now_ns() - t0 > c->wait_ns) break;
        }
    }
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

// A 16-byte piece of a K-major operand with 128-byte rows (64 elements a block): row, piece 0..7 of block.
__device__ __forceinline__ uint32_t piece(int block, int rows, int row, int p) {
    return (uint32_t)(block * rows * 128 + row * 128 + ((p ^ (row & 7)) << 4));
}

__device__ __forceinline__ void st_piece(uint8_t* base, uint32_t at, const uint32_t (&w)[4]) {
    *reinterpret_cast<uint4*>(base + at) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Positions of a tile as its threads read them: bf16 pieces of K.  Thread: rows 32 w + 8 i + lane % 8, the
// quarter lane / 8 of a row (D = 128: 16 bytes, one group; D = 64: 8 bytes, half a group).
template <int D>
struct KRows {
    uint32_t w[4][D / 32];
    uint32_t s[4];
};
template <int D>
__device__ __forceinline__ void load_k(KRows<D>& x, const PackedRows& p, const uint8_t* code, const uint16_t* scale,
                                       int64_t t0, int64_t end, int warp, int lane, uint32_t* err) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t t = t0 + warp * 32 + i * 8 + lane % 8;
        int64_t r = -1;
        if (t < end && (r = packed_row(p, t)) < 0) atomicOr(err, kErrPageIndex);
        x.s[i] = 0;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) x.w[i][k] = 0;
        if (r >= 0) {
            const uint8_t* c = code + r * (D / 2) + (lane / 8) * (D / 8);
            if (D == 128) {
                const uint4 v = __ldg(reinterpret_cast<const uint4*>(c));
                x.w[i][0] = v.x; x.w[i][1] = v.y; x.w[i][D / 32 - 2] = v.z; x.w[i][D / 32 - 1] = v.w;
            } else {
                const uint2 v = __ldg(reinterpret_cast<const uint2*>(c));
                x.w[i][0] = v.x; x.w[i][1] = v.y;
            }
            x.s[i] = __ldg(scale + r * (D / 32) + (lane / 8) * (D / 32) / 4);
        }
    }
}

// Eight positions 8 b .. 8 b + 7 of V, D / 64 words of eight elements of each.  b = 8 (warp % 2) + lane % 8,
// words (D / 64) (4 (warp / 2) + lane / 8) ..: eight neighbouring lanes write eight pieces of one row.
template <int D>
struct VRows {
    uint32_t w[8][D / 64];
    uint32_t s[8];
};
template <int D>
__device__ __forceinline__ void load_v(VRows<D>& x, const PackedRows& p, const uint8_t* code, const uint16_t* scale,
                                       int64_t t0, int64_t end, int warp, int lane, uint32_t* err) {
    const int at = 4 * (warp / 2) + lane / 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t t = t0 + 8 * (8 * (warp % 2) + lane % 8) + i;
        int64_t r = -1;
        if (t < end && (r = packed_row(p, t)) < 0) atomicOr(err, kErrPageIndex);
        x.s[i] = 0;
#pragma unroll
        for (int k = 0; k < D / 64; ++k) x.w[i][k] = 0;
        if (r >= 0) {
            const uint8_t* c = code + r * (D / 2) + at * (D / 16);
            if (D == 128) {
                const uint2 v = __ldg(reinterpret_cast<const uint2*>(c));
                x.w[i][0] = v.x; x.w[i][D / 64 - 1] = v.y;
            } else {
                x.w[i][0] = __ldg(reinterpret_cast<const uint32_t*>(c));
            }
            x.s[i] = __ldg(scale + r * (D / 32) + at * (D / 64) / 4);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreadsAt, 1) k_attend_tc(const __grid_constant__ AttendBatch b, int tiles_max,
                                                             int tile_rows) {
    constexpr int kOp = kTile * D * 2;              // bytes of an operand tile
    constexpr bool kOver = D == 128;                // P in S's columns
    extern __shared__ uint8_t raw[];
    Ctl* ctl = reinterpret_cast<Ctl*>(raw);
    uint8_t* sq = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1024 + 1023) & ~uintptr_t(1023));
    uint8_t* sk = sq + 2 * kOp;
    uint8_t* sv = sk + kStages * kOp;

    const AttendSeq& s = b.s[blockIdx.z];
    const int g = blockIdx.y / tiles_max, tile = blockIdx.y % tiles_max;
    if (tile >= s.tiles || (int)blockIdx.x >= s.splits) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int R = s.m * b.G, row0 = tile * tile_rows;
    const int rows = min(tile_rows, R - row0);      // of this block
    const bool both = rows > kTile;                 // a stream is a half of the rows, not every other tile
    const int64_t L = attend_length(s);
    const Span span = attend_span(b, s, L, row0, row0 + rows - 1, blockIdx.x, kTile);
    const int n_tiles = span.end > span.begin ? (int)((span.end - span.begin + kTile - 1) / kTile) : 0;
    const int items = both ? 2 * n_tiles : n_tiles;   // item i: stream i % 2, tile i / 2 or i

    if (threadIdx.x == 0) {
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
        ctl->wait_ns = b.wait_ns;
        ctl->abort = 0;
        fence_barrier_init();
    }
    if (warp == 16) {
        tmem_alloc(&ctl->tmem, 512);
        tmem_relinquish();
    }
    // Q: row 128 h + r of the block, zeros behind the last
    for (int e = threadIdx.x; e < 2 * kTile * (D / 8); e += kThreadsAt) {
        const int r = e / (D / 8), c = e % (D / 8), row = row0 + r;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < rows)
            v = __ldg(reinterpret_cast<const uint4*>(s.q + (int64_t)(row / b.G) * s.s_tok +
                                                     (int64_t)(g * b.G + row % b.G) * s.s_head + c * 8));
        *reinterpret_cast<uint4*>(sq + (r / kTile) * kOp + piece(c / 8, kTile, r % kTile, c % 8)) = v;
    }
    fence_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem;
    const int64_t head = (int64_t)g * s.kv.s_head;
    float M = -INFINITY, l = 0.f;                   // softmax threads: the row's maximum, and its sum of weights

    if (warp == 16) {
        if (elect_one()) {
            const uint64_t hi = smem_desc_sw128(0);
            const uint32_t q0 = smem_u32(sq) >> 4, k0 = smem_u32(sk) >> 4, v0 = smem_u32(sv) >> 4;
            bool ok = true;
            // S of item i: columns [64 half, 64 half + n)
            auto score = [&](int i, int half, int n) {
                const int h = i & 1, j = both ? i >> 1 : i;
                const uint32_t q = q0 + (both ? h : 0) * (kOp >> 4), k = k0 + (j % kStages) * (kOp >> 4) + half * (64 * 128 >> 4);
                const uint32_t id = idesc_bf16_f32(128, n);
#pragma unroll
                for (int x = 0; x < D / 16; ++x) {
                    const uint32_t off = (x / 4) * (kTile * 128 >> 4) + (x % 4) * 2;
                    umma_bf16(tmem + h * 128 + half * 64, hi | (q + off), hi | (k + off), id, x > 0);
                }
            };
            auto scored = [&](int i) {              // behind an item's last product with K
                const int j = both ? i >> 1 : i;
                umma_commit(&ctl->s_full[i & 1]);
                if (!both || (i & 1)) umma_commit(&ctl->k_empty[j % kStages]);
            };
            auto keys = [&](int i) {
                const int j = both ? i >> 1 : i;
                if (!wait(&ctl->k_full[j % kStages], (j / kStages) & 1, ctl, b.err, 0)) return false;
                tc_fence_after();
                return true;
            };
            for (int i = 0; i < 2 && i < items && ok; ++i) {
                if (!(ok = keys(i))) break;
                score(i, 0, 128);
                scored(i);
            }
            for (int i = 0; i < items && ok; ++i) {
                const int h = i & 1, j = both ? i >> 1 : i, n = i >> 1;     // n-th item of its stream
                if (!(ok = wait(&ctl->v_full[j % kStages], (j / kStages) & 1, ctl, b.err, 1))) break;
                if (!(ok = wait(&ctl->p_full[h], n & 1, ctl, b.err, 2))) break;
                tc_fence_after();
                const uint32_t p = kOver ? tmem + h * 128 : tmem + 384 + h * 64, v = v0 + (j % kStages) * (kOp >> 4);
#pragma unroll
                for (int x = 0; x < kTile / 16; ++x)
                    umma_f16_ts(tmem + 256 + h * D, p + x * 8, hi | (v + (x / 4) * (D * 128 >> 4) + (x % 4) * 2),
                                idesc_f16_f32(128, D), n > 0 || x > 0);
                umma_commit(&ctl->pv_done[h]);
                if (!both || h) umma_commit(&ctl->v_empty[j % kStages]);
                if (i + 2 < items) {
                    if (!(ok = keys(i + 2))) break;
                    if (kOver) {
                        score(i + 2, 1, 64);
                        if (!(ok = wait(&ctl->pv_done[h], n & 1, ctl, b.err, 3))) break;
                        tc_fence_after();
                        score(i + 2, 0, 64);
                    } else {
                        score(i + 2, 0, 128);
                    }
                    scored(i + 2);
                }
            }
            umma_commit(&ctl->done);
            drain(&ctl->done, 0);
        }
    } else if (warp >= 12) {
        // ---------------- V ----------------
        const uint8_t* code = s.kv.code[1] + head * (D / 2);
        const uint16_t* scale = s.kv.scale[1] + head * (D / 32);
        const int w = warp - 12;
        const int at = (D / 64) * (4 * (w / 2) + lane / 8), block = 8 * (w % 2) + lane % 8;
        uint32_t bad = 0;
        VRows<D> next;
        if (n_tiles) load_v<D>(next, s.kv, code, scale, span.begin, span.end, w, lane, b.err);
        for (int j = 0; j < n_tiles; ++j) {
            const VRows<D> x = next;
            if (j + 1 < n_tiles)
                load_v<D>(next, s.kv, code, scale, span.begin + (int64_t)(j + 1) * kTile, span.end, w, lane, b.err);
            if (j >= kStages && !wait_warp(&ctl->v_empty[j % kStages], (j / kStages - 1) & 1, ctl, b.err, 4)) break;
            uint8_t* to = sv + (j % kStages) * kOp;
            uint32_t s2[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) s2[i] = f16_scales(checked_scale(x.s[2 * i], bad), checked_scale(x.s[2 * i + 1], bad));
#pragma unroll
            for (int k = 0; k < D / 64; ++k) {
                uint32_t even[4][4], odd[4][4];          // [element / 2][pair of positions]
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t u[4], v[4];
                    values_f16<false>(__byte_perm(x.w[2 * i][k], x.w[2 * i + 1][k], 0x5410), s2[i], u);
                    values_f16<false>(__byte_perm(x.w[2 * i][k], x.w[2 * i + 1][k], 0x7632), s2[i], v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        even[e][i] = u[e];
                        odd[e][i] = v[e];
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    st_piece(to, piece(block / 8, D, (at + k) * 8 + 2 * e, block % 8), even[e]);
                    st_piece(to, piece(block / 8, D, (at + k) * 8 + 2 * e + 1, block % 8), odd[e]);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->v_full[j % kStages]);
        }
        if (bad) atomicOr(b.err, kErrPackScale);
    } else if (warp >= 8) {
        // ---------------- K ----------------
        const uint8_t* code = s.kv.code[0] + head * (D / 2);
        const uint16_t* scale = s.kv.scale[0] + head * (D / 32);
        const int w = warp - 8;
        uint32_t bad = 0;
        KRows<D> next;
        if (n_tiles) load_k<D>(next, s.kv, code, scale, span.begin, span.end, w, lane, b.err);
        for (int j = 0; j < n_tiles; ++j) {
            const KRows<D> x = next;
            if (j + 1 < n_tiles)
                load_k<D>(next, s.kv, code, scale, span.begin + (int64_t)(j + 1) * kTile, span.end, w, lane, b.err);
            if (j >= kStages && !wait_warp(&ctl->k_empty[j % kStages], (j / kStages - 1) & 1, ctl, b.err, 5)) break;
            uint8_t* to = sk + (j % kStages) * kOp;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t s2 = checked_scale(x.s[i], bad) * 0x10001u;
#pragma unroll
                for (int k = 0; k < D / 32; ++k) {
                    uint32_t v[4];
                    values_bf16(x.w[i][k], s2, v);
                    const int c = (lane / 8) * (D / 32) + k;             // piece of the row
                    st_piece(to, piece(c / 8, kTile, w * 32 + i * 8 + lane % 8, c % 8), v);
                }
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->k_full[j % kStages]);
        }
        if (bad) atomicOr(b.err, kErrPackScale);
    } else {
        // ---------------- softmax ----------------
        const int h = warp >> 2, r = (both ? h * kTile : 0) + (warp & 3) * 32 + lane, row = row0 + r;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;               // 32 (warp % 4) << 16
        const uint32_t ts = tmem + lanes + h * 128, to = tmem + lanes + 256 + h * D;
        const uint32_t tp = kOver ? ts : tmem + lanes + 384 + h * 64;
        const int64_t at = L - s.m + (row < R ? row : R - 1) / b.G;     // position of the row's token
        const bool any = (both ? h * kTile : 0) + (warp & 3) * 32 < rows;   // a row of the warp exists
        const uint64_t cc = pack2(b.scale_log2e, b.scale_log2e);
        const int mine = items > h ? (items - h + 1) / 2 : 0;            // items of the stream
        for (int n = 0; n < mine; ++n) {
            const int64_t t0 = span.begin + (int64_t)(both ? n : 2 * n + h) * kTile;
            if (!wait_warp(&ctl->s_full[h], n & 1, ctl, b.err, 6)) break;
            tc_fence_after();
            if (any) {
                // columns [c0, c1) of the row are seen
                const bool edge = t0 + kTile > span.all_from_here || t0 < span.all_to_here;
                int c0 = 0, c1 = kTile;
                if (edge) {
                    int64_t hi = span.end - t0, lo = 0;
                    if (b.causal) {
                        hi = min(hi, at + 1 - t0);
                        if (b.window) lo = at - b.window + 1 - t0;
                    }
                    c0 = (int)max((int64_t)0, min(lo, (int64_t)kTile));
                    c1 = (int)max((int64_t)0, min(hi, (int64_t)kTile));
                }
                float top = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < kTile; c += 32) {
                    float z[32];
                    tmem_ld32(ts + c, z);
                    tmem_wait_ld(z);
                    if (edge) {
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (c + k < c0 || c + k >= c1) z[k] = -INFINITY;
                    }
                    top = fmaxf(top, max_tree1(z));
                }
                top *= b.scale_log2e;
                const bool grow = top > M + kGrow || (M == -INFINITY && top > -INFINITY);
                if (__any_sync(0xFFFFFFFFu, grow)) {
                    const float f = grow ? exp2f(M - top) : 1.f;         // (0 for the first)
                    if (grow) M = top;
                    l *= f;
                    if (n > 0) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            float o[32];
                            tmem_ld32(to + c, o);
                            tmem_wait_ld(o);
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] *= f;
                            tmem_st32(to + c, o);
                        }
                    }
                }
                const float m = M == -INFINITY ? 0.f : M - kBits;
                const uint64_t nm = pack2(-m, -m);
                uint64_t l0 = 0, l1 = 0;
#pragma unroll 1
                for (int c = 0; c < kTile; c += 32) {
                    float z[32];
                    uint32_t p[16];
                    tmem_ld32(ts + c, z);
                    tmem_wait_ld(z);
                    if (edge) {
#pragma unroll
                        for (int k = 0; k < 32; ++k)
                            if (c + k < c0 || c + k >= c1) z[k] = -INFINITY;
                    }
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float y0, y1;
                        unpack2(ffma2(pack2(z[2 * k], z[2 * k + 1]), cc, nm), y0, y1);
                        y0 = ex2(y0);
                        y1 = ex2(y1);
                        if (k & 1) l1 = fadd2(l1, pack2(y0, y1));
                        else l0 = fadd2(l0, pack2(y0, y1));
                        const __half2 e = __floats2half2_rn(y0, y1);
                        p[k] = reinterpret_cast<const uint32_t&>(e);
                    }
                    tmem_st16(tp + c / 2, p);
                }
                float a, e;
                unpack2(fadd2(l0, l1), a, e);
                l += a + e;
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->p_full[h]);
        }
        wait_warp(&ctl->done, 0, ctl, b.err, 7);        // (returns at once where another role gave up)
        tc_fence_after();
    }

    // one stream's rows join the other's (alternate tiles): through the operands' memory, free by now
    float* so = reinterpret_cast<float*>(sq);           // [128 rows][D + 4]
    float2* sml = reinterpret_cast<float2*>(sq + kTile * (D + 4) * 4);
    const int h = warp >> 2, lr = (warp & 3) * 32 + lane;
    const uint32_t to = tmem + ((uint32_t)(warp & 3) << 21) + 256 + h * D;
    const float m = M - kBits;
    if (!both) {
        __syncthreads();                                // (every product has ended: the softmax warps waited for them)
        if (warp >= 4 && warp < 8) {
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
    if (warp < (both ? 8 : 4)) {
        const int r = (both ? h * kTile : 0) + lr, row = row0 + r;
        float f0 = 1.f, f1 = 0.f, mm = m, ll = l;
        if (!both) {
            const float2 x = sml[lr];
            mm = fmaxf(m, x.x);
            f0 = m == -INFINITY ? 0.f : exp2f(m - mm);
            f1 = x.x == -INFINITY ? 0.f : exp2f(x.x - mm);
            ll = l * f0 + x.y * f1;
        }
        const bool whole = s.splits == 1;
        const int64_t slot = s.slot0 + ((int64_t)g * s.tiles + tile) * s.splits + blockIdx.x;
        const int mine = h == 0 ? (items + 1) / 2 : items / 2;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
            float o[32];
            if (mine > 0) {
                tmem_ld32(to + c, o);
                tmem_wait_ld(o);
            }
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = mine > 0 && f0 > 0.f ? o[k] * f0 : 0.f;
            if (r < rows) {
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                    float4 y = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                    if (!both && items > 1 && f1 > 0.f) {
                        const float4 z = *reinterpret_cast<const float4*>(so + lr * (D + 4) + c + k);
                        y.x += z.x * f1; y.y += z.y * f1; y.z += z.z * f1; y.w += z.w * f1;
                    }
                    if (whole)
                        attend_write<D>(b, s, g, row, c + k, y, mm, ll);
                    else
                        *reinterpret_cast<float4*>(b.part + (slot * tile_rows + r) * D + c + k) = y;
                }
                if (!whole && c == 0) b.part_ml[slot * tile_rows + r] = make_float2(mm, ll);
            }
        }
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    if (warp == 16) tmem_dealloc(tmem, 512);
}

template <int D>
cudaError_t launch(const AttendBatch& b, dim3 grid, int tiles, int tile_rows, cudaStream_t st) {
    static bool set[64] = {};             // (the attribute belongs to the device's function)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !set[dev]) {
        e = cudaFuncSetAttribute(k_attend_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D>());
        if (e != cudaSuccess) return e;
        if (dev < 64) set[dev] = true;
    }
    k_attend_tc<D><<<grid, kThreadsAt, smem_bytes<D>(), st>>>(b, tiles, tile_rows);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_tc(AttendBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    int m = 0;
    for (int i = 0; i < b.n; ++i) m = b.s[i].m > m ? b.s[i].m : m;
    const int tile_rows = m * b.G <= kTile ? kTile : 2 * kTile;
    for (int64_t blocks = num_sms; !attend_plan(b, tile_rows, blocks, 2 * kTile, num_sms); blocks /= 2) {}
    int splits = 1, tiles = 1;
    for (int i = 0; i < b.n; ++i) {
        splits = b.s[i].splits > splits ? b.s[i].splits : splits;
        tiles = b.s[i].tiles > tiles ? b.s[i].tiles : tiles;
    }
    const dim3 grid((unsigned)splits, (unsigned)(b.n_kv_heads * tiles), (unsigned)b.n);
    cudaError_t e = head_dim == 128 ? launch<128>(b, grid, tiles, tile_rows, st) : launch<64>(b, grid, tiles, tile_rows, st);
    if (e == cudaSuccess) e = attend_join(b, head_dim, tile_rows, st);
    return e;
}

}  // namespace cbk
