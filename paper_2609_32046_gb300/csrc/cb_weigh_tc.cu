// Attention weights gathered from many query rows a KV head: tcgen05 (cb_weigh).
//
//   D [128 positions][128 query rows (token, head of the group)] = K Q^T     (bf16; fp32 in tensor memory, four buffers)
//   w[position] += sum over the columns of exp2(scale * log2(e) * D - lse * log2(e))
//
// A thread owns a position and 32 columns, so nothing is exchanged between threads but four partial sums.  28 warps:
//   0..15   sums: TMEM lane quarter = warp % 4, 32 columns a group of four
//   16..23  keys, unpacked as bf16, and query rows, copied (both K-major, 128-byte swizzle)
//   24      issues tcgen05.mma; 25 writes the weights; 26 finds the run's segments, one ahead
// Up to kStages tiles of query rows stay in shared memory while the tiles of positions pass through a ring; with
// more rows the ring's tiles of positions stay and the rows pass.
// lse * log2(e) is rounded once, and unlike in k_weigh_few what that leaves out is not multiplied into the weight, which would
// take a second read of shared memory for every product: weights are off by up to 2^-23 |lse| of themselves.
// A row whose lse is not finite is a row of zeros with an lse of infinity: it adds nothing.  A row's sum is one over its columns
// in a fixed order, whatever segment it is in.
//
// Measured (8 KV heads): 1024 tokens over 16384 positions, 32 heads of 128, 163 us, 0.82 PFLOP/s, where the products alone take
// 70; 33 drafts of 8 sequences over 6001, 16 heads of 64, 28 us. Bound by the sums: a tile's exponentials are 512 cycles, as long as
// its products, and the log-sum-exps read from shared memory compete with the products' operands (163 us of 190 without
// them); then by the chain of waits (107 us with no arithmetic in the sums, 73 with no products either). Other forms: the
// whole block meeting between segments 341; eight warps that sum 64 columns 181; masks in the same code as the rest 190;
// sums in shared memory by generic addresses 211; products issued by a lane that elect did not choose 214.
#include <atomic>
#include <cmath>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "cb_tc_roles.cuh"
#include "cb_weigh.cuh"

namespace cbk {
namespace {
using namespace sm100;

constexpr int kTile = 128;                  // positions a tile, query rows a tile
constexpr int kSumWarps = 16, kLoadWarps = 8, kIssueWarp = 24, kWriteWarp = 25, kFindWarp = 26, kWarpsWt = 28;
constexpr int kThreadsWt = kWarpsWt * 32;
constexpr int kReaders = kSumWarps + kLoadWarps + 2;   // warps that read a segment
constexpr int kLoadThreads = kLoadWarps * 32;
constexpr int kGroups = kSumWarps / 4;
constexpr int kBuffers = 4;                 // of 128 columns of tensor memory
constexpr int kTiles = 4;                   // tiles of positions in shared memory, and of their sums
template <int D> constexpr int kStages = D == 128 ? 2 : 4;    // tiles of query rows in shared memory
// Tiles of their log-sum-exps, which the sums read: rows are copied up to kStages tiles ahead of the products, and these are
// up to kBuffers + 1 buffers, of a tile each at most, ahead of the sums.
constexpr int kLse = 16;
constexpr int kMostTiles = 1024;              // of a segment (about a millisecond)
constexpr int kSeldomNs = 200;               // between looks of the warps that nothing waits for at once
static_assert(kLse >= 4 + kBuffers + 2, "");

// Positions that pass are in two of the tiles' places by turns; the other two hold their packed rows on their way, each of
// the warps that unpack its own share.
template <int D>
struct Share {
    static constexpr int kRows = kTile / kLoadWarps, kBytes = kRows * (D / 2 + D / 16);
    static constexpr int kAhead = 6;
    static_assert(kAhead * kBytes * kLoadWarps <= 2 * kTile * D * 2 && kBytes % 16 == 0, "");
    // Byte of piece p (16 bytes) of a row's codes: what eight lanes read at once (one quarter of eight rows) is in banks of its own.
    static __device__ __forceinline__ uint32_t at(int row, int p) {
        return row * (D / 2) + ((p ^ (D == 128 ? (row >> 1) & 3 : (row >> 2) & 1)) << 4);
    }
};

struct Ctl {
    uint64_t k_full[kTiles], k_empty[kTiles], q_full[4], q_empty[4];
    uint64_t d_full[kBuffers], d_empty[kBuffers], sum_full[kTiles], sum_empty[kTiles];
    uint64_t seg_full[2], seg_empty[2];
    uint64_t done, stall;
    uint64_t wait_ns;
    uint32_t tmem;
    int abort;
    int loaded;             // what the load warps' wait came to
};
// A segment of the run, and the tiles [q0, q1) of query rows that see something of it (n = 0: the run is over).
struct Part {
    Segment x;
    int q0, q1;
};
constexpr int kCtlBytes = 1024;
static_assert(sizeof(Ctl) <= kCtlBytes, "");

template <int D>
constexpr int smem_bytes() {
    return (kTiles + kStages<D>)*kTile * D * 2 + kLse * kTile * 4 + kTiles * kGroups * kTile * 4 + kCtlBytes + 1024;
}

// What a role knows of a segment.
struct View {
    WeighRows w;
    int rows, log2g, q0, q1, tiles;
    bool resident;          // the rows stay, the positions pass
    __device__ __forceinline__ View(const WeighBatch& b, const Part& p, int stages)
        : w(b, p.x), rows(p.x.rows), log2g(b.G >> 1), q0(p.q0), q1(p.q1), tiles((p.x.len + kTile - 1) / kTile),
          resident(p.q1 - p.q0 <= stages) {}
    __device__ __forceinline__ int first_token(int q) const { return (q * kTile) >> log2g; }
    __device__ __forceinline__ int last_token(int q) const { return (min(rows, (q + 1) * kTile) - 1) >> log2g; }
    // Tiles of positions [first, last) that some token of a .. b sees a position of; those before `low` and from `high` on
    // not every one of them sees whole.
    struct Span {
        int first, last, low, high;
    };
    __device__ __forceinline__ Span span(int a, int b) const {
        if (w.tree) return Span{0, tiles, 0, max(w.at, 0) / kTile};
        if (!w.causal) return Span{0, tiles, 0, tiles};
        // (position t is seen by the tokens from t - at on and before t - at + window)
        Span s{0, min(tiles, max(0, w.at + b + kTile) / kTile), 0, max(0, w.at + a + 1) / kTile};
        if (w.window) {
            s.first = max(0, w.at + a - w.window + 1) / kTile;
            s.low = max(0, w.at + b - w.window + kTile) / kTile;
        }
        return s;
    }
    __device__ __forceinline__ Span span_of(int q) const { return span(first_token(q), last_token(q)); }
    // Those that some tile of rows has something to add to.
    __device__ __forceinline__ Span used() const {
        return q0 < q1 ? span(first_token(q0), last_token(q1 - 1)) : Span{0, 0, 0, 0};
    }
};

// Copies 16 bytes into shared memory, or zeros.
__device__ __forceinline__ void copy16_or_0(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}

// Shared memory by its own addresses.
__device__ __forceinline__ float4 lds128(uint32_t at) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float lds(uint32_t at) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void sts(uint32_t at, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }

// A thread's share of a tile's keys on their way: a quarter of each of two rows.
template <int D>
struct Codes {
    uint4 x[2];
    uint32_t scale[2];
};

template <int D>
__global__ void __launch_bounds__(kThreadsWt, 1) k_weigh_tc(const __grid_constant__ WeighBatch b) {
    constexpr int kOp = kTile * D * 2;              // bytes of an operand tile
    extern __shared__ uint8_t raw[];
    __shared__ Part parts[2];
    __shared__ int pre[kMaxBatch + 1];
    Ctl* ctl = reinterpret_cast<Ctl*>(raw);
    uint8_t* sk = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + kCtlBytes + 1023) & ~uintptr_t(1023));
    uint8_t* sq = sk + kTiles * kOp;
    float* s_lse = reinterpret_cast<float*>(sq + kStages<D> * kOp);      // [tile of rows % kLse][row]: -lse * log2(e)
    float* s_sum = s_lse + kLse * kTile;                                  // [tile % kTiles][group][position]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    attend_units(b, kWeighRows, pre);
    if (threadIdx.x == 0) {
        for (int i = 0; i < kTiles; ++i) {
            mbar_init(&ctl->k_full[i], kLoadWarps);
            mbar_init(&ctl->k_empty[i], 1);
            mbar_init(&ctl->sum_full[i], kSumWarps);
            mbar_init(&ctl->sum_empty[i], 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&ctl->q_full[i], kLoadWarps);
            mbar_init(&ctl->q_empty[i], 1);
        }
        for (int i = 0; i < kBuffers; ++i) {
            mbar_init(&ctl->d_full[i], 1);
            mbar_init(&ctl->d_empty[i], kSumWarps);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&ctl->seg_full[i], 1);
            mbar_init(&ctl->seg_empty[i], kReaders);
        }
        mbar_init(&ctl->done, 1);
        mbar_init(&ctl->stall, 1);
        ctl->wait_ns = b.wait_ns;
        ctl->abort = 0;
        fence_barrier_init();
    }
    if (warp == kIssueWarp) {
        tmem_alloc(&ctl->tmem, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl->tmem;

    // Every role walks the run's segments by itself; what passes from one to another goes by the barriers alone.
    // nth: segments taken.  False at the end, or where a role gave up.
    uint32_t nth = 0;
    auto begin = [&]() {
        return wait_warp(&ctl->seg_full[nth & 1], nth >> 1 & 1, ctl, b.err, 9) && parts[nth & 1].x.n > 0;
    };
    auto finish = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(&ctl->seg_empty[nth & 1]);
        ++nth;
    };

    if (warp < kSumWarps) {
        // ---------------- sums ----------------
        const int group = warp >> 2, mine = (warp & 3) * 32 + lane;
        const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + 32 * group;      // (lane 32 (warp % 4) << 16)
        const uint64_t cc = pack2(b.scale_log2e, b.scale_log2e);
        const uint32_t sums = smem_u32(s_sum) + 4 * (group * kTile + mine), lses = smem_u32(s_lse) + 128 * group;
        uint32_t item = 0, n_q = 0, n_tile = 0;
        bool ok = true;
        while (ok && begin()) {
            const Part& part = parts[nth & 1];
            const View v(b, part, kStages<D>);
            // bit e: query row row0 + e sees the thread's position of tile k
            auto sees = [&](int row0, int k) {
                const int t = k * kTile + mine;
                if (v.w.tree) {
                    const TreeBits tree = b.w[part.x.seq].tree;
                    uint32_t bits = 0, rows = 0;
#pragma unroll 1
                    for (int e = 0; e < 32; ++e) {
                        if (((row0 + e) & (b.G - 1)) == 0)
                            rows = tree_bits(tree.seen + min((row0 + e) >> v.log2g, v.w.m - 1) * tree.s_row, (v.w.m + 31) / 32,
                                             t - lane - v.w.at) >> lane & 1u;
                        bits |= rows << e;
                    }
                    return bits;
                }
                // tokens from t - at on, and before t - at + window
                const int64_t lo = ((int64_t)(t - v.w.at) << v.log2g) - row0;
                const int64_t hi = v.w.window ? lo + ((int64_t)v.w.window << v.log2g) : 32;
                const int c0 = (int)max((int64_t)0, min(lo, (int64_t)32)), c1 = (int)max((int64_t)0, min(hi, (int64_t)32));
                return c0 >= c1 ? 0u : (0xFFFFFFFFu << c0) & (0xFFFFFFFFu >> (32 - c1));
            };
            // the sum of the thread's columns of one product; some: its group has any
            auto gather = [&](int row0, int k, bool some, bool edge, uint32_t lse) {
                const uint32_t d = item % kBuffers, phase = item / kBuffers & 1;
                ++item;
                if (!(ok = wait_warp(&ctl->d_full[d], phase, ctl, b.err, 10))) return 0.f;
                if (!some) {
                    if (lane == 0) mbar_arrive(&ctl->d_empty[d]);
                    return 0.f;
                }
                tc_fence_after();
                auto leave = [&]() {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl->d_empty[d]);
                };
                if (edge) {                                     // (apart: what is masked in place is moved about elsewhere too)
                    const uint32_t bits = sees(row0, k);
                    float sum = 0.f;
#pragma unroll 1
                    for (int c = 0; c < 32; c += 8) {
                        float z[8];
                        tmem_ld8(from + d * 128 + c, z);
                        tmem_wait_ld(z);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            sum += bits >> (c + e) & 1u ? ex2(fmaf(z[e], b.scale_log2e, lds(lse + 4 * (c + e)))) : 0.f;
                    }
                    leave();
                    return sum;
                }
                float z[32];
                tmem_ld32(from + d * 128, z);
                tmem_wait_ld(z);
                leave();
                uint64_t l0 = 0, l1 = 0;
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    const float4 nl = lds128(lse + 4 * e);
                    float y0, y1, y2, y3;
                    unpack2(ffma2(pack2(z[e], z[e + 1]), cc, pack2(nl.x, nl.y)), y0, y1);
                    unpack2(ffma2(pack2(z[e + 2], z[e + 3]), cc, pack2(nl.z, nl.w)), y2, y3);
                    l0 = fadd2(l0, pack2(ex2(y0), ex2(y1)));
                    l1 = fadd2(l1, pack2(ex2(y2), ex2(y3)));
                }
                float a0, a1;
                unpack2(fadd2(l0, l1), a0, a1);
                return a0 + a1;
            };
            auto place = [&](int k) { return sums + (n_tile + k) % kTiles * (kGroups * kTile * 4); };
            // a tile's place in shared memory, which the writer has left
            auto open = [&](int k) {
                const uint32_t n = n_tile + k;
                if (n >= kTiles && !wait_warp(&ctl->sum_empty[n % kTiles], (n / kTiles - 1) & 1, ctl, b.err, 11)) ok = false;
                return ok;
            };
            auto close = [&](int k) {
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->sum_full[(n_tile + k) % kTiles]);
            };
            auto lse_at = [&](int q) { return lses + (n_q + q - v.q0) % kLse * (kTile * 4); };
            if (v.resident) {
                for (int k = 0; k < v.tiles && open(k); ++k) {
                    float sum = 0.f;
                    for (int q = v.q0; q < v.q1 && ok; ++q) {
                        const View::Span s = v.span_of(q);
                        const int row0 = q * kTile + 32 * group;
                        if (k >= s.first && k < s.last) sum += gather(row0, k, row0 < v.rows, k < s.low || k >= s.high, lse_at(q));
                    }
                    sts(place(k), sum);
                    close(k);
                }
            } else {
                for (int k = 0; k < v.tiles && open(k); ++k) sts(place(k), 0.f);
                for (int q = v.q0; q < v.q1 && ok; ++q) {
                    const View::Span s = v.span_of(q);
                    const int row0 = q * kTile + 32 * group;
                    const uint32_t lse = lse_at(q);
#pragma unroll 1
                    for (int k = s.first; k < s.last && ok; ++k) {
                        const float sum = gather(row0, k, row0 < v.rows, k < s.low || k >= s.high, lse);
                        sts(place(k), lds(place(k)) + sum);
                    }
                }
                for (int k = 0; k < v.tiles; ++k) close(k);
            }
            n_tile += v.tiles;
            n_q += v.q1 - v.q0;
            finish();
        }
    } else if (warp < kIssueWarp) {
        // ---------------- keys and query rows ----------------
        const int lw = warp - kSumWarps, quarter = lane / 8;
        // rows 16 lw + 8 y + lane % 8 of a tile (whose last three bits the swizzle takes), pieces quarter (D / 32) + e
        const uint32_t at = piece(quarter * (D / 32) / 8, kTile, 16 * lw, 0) + (lane % 8) * 128;
        const uint32_t col = ((quarter * (D / 32) % 8) ^ (lane % 8)) << 4;
        // query rows: thread u has piece u % P of rows u / P, u / P + N ..., which all are of one head
        constexpr int P = D / 8, N = kLoadThreads / P, R = kTile / N;
        static_assert(N % 8 == 0, "");
        const int u = threadIdx.x - kSumWarps * 32;
        const uint32_t q_at = smem_u32(sq) + piece(u % P / 8, kTile, u / P, u % P % 8);
        uint8_t* share = sk + 2 * kOp + lw * (Share<D>::kAhead * Share<D>::kBytes);
        const uint32_t share32 = smem_u32(share);
        uint32_t n_q = 0, k_parity = 0, k_used = 0, bad = 0;      // bits: uses of a tile's place, any use
        // One warp waits for all eight, which meet at a barrier in hardware: eight warps that poll took the issue slots of
        // the sums.  (They meet whatever it saw, and all go by it.)
        auto together = [&](uint64_t* bar, uint32_t parity, int tag) {
            if (lw == 0) {
                const bool there = wait_warp(bar, parity, ctl, b.err, tag);
                if (lane == 0) ctl->loaded = there;
            }
            asm volatile("bar.sync 2, %0;" ::"n"(kLoadThreads) : "memory");
            const bool there = *reinterpret_cast<volatile int*>(&ctl->loaded);
            asm volatile("bar.sync 2, %0;" ::"n"(kLoadThreads) : "memory");
            return there;
        };
        bool ok = true;
        while (ok && together(&ctl->seg_full[nth & 1], nth >> 1 & 1, 9) && parts[nth & 1].x.n > 0) {
            const Part& part = parts[nth & 1];
            const Segment& x = part.x;
            const View v(b, part, kStages<D>);
            const AttendSeq& s = b.s[x.seq];
            const int head = (x.g << v.log2g) + ((u / P) & (b.G - 1));
            const float* lses = b.w[x.seq].lse + head;
            const uint16_t* q_from = s.q + (int64_t)head * s.s_head + u % P * 8;
            const int64_t tok_bytes = s.s_tok;
            auto vacant = [&](int slot) {
                return !(k_used >> slot & 1) || together(&ctl->k_empty[slot], (k_parity >> slot & 1) ^ 1, 13);
            };
            auto filled = [&](int slot) {
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->k_full[slot]);
                k_parity ^= 1u << slot;
                k_used |= 1u << slot;
            };
            auto lse_of = [&](int q, float (&lse)[R]) {
                const int row0 = q * kTile + u / P;
                const float* from = lses + (int64_t)(row0 >> v.log2g) * b.n_q_heads;
                const int step = (N >> v.log2g) * b.n_q_heads;
#pragma unroll
                for (int i = 0; i < R; ++i) lse[i] = row0 + i * N < v.rows ? __ldg(from + i * step) : INFINITY;
            };
            auto copy_rows = [&](int q, const float (&lse)[R]) {       // into a stage that the products have left
                const uint32_t n = n_q + q - v.q0;
                if (n >= (uint32_t)kStages<D> && !together(&ctl->q_empty[n % kStages<D>], (n / kStages<D> - 1) & 1, 12)) {
                    ok = false;
                    return;
                }
                const uint32_t to = q_at + n % kStages<D> * kOp;
                const uint16_t* from = q_from + (int64_t)((q * kTile + u / P) >> v.log2g) * tok_bytes;
                const int64_t step = (N >> v.log2g) * tok_bytes;
                float* l = s_lse + n % kLse * kTile + u / P;
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const bool there = isfinite(lse[i]);
                    copy16_or_0(to + i * N * 128, from + i * step, there);            // (reads nothing where it is not)
                    if (u % P == 0) l[i * N] = there ? lse[i] * -b.lse_log2e : -INFINITY;
                }
            };
            auto landed = [&](int q) {
                copy_commit();
                copy_wait<0>();
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->q_full[(n_q + q - v.q0) % kStages<D>]);
            };
            // a quarter of a row: codes as numbers
            auto unpack = [&](uint8_t* to, const uint32_t (&word)[4], uint32_t scale) {
                const uint32_t s2 = checked_scale(scale, bad) * 0x10001u;
#pragma unroll
                for (int e = 0; e < D / 32; ++e) {
                    uint32_t w[4];
                    values_bf16(word[e], s2, w);
                    st_piece(to, col ^ (e << 4), w);
                }
            };
            float lse[R];
            const View::Span used = v.used();
            const int q_first = min(v.q1, v.q0 + kStages<D>);           // the rows that stay, or the first that pass
            if (v.resident) {
                // tiles of positions pass: their packed rows kAhead tiles ahead, the block-table entries one more
                ok = vacant(2) && vacant(3);
                const int mine = 16 * lw + lane % 16;                   // (lanes 16 on look the same rows up)
                int ahead = used.first;
                uint32_t page = segment_page(x, ahead * kTile + mine);
                auto copy_keys = [&]() {
                    if (ahead < used.last) {
                        constexpr int C = D / 32;                       // pieces of a row's codes
                        const uint32_t to = share32 + ahead % Share<D>::kAhead * Share<D>::kBytes;
                        const int row = segment_row(x, ahead * kTile + mine, page, b.err);
#pragma unroll
                        for (int i = 0; i < C / 2; ++i) {
                            const int r = lane / C + i * (32 / C);
                            const int from = max(0, __shfl_sync(0xFFFFFFFFu, row, r));
                            copy16(to + Share<D>::at(r, lane % C), x.code[0] + (uint64_t)from * (D / 2) + lane % C * 16);
                        }
                        if (lane < 16)
                            copy_small<D / 16>(to + Share<D>::kRows * (D / 2) + lane * (D / 16),
                                               reinterpret_cast<const uint8_t*>(x.scale[0]) + (uint64_t)max(0, row) * (D / 16), row >= 0);
                    }
                    copy_commit();
                    ++ahead;
                    page = segment_page(x, ahead * kTile + mine);
                };
                // the rows' log-sum-exps, and the first packed rows, while they are on their way
                if (v.q0 < v.q1) lse_of(v.q0, lse);
                if (ok)
                    for (int i = 0; i < Share<D>::kAhead - 1; ++i) copy_keys();
                for (int q = v.q0; q < q_first && ok; ++q) {
                    if (q > v.q0) lse_of(q, lse);
                    copy_rows(q, lse);
                    if (ok) landed(q);
                }
                for (int k = used.first; k < used.last && ok; ++k) {
                    const int slot = (k - used.first) & 1;
                    copy_keys();
                    copy_wait<Share<D>::kAhead - 1>();
                    __syncwarp();
                    if (!(ok = vacant(slot))) break;
                    const uint8_t* rows = share + k % Share<D>::kAhead * Share<D>::kBytes;
                    uint8_t* to = sk + slot * kOp + at;
#pragma unroll
                    for (int y = 0; y < 2; ++y, to += 8 * 128) {
                        const int row = 8 * y + lane % 8;
                        const uint8_t* c = rows + Share<D>::at(row, D == 128 ? quarter : quarter / 2) + (D == 128 ? 0 : quarter % 2 * 8);
                        uint32_t word[4] = {};
                        if (D == 128) {
                            const uint4 w = *reinterpret_cast<const uint4*>(c);
                            word[0] = w.x; word[1] = w.y; word[2] = w.z; word[3] = w.w;
                        } else {
                            const uint2 w = *reinterpret_cast<const uint2*>(c);
                            word[0] = w.x; word[1] = w.y;
                        }
                        unpack(to, word, reinterpret_cast<const uint16_t*>(rows + Share<D>::kRows * (D / 2))[row * (D / 32) + quarter * (D / 32) / 4]);
                    }
                    filled(slot);
                }
                copy_wait<0>();
            } else {
                // at most kTiles tiles stay: read ahead into registers
                auto read_keys = [&](int k, Codes<D>& c) {
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int t = k * kTile + 16 * lw + 8 * y + lane % 8;
                        c.x[y] = make_uint4(0, 0, 0, 0);
                        c.scale[y] = 0;
                        const int r = k < used.last ? segment_row(x, t, segment_page(x, t), b.err) : -1;
                        if (r < 0) continue;
                        const uint8_t* from = x.code[0] + (uint64_t)r * (D / 2) + quarter * (D / 8);
                        if (D == 128) {
                            c.x[y] = __ldg(reinterpret_cast<const uint4*>(from));
                        } else {
                            const uint2 w = __ldg(reinterpret_cast<const uint2*>(from));
                            c.x[y].x = w.x;
                            c.x[y].y = w.y;
                        }
                        c.scale[y] = __ldg(x.scale[0] + (uint64_t)r * (D / 32) + quarter * (D / 32) / 4);
                    }
                };
                Codes<D> c0, c1;
                lse_of(v.q0, lse);
                read_keys(used.first, c0);
                read_keys(used.first + 1, c1);
                copy_rows(v.q0, lse);
                if (ok) landed(v.q0);
                for (int k = used.first; k < used.last && ok; ++k) {
                    const int slot = k - used.first;
                    if (!(ok = vacant(slot))) break;
                    uint8_t* to = sk + slot * kOp + at;
#pragma unroll
                    for (int y = 0; y < 2; ++y, to += 8 * 128) {
                        const uint32_t word[4] = {c0.x[y].x, c0.x[y].y, c0.x[y].z, c0.x[y].w};
                        unpack(to, word, c0.scale[y]);
                    }
                    filled(slot);
                    c0 = c1;
                    read_keys(k + 2, c1);
                }
                lse_of(v.q0 + 1, lse);
                for (int q = v.q0 + 1; q < v.q1 && ok; ++q) {
                    copy_rows(q, lse);
                    lse_of(min(q + 1, v.q1 - 1), lse);
                    if (ok) landed(q);
                }
            }
            n_q += v.q1 - v.q0;
            finish();
        }
        copy_wait<0>();
        if (bad) atomicOr(b.err, kErrPackScale);
    } else if (warp == kIssueWarp) {
        // ---------------- products ----------------
        const uint32_t hi = (uint32_t)(smem_desc_sw128(0) >> 32), lo = (uint32_t)smem_desc_sw128(0);
        const uint32_t kd = (smem_u32(sk) >> 4) + lo, qd = (smem_u32(sq) >> 4) + lo;
        // (one thread for all of it, by elect: with a lane chosen otherwise the descriptors are not kept in the
        // registers that the instruction takes them from)
        if (elect_one()) {
            uint32_t item = 0, n_q = 0, k_parity = 0;
            bool ok = !b.stall || blockIdx.x || wait(&ctl->stall, 0, ctl, b.err, 14);
            for (; ok && wait(&ctl->seg_full[nth & 1], nth >> 1 & 1, ctl, b.err, 9) && parts[nth & 1].x.n > 0; ++nth) {
                const View v(b, parts[nth & 1], kStages<D>);
                const View::Span used = v.used();
                auto q_there = [&](int q) {
                    const uint32_t n = n_q + q - v.q0;
                    return wait(&ctl->q_full[n % kStages<D>], n / kStages<D> & 1, ctl, b.err, 14);
                };
                auto k_there = [&](int slot) { return wait(&ctl->k_full[slot], k_parity >> slot & 1, ctl, b.err, 15); };
                auto k_done = [&](int slot) {
                    umma_commit(&ctl->k_empty[slot]);
                    k_parity ^= 1u << slot;
                };
                auto product = [&](uint32_t qa, uint32_t idesc, int slot) {
                    const uint32_t d = item % kBuffers;
                    if (item >= kBuffers && !wait(&ctl->d_empty[d], (item / kBuffers - 1) & 1, ctl, b.err, 16)) return false;
                    tc_fence_after();
                    const uint32_t ka = kd + slot * (kOp >> 4);
#pragma unroll
                    for (int y = 0; y < D / 16; ++y) {
                        const uint32_t off = (y / 4) * (kTile * 128 >> 4) + (y % 4) * 2;
                        umma_bf16(tmem + d * 128, desc(ka + off, hi), desc(qa + off, hi), idesc, y > 0);
                    }
                    umma_commit(&ctl->d_full[d]);
                    ++item;
                    return true;
                };
                auto rows_at = [&](int q) { return qd + (n_q + q - v.q0) % kStages<D> * (kOp >> 4); };
                auto idesc_of = [&](int q) { return idesc_bf16_f32(kTile, (min(kTile, v.rows - q * kTile) + 31) & ~31); };   // (what the sums read)
                if (v.resident) {
                    for (int q = v.q0; q < v.q1 && ok; ++q) ok = q_there(q);
                    for (int k = used.first; k < used.last && ok; ++k) {
                        const int slot = (k - used.first) & 1;
                        if (!(ok = k_there(slot))) break;
                        for (int q = v.q0; q < v.q1 && ok; ++q) {
                            const View::Span s = v.span_of(q);
                            if (k >= s.first && k < s.last) ok = product(rows_at(q), idesc_of(q), slot);
                        }
                        k_done(slot);
                    }
                    for (int q = v.q0; q < v.q1; ++q) umma_commit(&ctl->q_empty[(n_q + q - v.q0) % kStages<D>]);
                } else {
                    uint32_t there = 0;
                    for (int q = v.q0; q < v.q1 && ok; ++q) {
                        if (!(ok = q_there(q))) break;
                        const View::Span s = v.span_of(q);
                        for (int k = s.first; k < s.last && ok; ++k) {
                            const int slot = k - used.first;
                            if (!(there >> slot & 1)) ok = k_there(slot);
                            there |= 1u << slot;
                            if (ok) ok = product(rows_at(q), idesc_of(q), slot);
                        }
                        umma_commit(&ctl->q_empty[(n_q + q - v.q0) % kStages<D>]);
                    }
                    for (int k = used.first; k < used.last; ++k) k_done(k - used.first);
                }
                n_q += v.q1 - v.q0;
                mbar_arrive(&ctl->seg_empty[nth & 1]);
            }
            umma_commit(&ctl->done);
            drain(&ctl->done, 0);
        }
        __syncwarp();
    } else if (warp == kWriteWarp) {
        // ---------------- weights ----------------
        uint32_t n_tile = 0;
        bool ok = true;
        while (ok && begin()) {
            const Part& part = parts[nth & 1];
            const View v(b, part, kStages<D>);
            const WeighSeq& ws = b.w[part.x.seq];
            const int g = part.x.g;
            float* to = ws.weights + (int64_t)g * ws.w_head + v.w.begin;
            for (int k = 0; k < v.tiles && ok; ++k, ++n_tile) {
                float before[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) before[i] = v.w.before(ws, g, k * kTile + 32 * i + lane);
                if (!(ok = wait_warp<kSeldomNs>(&ctl->sum_full[n_tile % kTiles], n_tile / kTiles & 1, ctl, b.err, 17))) break;
                const float* sums = s_sum + n_tile % kTiles * kGroups * kTile + lane;
                float sum[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    sum[i] = sums[32 * i];
#pragma unroll
                    for (int y = 1; y < kGroups; ++y) sum[i] += sums[y * kTile + 32 * i];
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->sum_empty[n_tile % kTiles]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = k * kTile + 32 * i + lane;
                    if (t < v.w.len) to[t] = fmaf(b.decay, before[i], sum[i]);
                }
            }
            finish();
        }
    } else if (warp == kFindWarp) {
        // ---------------- segments ----------------
        if (lane == 0) {
            const Runs runs = attend_runs(pre[b.pairs] * b.n_kv_heads, gridDim.x);
            const int run = min((int)blockIdx.x, runs.blocks), end = attend_run(runs, min(run + 1, runs.blocks));
            int unit = attend_run(runs, run);
            for (bool more = true; more; ++nth) {
                Part& part = parts[nth & 1];
                if (nth >= 2 && !wait<kSeldomNs>(&ctl->seg_empty[nth & 1], (nth / 2 - 1) & 1, ctl, b.err, 18)) break;
                more = unit < end;
                part.x.n = 0;
                if (more) {
                    attend_segment(b, pre, b.n_kv_heads, 0, unit, end, D, kWeighRows, &part.x);
                    part.q0 = 0;
                    part.q1 = part.x.len ? (part.x.rows + kTile - 1) / kTile : 0;
                    // no more tiles than fit where they stay, nor than pass in a small part of a wait's limit
                    const int most = part.q1 > kStages<D> ? kTiles : kMostTiles;
                    if (part.x.n > most) {
                        part.x.n = most;
                        part.x.len = min(part.x.len, most * kTile);
                    }
                    const View v(b, part, kStages<D>);
                    auto idle = [&](int q) {
                        const View::Span s = v.span_of(q);
                        return s.first >= s.last;
                    };
                    while (part.q0 < part.q1 && idle(part.q0)) ++part.q0;
                    while (part.q1 > part.q0 && idle(part.q1 - 1)) --part.q1;
                    unit += part.x.n;
                }
                mbar_arrive(&ctl->seg_full[nth & 1]);
            }
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kIssueWarp) tmem_dealloc(tmem, 512);
}

template <int D>
cudaError_t launch(const WeighBatch& b, int blocks, cudaStream_t st) {
    static std::atomic<bool> set[64];     // (the attribute belongs to the device's function)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !set[dev]) {
        e = cudaFuncSetAttribute(k_weigh_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<D>());
        if (e != cudaSuccess) return e;
        if (dev < 64) set[dev] = true;
    }
    k_weigh_tc<D><<<blocks, kThreadsWt, smem_bytes<D>(), st>>>(b);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_weigh_tc(WeighBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    const int64_t units = attend_pairs(b, kWeighRows);
    const int blocks = (int)(units < num_sms ? units : num_sms);
    const cudaError_t e = head_dim == 128 ? launch<128>(b, blocks, st) : launch<64>(b, blocks, st);
    b.stall = 0;
    return e;
}

}  // namespace cbk
