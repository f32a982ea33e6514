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
// A row whose lse is not finite is a row of zeros with an lse of infinity: it adds nothing.
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
static_assert(kLse >= 4 + kBuffers + 2, "");

struct Ctl {
    uint64_t k_full[kTiles], k_empty[kTiles], q_full[4], q_empty[4];
    uint64_t d_full[kBuffers], d_empty[kBuffers], sum_full[kTiles], sum_empty[kTiles];
    uint64_t seg_full[2], seg_empty[2];
    uint64_t done, stall;
    uint64_t wait_ns;
    uint32_t tmem;
    int abort;
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
    // Some token of first .. last sees one of the n positions from t0 on.
    __device__ __forceinline__ bool see(int first, int last, int t0, int n) const {
        return w.tree || !w.causal || (t0 <= w.at + last && !(w.window && t0 + n - 1 <= w.at + first - w.window));
    }
    // Tile q of rows and tile k of positions have something to add; tile k has with some tile of rows.
    __device__ __forceinline__ bool met(int q, int k) const { return see(first_token(q), last_token(q), k * kTile, kTile); }
    __device__ __forceinline__ bool used(int k) const { return q0 < q1 && see(first_token(q0), last_token(q1 - 1), k * kTile, kTile); }
};

// Copies 16 bytes into shared memory, or zeros.
__device__ __forceinline__ void copy16_or_0(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}

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
        uint32_t item = 0, n_q = 0, n_tile = 0;
        bool ok = true;
        while (ok && begin()) {
            const Part& part = parts[nth & 1];
            const View v(b, part, kStages<D>);
            const TreeBits tree = b.w[part.x.seq].tree;
            // bit e: query row row0 + e sees the thread's position of tile k
            auto sees = [&](int q, int k, int row0) {
                const int t = k * kTile + mine;
                if (v.w.tree) {
                    if ((k + 1) * kTile <= v.w.at) return 0xFFFFFFFFu;
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
                const bool edge = v.w.causal && ((k + 1) * kTile - 1 > v.w.at + v.first_token(q) ||
                                                 (v.w.window && k * kTile <= v.w.at + v.last_token(q) - v.w.window));
                if (!edge) return 0xFFFFFFFFu;
                // tokens from t - at on, and before t - at + window
                const int64_t lo = ((int64_t)(t - v.w.at) << v.log2g) - row0;
                const int64_t hi = v.w.window ? lo + ((int64_t)v.w.window << v.log2g) : 32;
                const int c0 = (int)max((int64_t)0, min(lo, (int64_t)32)), c1 = (int)max((int64_t)0, min(hi, (int64_t)32));
                return c0 >= c1 ? 0u : (0xFFFFFFFFu << c0) & (0xFFFFFFFFu >> (32 - c1));
            };
            // the sum of the thread's columns of one product
            auto gather = [&](int q, int k) {
                const uint32_t d = item % kBuffers, phase = item / kBuffers & 1;
                ++item;
                if (!(ok = wait_warp(&ctl->d_full[d], phase, ctl, b.err, 10))) return 0.f;
                const int row0 = q * kTile + 32 * group;
                float sum = 0.f;
                if (row0 < v.rows) {
                    const uint32_t bits = sees(q, k, row0);
                    tc_fence_after();
                    float z[32];
                    tmem_ld32(from + d * 128, z);
                    tmem_wait_ld(z);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl->d_empty[d]);
                    if (bits != 0xFFFFFFFFu) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(bits >> e & 1u)) z[e] = -INFINITY;
                    }
                    const float* lse = s_lse + (n_q + q - v.q0) % kLse * kTile + 32 * group;
                    uint64_t l0 = 0, l1 = 0;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 nl = *reinterpret_cast<const float4*>(lse + e);
                        float y0, y1, y2, y3;
                        unpack2(ffma2(pack2(z[e], z[e + 1]), cc, pack2(nl.x, nl.y)), y0, y1);
                        unpack2(ffma2(pack2(z[e + 2], z[e + 3]), cc, pack2(nl.z, nl.w)), y2, y3);
                        l0 = fadd2(l0, pack2(ex2(y0), ex2(y1)));
                        l1 = fadd2(l1, pack2(ex2(y2), ex2(y3)));
                    }
                    float a0, a1;
                    unpack2(fadd2(l0, l1), a0, a1);
                    sum = a0 + a1;
                } else {
                    if (lane == 0) mbar_arrive(&ctl->d_empty[d]);
                }
                return sum;
            };
            auto place = [&](int k) { return s_sum + ((n_tile + k) % kTiles * kGroups + group) * kTile + mine; };
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
            if (v.resident) {
                for (int k = 0; k < v.tiles && open(k); ++k) {
                    float sum = 0.f;
                    for (int q = v.q0; q < v.q1 && ok; ++q)
                        if (v.met(q, k)) sum += gather(q, k);
                    *place(k) = sum;
                    close(k);
                }
            } else {
                for (int k = 0; k < v.tiles && open(k); ++k) *place(k) = 0.f;
                for (int q = v.q0; q < v.q1 && ok; ++q)
                    for (int k = 0; k < v.tiles && ok; ++k)
                        if (v.met(q, k)) *place(k) += gather(q, k);
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
        // query rows: thread u has piece u % P of rows u / P, u / P + N ...
        constexpr int P = D / 8, N = kLoadThreads / P, R = kTile / N;
        const int u = threadIdx.x - kSumWarps * 32;
        uint32_t n_q = 0, n_k = 0, bad = 0;
        bool ok = true;
        while (ok && begin()) {
            const Part& part = parts[nth & 1];
            const Segment& x = part.x;
            const View v(b, part, kStages<D>);
            const AttendSeq& s = b.s[x.seq];
            const float* lses = b.w[x.seq].lse;
            auto page_of = [&](int k, uint32_t (&page)[2]) {
#pragma unroll
                for (int y = 0; y < 2; ++y) page[y] = segment_page(x, k * kTile + 16 * lw + 8 * y + lane % 8);
            };
            auto read_keys = [&](int k, const uint32_t (&page)[2], Codes<D>& c) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    c.x[y] = make_uint4(0, 0, 0, 0);
                    c.scale[y] = 0;
                    const int r = segment_row(x, k * kTile + 16 * lw + 8 * y + lane % 8, page[y], b.err);
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
            auto lse_of = [&](int q, float (&lse)[R]) {
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const int row = q * kTile + u / P + i * N;
                    lse[i] = INFINITY;
                    if (row < v.rows)
                        lse[i] = __ldg(lses + (int64_t)(row >> v.log2g) * b.n_q_heads + (x.g << v.log2g) + (row & (b.G - 1)));
                }
            };
            auto copy_rows = [&](int q, const float (&lse)[R]) {       // into a stage that the products have left
                const uint32_t n = n_q + q - v.q0;
                if (n >= (uint32_t)kStages<D> && !wait_warp(&ctl->q_empty[n % kStages<D>], (n / kStages<D> - 1) & 1, ctl, b.err, 12)) {
                    ok = false;
                    return;
                }
                const uint32_t to = smem_u32(sq) + n % kStages<D> * kOp;
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const int r = u / P + i * N, row = q * kTile + r;
                    const bool there = isfinite(lse[i]);
                    copy16_or_0(to + piece(u % P / 8, kTile, r, u % P % 8),
                                there ? s.q + (int64_t)(row >> v.log2g) * s.s_tok +
                                            (int64_t)((x.g << v.log2g) + (row & (b.G - 1))) * s.s_head + u % P * 8
                                      : s.q,
                                there);
                    if (u % P == 0) s_lse[n % kLse * kTile + r] = there ? lse[i] * -1.4426950408889634f : -INFINITY;
                }
            };
            auto landed = [&](int q) {
                copy_commit();
                copy_wait<0>();
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->q_full[(n_q + q - v.q0) % kStages<D>]);
            };
            // tiles of positions that are used: k, and the next one on its way
            auto next = [&](int k) {
                do ++k;
                while (k < v.tiles && !v.used(k));
                return k;
            };
            Codes<D> c0, c1;
            uint32_t page[2];
            int k0 = next(-1), k1 = next(k0), k2 = next(k1);
            page_of(k0, page);
            read_keys(k0, page, c0);
            page_of(k1, page);
            read_keys(k1, page, c1);
            page_of(k2, page);
            float lse[R];
            const int q_first = min(v.q1, v.q0 + kStages<D>);           // the rows that stay, or the first that pass
            for (int q = v.q0; q < q_first && ok; ++q) {
                lse_of(q, lse);
                copy_rows(q, lse);
                if (ok) landed(q);
            }
            while (k0 < v.tiles && ok) {
                const uint32_t slot = n_k % kTiles;
                if (n_k >= kTiles && !(ok = wait_warp(&ctl->k_empty[slot], (n_k / kTiles - 1) & 1, ctl, b.err, 13))) break;
                ++n_k;
                uint8_t* to = sk + slot * kOp + at;
#pragma unroll
                for (int y = 0; y < 2; ++y, to += 8 * 128) {
                    const uint32_t s2 = checked_scale(c0.scale[y], bad) * 0x10001u;
                    const uint32_t word[4] = {c0.x[y].x, c0.x[y].y, c0.x[y].z, c0.x[y].w};
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) {
                        uint32_t w[4];
                        values_bf16(word[e], s2, w);
                        st_piece(to, col ^ (e << 4), w);
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->k_full[slot]);
                c0 = c1;
                k0 = k1;
                k1 = k2;
                read_keys(k1, page, c1);
                k2 = next(k2);
                page_of(k2, page);
            }
            lse_of(min(q_first, max(v.q1 - 1, 0)), lse);
            for (int q = q_first; q < v.q1 && ok; ++q) {
                copy_rows(q, lse);
                lse_of(min(q + 1, v.q1 - 1), lse);
                if (ok) landed(q);
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
        uint32_t item = 0, n_q = 0, n_k = 0;
        bool ok = !b.stall || blockIdx.x || wait_warp(&ctl->stall, 0, ctl, b.err, 14);
        while (ok && begin()) {
            const View v(b, parts[nth & 1], kStages<D>);
            uint32_t n_used = 0;
            if (lane == 0) {
                auto q_there = [&](int q) {
                    const uint32_t n = n_q + q - v.q0;
                    return wait(&ctl->q_full[n % kStages<D>], n / kStages<D> & 1, ctl, b.err, 14);
                };
                auto k_there = [&](uint32_t n) { return wait(&ctl->k_full[n % kTiles], n / kTiles & 1, ctl, b.err, 15); };
                auto product = [&](int q, uint32_t nk) {
                    const uint32_t d = item % kBuffers;
                    if (item >= kBuffers && !wait(&ctl->d_empty[d], (item / kBuffers - 1) & 1, ctl, b.err, 16)) return false;
                    tc_fence_after();
                    const uint32_t idesc = idesc_bf16_f32(kTile, (min(kTile, v.rows - q * kTile) + 31) & ~31);   // (what the sums read)
                    const uint32_t ka = kd + nk % kTiles * (kOp >> 4), qa = qd + (n_q + q - v.q0) % kStages<D> * (kOp >> 4);
#pragma unroll
                    for (int y = 0; y < D / 16; ++y) {
                        const uint32_t off = (y / 4) * (kTile * 128 >> 4) + (y % 4) * 2;
                        umma_bf16(tmem + d * 128, desc(ka + off, hi), desc(qa + off, hi), idesc, y > 0);
                    }
                    umma_commit(&ctl->d_full[d]);
                    ++item;
                    return true;
                };
                if (v.resident) {
                    bool first = true;
                    for (int k = 0; k < v.tiles && ok; ++k) {
                        if (!v.used(k)) continue;
                        if (first)
                            for (int q = v.q0; q < v.q1 && ok; ++q) ok = q_there(q);
                        first = false;
                        const uint32_t n = n_k + n_used;
                        if (!ok || !(ok = k_there(n))) break;
                        for (int q = v.q0; q < v.q1 && ok; ++q)
                            if (v.met(q, k)) ok = product(q, n);
                        umma_commit(&ctl->k_empty[n % kTiles]);
                        ++n_used;
                    }
                    for (int q = v.q0; q < v.q1; ++q) umma_commit(&ctl->q_empty[(n_q + q - v.q0) % kStages<D>]);
                } else {
                    uint32_t there = 0;
                    for (int k = 0; k < v.tiles; ++k) n_used += v.used(k);
                    for (int q = v.q0; q < v.q1 && ok; ++q) {
                        if (!(ok = q_there(q))) break;
                        uint32_t n = n_k;
                        for (int k = 0; k < v.tiles && ok; ++k) {
                            if (!v.used(k)) continue;
                            if (v.met(q, k)) {
                                if (!(there >> k & 1)) ok = k_there(n);
                                there |= 1u << k;
                                if (ok) ok = product(q, n);
                            }
                            ++n;
                        }
                        umma_commit(&ctl->q_empty[(n_q + q - v.q0) % kStages<D>]);
                    }
                    for (uint32_t n = 0; n < n_used; ++n) umma_commit(&ctl->k_empty[(n_k + n) % kTiles]);
                }
            }
            ok = __shfl_sync(0xFFFFFFFFu, (int)ok, 0);
            n_k += n_used;                          // (lane 0's; it alone uses them)
            n_q += v.q1 - v.q0;
            finish();
        }
        if (lane == 0) {
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
                if (!(ok = wait_warp(&ctl->sum_full[n_tile % kTiles], n_tile / kTiles & 1, ctl, b.err, 17))) break;
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
                if (nth >= 2 && !wait(&ctl->seg_empty[nth & 1], (nth / 2 - 1) & 1, ctl, b.err, 18)) break;
                more = unit < end;
                part.x.n = 0;
                if (more) {
                    attend_segment(b, pre, b.n_kv_heads, 0, unit, end, D, kWeighRows, &part.x);
                    part.q0 = 0;
                    part.q1 = part.x.len ? (part.x.rows + kTile - 1) / kTile : 0;
                    if (part.q1 > kStages<D> && part.x.n > kTiles) {            // the positions stay: no more than fit
                        part.x.n = kTiles;
                        part.x.len = min(part.x.len, kTiles * kTile);
                    }
                    const View v(b, part, kStages<D>);
                    while (part.q0 < part.q1 && !v.see(v.first_token(part.q0), v.last_token(part.q0), 0, part.x.len)) ++part.q0;
                    while (part.q1 > part.q0 && !v.see(v.first_token(part.q1 - 1), v.last_token(part.q1 - 1), 0, part.x.len)) --part.q1;
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
