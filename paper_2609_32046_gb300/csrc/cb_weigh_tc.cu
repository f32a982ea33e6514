// Attention weights gathered from many query rows a KV head: tcgen05 (cb_weigh).
//
// A block takes up to kTiles tiles of 128 positions of one KV head at a time, unpacks their keys into shared memory once and
// walks all the query rows (token, head of the group) past them, 128 at a time:
//   D [128 positions][128 query rows] = K Q^T        (bf16; fp32 in tensor memory, four buffers)
//   w[position] += sum over the columns of exp2(scale * log2(e) * D - lse * log2(e))
// A thread owns a position, so nothing is exchanged between threads but the halves of the columns.  17 warps:
//   0..7    sums: four warps a group (TMEM lane quarter = warp % 4), a group takes every other 32 columns
//   8..15   keys, unpacked as bf16 (K-major, 128-byte swizzle); then query rows, copied beside the products
//   16      issues tcgen05.mma
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
constexpr int kSumWarps = 8, kLoadWarps = 8, kWarpsWt = kSumWarps + kLoadWarps + 1;
constexpr int kThreadsWt = kWarpsWt * 32;
constexpr int kLoadThreads = kLoadWarps * 32;
constexpr int kBuffers = 4;                 // of 128 columns of tensor memory
template <int D> constexpr int kTiles = 4;                    // tiles of positions at a time
template <int D> constexpr int kStages = D == 128 ? 2 : 4;    // tiles of query rows in shared memory
constexpr int kLse = 8;                     // tiles of their log-sum-exps: the products are up to kStages tiles of rows and
                                            // kBuffers buffers ahead of the sums, which read them

struct Ctl {
    uint64_t k_full[4], q_full[4], q_empty[4];
    uint64_t d_full[kBuffers], d_empty[kBuffers];
    uint64_t done, stall;
    uint64_t wait_ns;
    uint32_t tmem;
    int abort;
    int unit, run1;                         // the run: its next unit, its end
    int q0, q1;                             // tiles of query rows that see something of the segment
};
constexpr int kCtlBytes = 1024;
static_assert(sizeof(Ctl) <= 512, "");

template <int D>
constexpr int smem_bytes() {
    return (kTiles<D> + kStages<D>)*kTile * D * 2 + kLse * kTile * 4 + 2 * kTiles<D> * kTile * 4 + kCtlBytes + 1024;
}

// Whether a tile of query rows (the q-th) and one of positions (from t0 on) have anything to add.
__device__ __forceinline__ bool met(const WeighRows& w, int q, int rows, int t0) {
    if (w.tree || !w.causal) return true;
    const int first = q * kTile / w.G, last = (min(rows, (q + 1) * kTile) - 1) / w.G;
    return t0 <= w.at + last && !(w.window && t0 + kTile - 1 <= w.at + first - w.window);
}

// Copies 16 bytes into shared memory, or zeros.
__device__ __forceinline__ void copy16_or_0(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}

template <int D>
__global__ void __launch_bounds__(kThreadsWt, 1) k_weigh_tc(const __grid_constant__ WeighBatch b) {
    constexpr int kOp = kTile * D * 2;              // bytes of an operand tile
    extern __shared__ uint8_t raw[];
    __shared__ Segment seg;
    __shared__ int pre[kMaxBatch + 1];
    Ctl* ctl = reinterpret_cast<Ctl*>(raw);
    uint8_t* sk = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + kCtlBytes + 1023) & ~uintptr_t(1023));
    uint8_t* sq = sk + kTiles<D> * kOp;
    float* s_lse = reinterpret_cast<float*>(sq + kStages<D> * kOp);      // [tile of rows % kLse][row]: -lse * log2(e)
    float* s_sum = s_lse + kLse * kTile;                            // [group][tile][position]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    attend_units(b, kWeighRows, pre);
    if (threadIdx.x == 0) {
        const Runs runs = attend_runs(pre[b.pairs] * b.n_kv_heads, gridDim.x);
        const int at = min((int)blockIdx.x, runs.blocks);
        ctl->unit = attend_run(runs, at);
        ctl->run1 = attend_run(runs, min(at + 1, runs.blocks));
        for (int i = 0; i < 4; ++i) {
            mbar_init(&ctl->k_full[i], 4);
            mbar_init(&ctl->q_full[i], kLoadWarps);
            mbar_init(&ctl->q_empty[i], 1);
        }
        for (int i = 0; i < kBuffers; ++i) {
            mbar_init(&ctl->d_full[i], 1);
            mbar_init(&ctl->d_empty[i], kSumWarps);
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
    const uint32_t tmem = ctl->tmem;

    // Every role walks the run's segments by itself; all of the block meets at a segment's beginning and end.
    uint32_t n_seg = 0, n_item = 0, n_q = 0, n_k = 0;      // segments, products, tiles of rows; bit k: parity of k_full[k]
    while (ctl->unit < ctl->run1 && !*reinterpret_cast<volatile int*>(&ctl->abort)) {
        if (threadIdx.x == 0) {
            attend_segment(b, pre, b.n_kv_heads, 0, ctl->unit, min(ctl->run1, ctl->unit + kTiles<D>), D, kWeighRows, &seg);
            // (what is met of a tile of positions is a run of tiles of rows, and neighbours' runs touch: none between is idle)
            const WeighRows w(b, seg);
            const int nk = (seg.len + kTile - 1) / kTile, nq = (seg.rows + kTile - 1) / kTile;
            int q0 = 0, q1 = nk ? nq : 0;
            auto any = [&](int q) {
                for (int k = 0; k < nk; ++k)
                    if (met(w, q, seg.rows, k * kTile)) return true;
                return false;
            };
            while (q0 < q1 && !any(q0)) ++q0;
            while (q1 > q0 && !any(q1 - 1)) --q1;
            ctl->q0 = q0;
            ctl->q1 = q1;
        }
        __syncthreads();
        const WeighRows w(b, seg);
        const WeighSeq& ws = b.w[seg.seq];
        const int first = ctl->q0, last = ctl->q1;      // tiles of rows
        const int nk = first < last ? (seg.len + kTile - 1) / kTile : 0;

        if (warp == 16) {
            // ---------------- products ----------------
            if (elect_one()) {
                const uint32_t hi = (uint32_t)(smem_desc_sw128(0) >> 32), lo = (uint32_t)smem_desc_sw128(0);
                const uint32_t k0 = (smem_u32(sk) >> 4) + lo, q0 = (smem_u32(sq) >> 4) + lo;
                bool ok = !b.stall || blockIdx.x || wait(&ctl->stall, 0, ctl, b.err, 9);
                uint32_t seen = 0, item = n_item;
                for (int q = first; q < last && ok; ++q) {
                    const uint32_t nth = n_q + q - first;
                    if (!(ok = wait(&ctl->q_full[nth % kStages<D>], nth / kStages<D> & 1, ctl, b.err, 10))) break;
                    const int columns = (min(kTile, seg.rows - q * kTile) + 31) & ~31;      // (as many as the sums read)
                    const uint32_t idesc = idesc_bf16_f32(kTile, columns), qd = q0 + nth % kStages<D> * (kOp >> 4);
                    for (int k = 0; k < nk && ok; ++k) {
                        if (!met(w, q, seg.rows, k * kTile)) continue;
                        if (!(seen >> k & 1)) {
                            if (!(ok = wait(&ctl->k_full[k], n_k >> k & 1, ctl, b.err, 11))) break;
                            seen |= 1u << k;
                        }
                        const uint32_t d = item % kBuffers;
                        if (item >= kBuffers && !(ok = wait(&ctl->d_empty[d], (item / kBuffers - 1) & 1, ctl, b.err, 12))) break;
                        tc_fence_after();
                        const uint32_t kd = k0 + k * (kOp >> 4);
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            const uint32_t off = (x / 4) * (kTile * 128 >> 4) + (x % 4) * 2;
                            umma_bf16(tmem + d * 128, desc(kd + off, hi), desc(qd + off, hi), idesc, x > 0);
                        }
                        umma_commit(&ctl->d_full[d]);
                        ++item;
                    }
                    if (ok) umma_commit(&ctl->q_empty[nth % kStages<D>]);
                }
                // (a tile that no row met was unpacked all the same)
                for (int k = 0; k < nk && ok; ++k)
                    if (!(seen >> k & 1)) ok = wait(&ctl->k_full[k], n_k >> k & 1, ctl, b.err, 11);
                umma_commit(&ctl->done);
                drain(&ctl->done, n_seg & 1);
            }
            __syncwarp();
        } else if (warp >= kSumWarps) {
            // ---------------- keys, then query rows ----------------
            const int lw = warp - kSumWarps, g4 = lw / 4, w4 = lw % 4, quarter = lane / 8;
            const uint32_t at = piece(quarter * (D / 32) / 8, kTile, 32 * w4, 0) + (lane % 8) * 128;
            const uint32_t col = ((quarter * (D / 32) % 8) ^ (lane % 8)) << 4;
            // tiles g4, g4 + 2: rows 32 w4 + 8 y + lane % 8, the quarter of each, all read ahead
            uint4 x[kTiles<D> / 2][4];
            uint32_t sc[kTiles<D> / 2][4];
#pragma unroll
            for (int i = 0; i < kTiles<D> / 2; ++i)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int t = (g4 + 2 * i) * kTile + 32 * w4 + 8 * y + lane % 8;
                    x[i][y] = make_uint4(0, 0, 0, 0);
                    sc[i][y] = 0;
                    const int r = segment_row(seg, t, segment_page(seg, t), b.err);
                    if (r < 0) continue;
                    const uint8_t* c = seg.code[0] + (uint64_t)r * (D / 2) + quarter * (D / 8);
                    if (D == 128) {
                        x[i][y] = __ldg(reinterpret_cast<const uint4*>(c));
                    } else {
                        const uint2 v = __ldg(reinterpret_cast<const uint2*>(c));
                        x[i][y].x = v.x;
                        x[i][y].y = v.y;
                    }
                    sc[i][y] = __ldg(seg.scale[0] + (uint64_t)r * (D / 32) + quarter * (D / 32) / 4);
                }
            // query rows: thread u has piece u % (D / 8) of rows u / (D / 8), + 256 / (D / 8) ...
            constexpr int P = D / 8, N = kLoadThreads / P;
            const int u = threadIdx.x - kSumWarps * 32;
            const AttendSeq& s = b.s[seg.seq];
            auto copy_rows = [&](int q, uint32_t nth) {
                const uint32_t to = smem_u32(sq) + nth % kStages<D> * kOp;
#pragma unroll
                for (int i = 0; i < kTile / N; ++i) {
                    const int r = u / P + i * N, row = q * kTile + r;
                    bool there = row < seg.rows;
                    const int token = row / b.G, head = seg.g * b.G + row % b.G;
                    float lse = INFINITY;
                    if (there) lse = __ldg(ws.lse + (int64_t)token * b.n_q_heads + head);
                    there = there && isfinite(lse);
                    copy16_or_0(to + piece(u % P / 8, kTile, r, u % P % 8),
                                there ? s.q + (int64_t)token * s.s_tok + (int64_t)head * s.s_head + u % P * 8 : s.q, there);
                    if (u % P == 0) s_lse[nth % kLse * kTile + r] = there ? lse * -1.4426950408889634f : -INFINITY;
                }
                copy_commit();
            };
            bool ok = true;
            int copied = first;                      // tiles of rows before this one are on their way or there
            auto more_rows = [&]() {                 // one more, into a stage that the products have left
                const uint32_t nth = n_q + copied - first;
                if (nth >= (uint32_t)kStages<D> &&
                    !(ok = wait_warp(&ctl->q_empty[nth % kStages<D>], (nth / kStages<D> - 1) & 1, ctl, b.err, 13)))
                    return;
                copy_rows(copied, nth);
                ++copied;
            };
            auto landed = [&](int q) {
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->q_full[(n_q + q - first) % kStages<D>]);
            };
            if (first < last) more_rows();
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < kTiles<D> / 2; ++i) {
                const int k = g4 + 2 * i;
                if (k >= nk) break;
                uint8_t* to = sk + k * kOp + at;
#pragma unroll
                for (int y = 0; y < 4; ++y, to += 8 * 128) {
                    const uint32_t s2 = checked_scale(sc[i][y], bad) * 0x10001u;
                    const uint32_t word[4] = {x[i][y].x, x[i][y].y, x[i][y].z, x[i][y].w};
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) {
                        uint32_t v[4];
                        values_bf16(word[e], s2, v);
                        st_piece(to, col ^ (e << 4), v);
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->k_full[k]);
            }
            if (bad) atomicOr(b.err, kErrPackScale);
            for (int q = first; q < last && ok; ++q) {
                while (copied < last && copied - q < kStages<D> - 1 && ok) more_rows();
                if (!ok) break;
                if (copied - q > 1) {
                    // (the oldest group of those in flight)
                    if (copied - q == 2) copy_wait<1>();
                    else copy_wait<2>();
                } else {
                    copy_wait<0>();
                }
                landed(q);
                if (kStages<D> <= 2 && copied < last) more_rows();
            }
            copy_wait<0>();
        } else {
            // ---------------- sums ----------------
            const int group = warp >> 2, mine = (warp & 3) * 32 + lane;
            const uint32_t lanes = (uint32_t)(warp & 3) << 21;               // 32 (warp % 4) << 16
            float* sums = s_sum + group * kTiles<D> * kTile + mine;
            const int tiles = (seg.len + kTile - 1) / kTile;
            for (int k = 0; k < tiles; ++k) sums[k * kTile] = 0.f;
            uint32_t item = n_item;
            bool ok = true;
            const uint64_t cc = pack2(b.scale_log2e, b.scale_log2e);
            for (int q = first; q < last && ok; ++q) {
                const int columns = min(kTile, seg.rows - q * kTile);
                const float* lse = s_lse + (n_q + q - first) % kLse * kTile;
                for (int k = 0; k < nk; ++k) {
                    if (!met(w, q, seg.rows, k * kTile)) continue;
                    const uint32_t d = item % kBuffers;
                    if (!(ok = wait_warp(&ctl->d_full[d], item / kBuffers & 1, ctl, b.err, 14))) break;
                    tc_fence_after();
                    const int token0 = q * kTile / b.G, t = k * kTile + mine;
                    const bool edge = w.tree ? (k + 1) * kTile > w.at
                                             : w.causal && ((k + 1) * kTile - 1 > w.at + token0 ||
                                                            (w.window && k * kTile <= w.at + (q * kTile + columns - 1) / b.G - w.window));
                    uint64_t l0 = 0, l1 = 0;
#pragma unroll 1
                    for (int c = 32 * group; c < columns; c += 64) {
                        float z[32];
                        tmem_ld32(tmem + lanes + d * 128 + c, z);
                        tmem_wait_ld(z);
                        if (edge) {
                            if (w.tree) {
                                uint32_t bits = 0;
#pragma unroll
                                for (int e = 0; e < 32; ++e) {
                                    const int row = q * kTile + c + e;
                                    if (row % b.G == 0)
                                        bits = tree_bits(ws.tree.seen + min(row / b.G, w.m - 1) * ws.tree.s_row, (w.m + 31) / 32,
                                                         t - lane - w.at);
                                    if (!(bits >> lane & 1u)) z[e] = -INFINITY;
                                }
                            } else {
                                // tokens from t - at on, and before t - at + window, see the position
                                const int64_t c0 = (t - w.at) * b.G - (q * kTile + c);
                                const int64_t c1 = w.window ? c0 + w.window * b.G : 32;
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (e < c0 || e >= c1) z[e] = -INFINITY;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 nl = *reinterpret_cast<const float4*>(lse + c + e);
                            float y0, y1, y2, y3;
                            unpack2(ffma2(pack2(z[e], z[e + 1]), cc, pack2(nl.x, nl.y)), y0, y1);
                            unpack2(ffma2(pack2(z[e + 2], z[e + 3]), cc, pack2(nl.z, nl.w)), y2, y3);
                            l0 = fadd2(l0, pack2(ex2(y0), ex2(y1)));
                            l1 = fadd2(l1, pack2(ex2(y2), ex2(y3)));
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl->d_empty[d]);
                    float a0, a1;
                    unpack2(fadd2(l0, l1), a0, a1);
                    sums[k * kTile] += a0 + a1;
                    ++item;
                }
            }
            // (all eight warps come here, whatever they saw)
            asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
            for (int k = group; k < tiles; k += 2) {
                const int t = k * kTile + mine;
                if (t >= seg.len) continue;
                const float sum = s_sum[k * kTile + mine] + s_sum[(kTiles<D> + k) * kTile + mine];
                ws.weights[(int64_t)seg.g * ws.w_head + seg.begin + t] = fmaf(b.decay, w.before(ws, seg.g, t), sum);
            }
        }
        for (int q = first; q < last; ++q)
            for (int k = 0; k < nk; ++k) n_item += met(w, q, seg.rows, k * kTile);
        n_q += last - first;
        n_k ^= (1u << nk) - 1;
        ++n_seg;
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (threadIdx.x == 0) ctl->unit += seg.n;
        __syncthreads();
    }
    __syncthreads();
    if (warp == 16) tmem_dealloc(tmem, 512);
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
