// Rows of 4-bit caches that stay (cb_evict, cb_keep): which (k_rank), and their moving together (k_move).
#include <cooperative_groups.h>
#include <cstdint>
#include <cuda_runtime.h>

#include "cb_receiver.cuh"

namespace cbk {
namespace {
namespace cg = cooperative_groups;

__device__ __forceinline__ int64_t rows_of(int64_t T, const int32_t* length) {
    if (!length) return T;
    const int64_t l = __ldcg(length);
    return l < 0 ? 0 : l < T ? l : T;
}

// ---- which rows stay ----------------------------------------------------------------------------

constexpr int kRankThreads = 512;
constexpr int kBins = 2048;
constexpr int kRankPasses = 3;
constexpr int kRankKeys = 24 * 1024;         // keys of a block's slice held in shared memory at most (96 KB)
constexpr int kRankCluster = 8;

// Larger weights have larger keys; -0 is 0, NaN below all.
__device__ __forceinline__ uint32_t rank_key(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the block of a value a thread, and (before) those of the threads before this one.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t& before, uint32_t* sh) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t x = v;
#pragma unroll
    for (int k = 1; k < 32; k *= 2) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, k);
        if (lane >= k) x += y;
    }
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    uint32_t all = 0, mine = 0;
#pragma unroll
    for (int i = 0; i < kRankThreads / 32; ++i) {
        if (i == warp) mine = all;
        all += sh[i];
    }
    __syncthreads();
    before = mine + x - v;
    return all;
}

// A cluster of blocks ranks one list (cache, layer, KV head), a slice of its inner rows each: a radix select by 11, 11 and
// 10 bits from the top finds the key where the budget runs out (histograms joined in the first block's shared
// memory); rows above it stay, and of those at it the lowest.
template <int C>
__global__ void __launch_bounds__(kRankThreads) k_rank(const __grid_constant__ RankBatch b, uint32_t held) {
    extern __shared__ uint32_t keys[];                   // [held]
    __shared__ uint32_t own[kBins], all[C > 1 ? kRankPasses : 1][C > 1 ? kBins : 1];
    __shared__ uint32_t scan[kRankThreads / 32];
    __shared__ uint32_t found[3];                        // bin, keys above it, keys in it
    __shared__ uint32_t counts[2];                       // this block's keys above the last, and at it
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = C > 1 ? (int)cluster.block_rank() : 0;
    const int list = blockIdx.x / C, lists = b.n_layers * b.n_kv_heads;
    const RankSeq& s = b.s[blockIdx.y];
    const int64_t L = rows_of(s.T, s.length);
    int32_t* idx = s.idx + list * s.keep;
    if (list >= lists) return;
    if (L <= s.keep) {
        for (int64_t j = (int64_t)rank * kRankThreads + threadIdx.x; j < s.keep; j += C * kRankThreads)
            idx[j] = j < L ? (int32_t)j : -1;
        return;
    }
    for (int64_t j = (int64_t)rank * kRankThreads + threadIdx.x; j < s.first; j += C * kRankThreads) idx[j] = (int32_t)j;
    for (int64_t j = (int64_t)rank * kRankThreads + threadIdx.x; j < s.last; j += C * kRankThreads)
        idx[s.keep - s.last + j] = (int32_t)(L - s.last + j);
    const uint32_t want = (uint32_t)(s.keep - s.first - s.last);
    if (want == 0) return;
    const uint32_t n = (uint32_t)(L - s.first - s.last);
    const float* w = s.weights + (list / b.n_kv_heads) * s.w_layer + (list % b.n_kv_heads) * s.w_head + s.first;
    const uint32_t per = ((n + C - 1) / C + 3) & ~3u;
    const uint32_t lo = min(n, rank * per), len = min(n, lo + per) - lo;
    w += lo;
    auto key = [&](uint32_t i) { return i < held ? keys[i] : rank_key(__ldg(w + i)); };

    if (C > 1)
        for (int i = threadIdx.x; i < kRankPasses * kBins; i += kRankThreads) all[i / kBins][i % kBins] = 0;
#pragma unroll 8
    for (uint32_t i = threadIdx.x; i < min(len, held); i += kRankThreads) keys[i] = rank_key(__ldg(w + i));
    if (C > 1) cluster.sync();
    uint32_t need = want, prefix = 0, above = 0, equal = 0;      // above, equal: this block's
    int shift = 32;
#pragma unroll 1
    for (int pass = 0; pass < kRankPasses; ++pass) {
        const int bits = pass == 2 ? 10 : 11, up = shift;        // keys that match `prefix` in the bits from `up` on
        shift -= bits;
        for (int i = threadIdx.x; i < kBins; i += kRankThreads) own[i] = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < len; i += kRankThreads) {
            const uint32_t k = key(i);
            if (pass == 0 || k >> up == prefix) atomicAdd(&own[(k >> shift) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        uint32_t* joined = C > 1 ? cluster.map_shared_rank(all[C > 1 ? pass : 0], 0) : own;
        if (C > 1) {
            for (int i = threadIdx.x; i < kBins; i += kRankThreads)
                if (own[i]) atomicAdd(joined + i, own[i]);
            cluster.sync();
        }
        // bins from the top: thread t has bins 4 (511 - t) .. + 3
        const int bin0 = kBins - 4 - 4 * threadIdx.x;
        uint32_t c[4], before;
#pragma unroll
        for (int k = 0; k < 4; ++k) c[k] = joined[bin0 + 3 - k];
        block_scan(c[0] + c[1] + c[2] + c[3], before, scan);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (before < need && need <= before + c[k]) {
                found[0] = bin0 + 3 - k;
                found[1] = before;
                found[2] = c[k];
            }
            before += c[k];
        }
        __syncthreads();
        const uint32_t bin = found[0];
        uint32_t mine = 0, nothing;
#pragma unroll
        for (int k = 0; k < 4; ++k) mine += (uint32_t)(bin0 + 3 - k) > bin ? own[bin0 + 3 - k] : 0;
        above += block_scan(mine, nothing, scan);
        equal = own[bin];
        need -= found[1];
        prefix = prefix << bits | bin;
        const bool whole = found[2] == need;
        __syncthreads();
        if (whole) break;                                        // (all that share the bits so far)
    }
    // rows of keys above `prefix` in the bits from `shift` on stay, and the first `need` of those at it
    if (threadIdx.x == 0) {
        counts[0] = above;
        counts[1] = equal;
    }
    uint32_t above0 = 0, equal0 = 0;                             // of the blocks before
    if (C > 1) {
        cluster.sync();
        for (int r = 0; r < rank; ++r) {
            const uint32_t* o = cluster.map_shared_rank(counts, r);
            above0 += o[0];
            equal0 += o[1];
        }
        cluster.sync();                                          // (no block leaves while another reads its memory)
    }
    for (uint32_t i0 = 0; i0 < len; i0 += 4 * kRankThreads) {
        const uint32_t i = i0 + 4 * threadIdx.x;
        uint32_t v = 0, stays[4];                                // above in the low half, at it in the high half
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t x = i + k < len ? key(i + k) >> shift : 0;
            stays[k] = i + k >= len ? 0u : x > prefix ? 1u : x == prefix ? 0x10000u : 0u;
            v += stays[k];
        }
        uint32_t before;
        const uint32_t sum = block_scan(v, before, scan);
        uint32_t a = above0 + (before & 0xFFFFu), e = equal0 + (before >> 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (stays[k] == 1u || (stays[k] && e < need))
                idx[s.first + a + min(e, need)] = (int32_t)(s.first + lo + i + k);
            a += stays[k] & 0xFFFFu;
            e += stays[k] >> 16;
        }
        above0 += sum & 0xFFFFu;
        equal0 += sum >> 16;
    }
}

// ---- their moving ---------------------------------------------------------------------------------

constexpr uint32_t kNone = 0xFFFFFFFFu;

__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld8(const void* p) {
    uint2 v;
    asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld4(const void* p) {
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// Rows of a step of one group, as a thread holds them: pieces of codes, its own row's scales and weight.
template <int D>
struct Held {
    uint4 code[D / 32];
    uint2 scale;
    uint32_t weight;
};

// A group of threads moves the rows of K or of V of one list, a row a thread a step: GROUP = 32, a warp; else a block, or
// the blocks of a cluster together.  In place a row's source is never before its place, so what a step writes is
// read by no later one; within a step every group reads before any writes (a barrier), and the next step's rows are on
// their way by then.
template <int D, int GROUP>
__global__ void __launch_bounds__(256) k_move(const __grid_constant__ MoveBatch b, int blocks, int clustered) {
    constexpr int P = D / 32;                 // pieces of a row's codes
    constexpr int N = GROUP / P;              // rows that a piece a thread covers
    __shared__ uint2 where[2][256];           // rows of the cache: from, to
    const MoveSeq& s = b.s[blockIdx.z];
    const int lists = b.n_layers * b.n_kv_heads;
    const int t = threadIdx.x % GROUP;
    const int group = GROUP == 32 ? blockIdx.x * (256 / 32) + threadIdx.x / 32 : blockIdx.x;
    const int unit = group / blocks, part = group % blocks;
    // (of lists of their own, only the thread that writes the number of rows reads the length)
    const bool lists_own = s.drafted < 0, says = group == 0 && t == 0 && s.left && !s.left_later;
    const int64_t L = !lists_own || says ? rows_of(s.T, s.length) : 0;
    const int64_t base = lists_own ? 0 : L - s.drafted, limit = lists_own ? s.T : s.drafted;
    int64_t count = s.count;
    if (s.n_kept) count = max((int64_t)0, min((int64_t)*s.n_kept, count));
    if (base < 0) {
        if (group == 0 && t == 0) atomicOr(b.err, kErrPackRow);
        return;
    }
    if (says) *s.left = (int32_t)(lists_own ? min(L, count) : base + count);
    if (unit >= 2 * lists) return;            // (a whole group)
    const int kv = unit % 2, list = unit / 2, l = list / b.n_kv_heads, g = list % b.n_kv_heads;
    const int64_t from0 = l * s.from.s_layer + g * s.from.s_head, to0 = l * s.to.s_layer + g * s.to.s_head;
    const uint8_t* code = s.from.code[kv] + from0 * (D / 2) + t % P * 16;
    const uint8_t* scale = reinterpret_cast<const uint8_t*>(s.from.scale[kv]) + from0 * (D / 16);
    uint8_t* code_to = s.to.code[kv] + to0 * (D / 2) + t % P * 16;
    uint8_t* scale_to = reinterpret_cast<uint8_t*>(s.to.scale[kv]) + to0 * (D / 16);
    const bool weigh = kv == 0 && s.w;
    const float* w = weigh ? s.w + l * s.w_layer + g * s.w_head + base : nullptr;
    float* w_to = weigh ? s.w_to + l * s.t_layer + g * s.t_head + base : nullptr;
    const int32_t* idx = s.idx + list * s.idx_list;
    uint2* rows = where[0] + threadIdx.x / GROUP * GROUP;      // and 256 on

    // the row of the thread at step j0, looked up: its entry (-1: none)
    auto look_up = [&](int64_t j0, uint2* to) {
        const int64_t j = j0 + t;
        uint2 r = make_uint2(kNone, kNone);
        int64_t i = -1;
        if (j < count) {
            i = idx[j];
            if (lists_own && i == -1) {
            } else if (i < j || i >= limit) {
                atomicOr(b.err, kErrCompactIndex);
                i = -1;
            }
        }
        if (i >= 0 && (i != j || !s.in_place)) {
            const int64_t x = packed_row(s.from, base + i), y = packed_row(s.to, base + j);
            if (x < 0 || y < 0) {
                atomicOr(b.err, kErrPageIndex);
                i = -1;
            } else {
                r = make_uint2((uint32_t)x, (uint32_t)y);
            }
        } else {
            i = -1;
        }
        to[t] = r;
        return i;
    };
    auto meet = [&] {
        if (GROUP == 32) __syncwarp();
        else __syncthreads();
    };
    auto load = [&](const uint2* at, int64_t i, Held<D>& h) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const uint32_t r = at[t / P + k * N].x;
            if (r != kNone) h.code[k] = ld16(code + (uint64_t)r * (D / 2));
        }
        if (i >= 0) {
            const uint64_t off = (uint64_t)at[t].x * (D / 16);
            if (D == 128) h.scale = ld8(scale + off);
            else h.scale.x = ld4(scale + off);
            if (weigh) h.weight = ld4(w + i);
        }
    };
    const int64_t step = (int64_t)GROUP * blocks;
    int64_t j0 = (int64_t)part * GROUP;
    const int64_t steps = (count + step - 1) / step;      // (the same for all of a cluster)
    int64_t i = look_up(j0, rows);
    meet();
    Held<D> h;
    load(rows, i, h);
    for (int64_t n = 0; n < steps; ++n, j0 += step) {
        uint2* here = rows + (n & 1) * 256;
        uint2* next = rows + (~n & 1) * 256;
        const int64_t i1 = n + 1 < steps ? look_up(j0 + step, next) : -1;
        if (GROUP != 32 && clustered) cg::this_cluster().sync();
        else meet();
        Held<D> h1;
        if (n + 1 < steps) load(next, i1, h1);
#pragma unroll
        for (int k = 0; k < P; ++k) {
            const uint32_t r = here[t / P + k * N].y;
            if (r != kNone) *reinterpret_cast<uint4*>(code_to + (uint64_t)r * (D / 2)) = h.code[k];
        }
        if (i >= 0) {
            const uint64_t off = (uint64_t)here[t].y * (D / 16);
            if (D == 128) *reinterpret_cast<uint2*>(scale_to + off) = h.scale;
            else *reinterpret_cast<uint32_t*>(scale_to + off) = h.scale.x;
            if (weigh) reinterpret_cast<uint32_t*>(w_to)[j0 + t] = h.weight;
        }
        meet();                                            // (`here` is written again two steps on)
        i = i1;
        h = h1;
    }
}

// How many rows are left of the caches whose lengths k_move's groups read.
__global__ void k_left(const __grid_constant__ MoveBatch b) {
    const int i = threadIdx.x;
    if (i >= b.n || !b.s[i].left_later) return;
    const MoveSeq& s = b.s[i];
    const int64_t L = rows_of(s.T, s.length);
    int64_t count = s.count;
    if (s.n_kept) count = max((int64_t)0, min((int64_t)*s.n_kept, count));
    if (s.drafted < 0) *s.left = (int32_t)min(L, count);
    else if (L >= s.drafted) *s.left = (int32_t)(L - s.drafted + count);
}

template <int D>
cudaError_t launch(const MoveBatch& b, int64_t most, bool in_place, int num_sms, cudaStream_t st) {
    const int units = 2 * b.n_layers * b.n_kv_heads;
    if (!in_place || most <= 64) {
        // warps of a list: as many as fill the GPU, a step's rows each at least
        int64_t warps = 1;
        if (!in_place) {
            warps = 48 * (int64_t)num_sms / ((int64_t)units * b.n);
            if (warps > (most + 31) / 32) warps = (most + 31) / 32;
            if (warps < 1) warps = 1;
        }
        k_move<D, 32><<<dim3((unsigned)((units * warps + 7) / 8), 1, b.n), 256, 0, st>>>(b, (int)warps, 0);
        return cudaGetLastError();
    }
    // blocks of a list: as many as fill the GPU, a step's rows each at least
    int blocks = 1;
    while (blocks < 8 && (int64_t)units * b.n * blocks < 4 * num_sms && most > 256 * blocks) blocks *= 2;
    if (blocks == 1) {
        k_move<D, 256><<<dim3(units, 1, b.n), 256, 0, st>>>(b, 1, 0);
        return cudaGetLastError();
    }
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = blocks;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(units * blocks, 1, b.n);
    config.blockDim = dim3(256);
    config.stream = st;
    config.attrs = &cluster;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, k_move<D, 256>, b, blocks, 1);
}

template <int C>
cudaError_t launch_rank_by(const RankBatch& b, int64_t most, cudaStream_t st) {
    const cudaError_t e = cudaFuncSetAttribute(k_rank<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRankKeys * 4);
    if (e != cudaSuccess) return e;
    const int64_t slice = (most + C - 1) / C + 4;
    const uint32_t held = (uint32_t)(slice < kRankKeys ? slice : kRankKeys);
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = C;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(b.n_layers * b.n_kv_heads * C, b.n);
    config.blockDim = dim3(kRankThreads);
    config.dynamicSmemBytes = held * 4;
    config.stream = st;
    config.attrs = &cluster;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, k_rank<C>, b, held);
}

}  // namespace

cudaError_t launch_rank(const RankBatch& b, cudaStream_t st, int num_sms) {
    int64_t most = 0;
    for (int i = 0; i < b.n; ++i) most = b.s[i].T > most ? b.s[i].T : most;
    // blocks of a list: as many as hold it, and while the lists leave SMs idle
    const int64_t lists = (int64_t)b.n * b.n_layers * b.n_kv_heads;
    int c = 1;
    while (c < kRankCluster && (most > (int64_t)c * kRankKeys || (2 * lists * c <= num_sms && most > 2048 * c))) c *= 2;
    return c == 1 ? launch_rank_by<1>(b, most, st) : c == 2 ? launch_rank_by<2>(b, most, st)
         : c == 4 ? launch_rank_by<4>(b, most, st) : launch_rank_by<8>(b, most, st);
}

cudaError_t launch_move(const MoveBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    int64_t most = 0;
    bool in_place = false;
    for (int i = 0; i < b.n; ++i) {
        most = b.s[i].count > most ? b.s[i].count : most;
        in_place |= b.s[i].in_place != 0;
    }
    bool left = false;
    for (int i = 0; i < b.n; ++i) left |= b.s[i].left && !b.s[i].left_later;
    if (most == 0 && !left) return cudaSuccess;
    return head_dim == 128 ? launch<128>(b, most, in_place, num_sms, st) : launch<64>(b, most, in_place, num_sms, st);
}

cudaError_t launch_left(const MoveBatch& b, cudaStream_t st) {
    static_assert(kMaxPackBatch == 32, "a warp");
    for (int i = 0; i < b.n; ++i)
        if (b.s[i].left_later) {
            k_left<<<1, kMaxPackBatch, 0, st>>>(b);
            return cudaGetLastError();
        }
    return cudaSuccess;
}

}  // namespace cbk
