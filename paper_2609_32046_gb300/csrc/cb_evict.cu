// Rows of 4-bit caches that stay (cb_evict, cb_keep): which (k_rank), and their moving together (k_move).
#include <atomic>
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

constexpr int kRankThreads = 1024, kRankWarps = kRankThreads / 32;
constexpr int kBins = 2048;
constexpr int kRankPasses = 3;

// Larger weights have larger keys; -0 is 0, NaN below all.
__device__ __forceinline__ uint32_t rank_key(float w) {
    const uint32_t u = __float_as_uint(w + 0.f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the warps before this one of a number each warp has, and over all.
__device__ __forceinline__ uint32_t warps_before(uint32_t mine, uint32_t& all, uint32_t* sh) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) sh[warp] = mine;
    __syncthreads();
    const uint32_t w = sh[lane];                         // (as many warps as lanes)
    all = __reduce_add_sync(0xFFFFFFFFu, w);
    const uint32_t before = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? w : 0u);
    __syncthreads();
    return before;
}
static_assert(kRankWarps == 32 && kBins == 2 * kRankThreads, "");

// A cluster of blocks ranks one list (cache, layer, KV head), a slice of its inner rows each: a radix select by 11, 11 and
// 10 bits from the top finds the key where the budget runs out (histograms joined in the first block's shared
// memory); rows above it stay, and of those at it the lowest.  288 lists of 16384 rows, a block each, 20 us: loads (4), counting in
// shared memory, whose adds to a few bins of like exponents queue, and barriers of 1024 threads; with every warp scanning every
// count 25, with 512 threads and a scan for each 2048 keys 31.  HELD: no slice has more keys than shared memory holds.
template <int C, bool HELD>
__global__ void __launch_bounds__(kRankThreads) k_rank(const __grid_constant__ RankBatch b, uint32_t held) {
    extern __shared__ uint32_t keys[];                   // [held]
    __shared__ uint32_t own[kBins], all[C > 1 ? kRankPasses : 1][C > 1 ? kBins : 1];
    __shared__ uint32_t scan[kRankWarps];
    __shared__ uint32_t found[3];                        // bin, keys above it, keys in it
    __shared__ uint32_t counts[2];                       // this block's keys above the last, and at it
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = C > 1 ? (int)cluster.block_rank() : 0;
    const int list = blockIdx.x / C, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const RankSeq& s = b.s[blockIdx.y];
    const int64_t L = rows_of(s.T, s.length);
    int32_t* idx = s.idx + list * s.keep;
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
    auto key = [&](uint32_t i) { return HELD || i < held ? keys[i] : rank_key(__ldg(w + i)); };

    for (int i = threadIdx.x; i < kBins; i += kRankThreads) {
        own[i] = 0;
        if (C > 1) all[0][i] = all[C > 1 ? 1 : 0][i] = all[C > 1 ? 2 : 0][i] = 0;
    }
    __syncthreads();
    for (uint32_t i0 = threadIdx.x; i0 < len; i0 += 8 * kRankThreads) {
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = i0 + k * kRankThreads < len ? __ldg(w + i0 + k * kRankThreads) : 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t i = i0 + k * kRankThreads, y = rank_key(x[k]);
            if (i >= len) break;
            if (HELD || i < held) keys[i] = y;
            atomicAdd(&own[y >> 21], 1u);                        // the first pass
        }
    }
    if (C > 1) cluster.sync();
    else __syncthreads();
    uint32_t need = want, prefix = 0, above = 0, equal = 0;      // above, equal: this block's
    int shift = 32;
#pragma unroll 1
    for (int pass = 0; pass < kRankPasses; ++pass) {
        const int bits = pass == 2 ? 10 : 11, up = shift;        // keys that match `prefix` in the bits from `up` on
        shift -= bits;
        if (pass) {
            for (int i = threadIdx.x; i < kBins; i += kRankThreads) own[i] = 0;
            __syncthreads();
#pragma unroll 4
            for (uint32_t i = threadIdx.x; i < len; i += kRankThreads) {
                const uint32_t k = key(i);
                if (k >> up == prefix) atomicAdd(&own[(k >> shift) & ((1u << bits) - 1)], 1u);
            }
            __syncthreads();
        }
        uint32_t* joined = C > 1 ? cluster.map_shared_rank(all[C > 1 ? pass : 0], 0) : own;
        if (C > 1) {
            for (int i = threadIdx.x; i < kBins; i += kRankThreads)
                if (own[i]) atomicAdd(joined + i, own[i]);
            cluster.sync();
        }
        // bins from the top: warp w has 64 of them, its lanes two each, bin0 + 1 and bin0
        const int bin0 = kBins - 2 - 2 * threadIdx.x;
        const uint32_t c0 = joined[bin0 + 1], c1 = joined[bin0];
        uint32_t total;
        const uint32_t here = __reduce_add_sync(0xFFFFFFFFu, c0 + c1);
        uint32_t before = warps_before(here, total, scan);
        if (before < need && need <= before + here) {            // the warp where the budget runs out
            uint32_t x = c0 + c1;
#pragma unroll
            for (int k = 1; k < 32; k *= 2) {
                const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, x, k);
                if (lane >= k) x += y;
            }
            before += x - c0 - c1;
            if (before < need && need <= before + c0 + c1) {
                const bool upper = need <= before + c0;
                found[0] = bin0 + upper;
                found[1] = upper ? before : before + c0;
                found[2] = upper ? c0 : c1;
            }
        }
        __syncthreads();
        const uint32_t bin = found[0];
        if (C > 1) {
            warps_before(__reduce_add_sync(0xFFFFFFFFu, ((uint32_t)bin0 + 1 > bin ? own[bin0 + 1] : 0) + ((uint32_t)bin0 > bin ? own[bin0] : 0)),
                         total, scan);
            above += total;
        }
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
    // every warp a run of the keys: counted, then written
    const uint32_t run = ((len + kRankWarps - 1) / kRankWarps + 31) & ~31u, from = min(len, warp * run), to = min(len, from + run);
    uint32_t n_above = 0, n_equal = 0, total;
#pragma unroll 4
    for (uint32_t i = from + lane; i < to; i += 32) {
        const uint32_t x = key(i) >> shift;
        n_above += x > prefix;
        n_equal += x == prefix;
    }
    above0 += warps_before(__reduce_add_sync(0xFFFFFFFFu, n_above), total, scan);
    equal0 += warps_before(__reduce_add_sync(0xFFFFFFFFu, n_equal), total, scan);
    const uint32_t below = (1u << lane) - 1;
#pragma unroll 4
    for (uint32_t i = from; i < to; i += 32) {
        const uint32_t x = i + lane < to ? key(i + lane) >> shift : 0;
        const bool over = i + lane < to && x > prefix, at = i + lane < to && x == prefix;
        const uint32_t o = __ballot_sync(0xFFFFFFFFu, over), e = __ballot_sync(0xFFFFFFFFu, at);
        const uint32_t mine = equal0 + __popc(e & below);
        if (over || (at && mine < need)) idx[s.first + above0 + __popc(o & below) + min(mine, need)] = (int32_t)(s.first + lo + i + lane);
        above0 += __popc(o);
        equal0 += __popc(e);
    }
}

// ---- their moving ---------------------------------------------------------------------------------

constexpr uint32_t kNone = 0xFFFFFFFFu;

__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.L2::64B.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld8(const void* p) {
    uint2 v;
    asm volatile("ld.global.L2::64B.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld4(const void* p) {
    uint32_t v;
    asm volatile("ld.global.L2::64B.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// Rows of a step of one group, as a thread holds them: pieces of codes, its own row's scales and weight.
template <int D>
struct Held {
    uint4 code[D / 32];
    uint2 scale;
    uint32_t weight;
};

// What a call makes of one cache: row base + j becomes row base + idx[j], j < count, idx[j] in j .. limit - 1.
struct Moving {
    int64_t base, count, limit;
    bool lists_own;
    // first: of the thread that says how many rows are left, and what was wrong.  (Of lists of their own, no other reads the
    // length.)
    __device__ __forceinline__ Moving(const MoveBatch& b, const MoveSeq& s, bool first) : lists_own(s.drafted < 0) {
        const bool says = first && s.left && !s.left_later;
        const int64_t L = !lists_own || says ? rows_of(s.T, s.length) : 0;
        base = lists_own ? 0 : L - s.drafted;
        limit = lists_own ? s.T : s.drafted;
        count = s.count;
        if (s.n_kept) count = max((int64_t)0, min((int64_t)__ldcg(s.n_kept), count));
        if (base < 0) {                       // fewer rows than `drafted`
            count = 0;
            if (first) atomicOr(b.err, kErrPackRow);
        } else if (says) {
            *s.left = (int32_t)(lists_own ? min(L, count) : base + count);
        }
    }
    // Entry j's row of `from` and of `to`; false where nothing is moved.
    __device__ __forceinline__ bool rows(const MoveBatch& b, const MoveSeq& s, int64_t j, int64_t i, uint2& r) const {
        if (lists_own && i == -1) return false;
        if (i < j || i >= limit) {
            atomicOr(b.err, kErrCompactIndex);
            return false;
        }
        if (i == j && s.in_place) return false;
        const int64_t x = packed_row(s.from, base + i), y = packed_row(s.to, base + j);
        if (x < 0 || y < 0) {
            atomicOr(b.err, kErrPageIndex);
            return false;
        }
        r = make_uint2((uint32_t)x, (uint32_t)y);
        return true;
    }
};

// (5 rows of 36 layers 2.9 us, 4 of 32 sequences in pages 5.7, 1.9 TB/s: launch, then three reads one after the other; a warp a
// list took 22.6.)
// Up to 32 entries: a thread moves a row of K or of V of one list, the block 256 / C of them (C: the power of two that
// has room for the entries).  All read before any writes.
template <int D>
__global__ void __launch_bounds__(256) k_move_few(const __grid_constant__ MoveBatch b, int C) {
    const MoveSeq& s = b.s[blockIdx.z];
    const int per = 256 / C, j = threadIdx.x % C, unit = blockIdx.x * per + threadIdx.x / C;
    const Moving m(b, s, blockIdx.x == 0 && threadIdx.x == 0);
    const int kv = unit & 1, list = unit >> 1, l = list / b.n_kv_heads, g = list % b.n_kv_heads;
    uint2 r = make_uint2(0, 0);
    uint4 code[D / 32];
    uint2 scale;
    uint32_t weight;
    int64_t i = 0;
    bool moves = list < b.n_layers * b.n_kv_heads && j < m.count;
    if (moves) {
        i = s.idx[list * s.idx_list + j];
        moves = m.rows(b, s, j, i, r);
    }
    const bool weigh = kv == 0 && s.w;
    if (moves) {
        const uint64_t row = (uint64_t)(l * s.from.s_layer + g * s.from.s_head) + r.x;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) code[k] = ld16(s.from.code[kv] + row * (D / 2) + 16 * k);
        if (D == 128) scale = ld8(s.from.scale[kv] + row * (D / 32));
        else scale.x = ld4(s.from.scale[kv] + row * (D / 32));
        if (weigh) weight = ld4(s.w + l * s.w_layer + g * s.w_head + m.base + i);
    }
    __syncthreads();
    if (moves) {
        const uint64_t row = (uint64_t)(l * s.to.s_layer + g * s.to.s_head) + r.y;
#pragma unroll
        for (int k = 0; k < D / 32; ++k) *reinterpret_cast<uint4*>(s.to.code[kv] + row * (D / 2) + 16 * k) = code[k];
        if (D == 128) *reinterpret_cast<uint2*>(s.to.scale[kv] + row * (D / 32)) = scale;
        else *reinterpret_cast<uint32_t*>(s.to.scale[kv] + row * (D / 32)) = scale.x;
        if (weigh) reinterpret_cast<uint32_t*>(s.w_to)[l * s.t_layer + g * s.t_head + m.base + j] = weight;
    }
}

// Rows into another cache: nothing that is read is written, so a warp takes 32 entries by itself, four (two) lanes a row.
// 2048 of 16384 rows, 36 layers x 8 heads of 128: 35 us for 170 MB. A scale's 8 bytes cost a read of 64, so DRAM moves 190 MB;
// reads that ask for 128 bytes (the default) moved 227 MB of them and took 49 us, with entries read ahead in a loop 41.
// (Blocks in the order of entries within a list: neighbours' places are neighbours.)
template <int D>
__global__ void __launch_bounds__(256) k_move_into(const __grid_constant__ MoveBatch b, int blocks) {
    constexpr int P = D / 32;                 // pieces of a row's codes, and rows of a lane
    const MoveSeq& s = b.s[blockIdx.z];
    const int unit = blockIdx.x / blocks, kv = unit & 1, list = unit >> 1, l = list / b.n_kv_heads, g = list % b.n_kv_heads;
    const int lane = threadIdx.x & 31, p = lane % P;
    const int64_t j0 = (int64_t)(blockIdx.x % blocks) * 256 + (threadIdx.x & ~31);
    const Moving m(b, s, blockIdx.x == 0 && threadIdx.x == 0);
    if (j0 >= m.count) return;
    const int32_t* idx = s.idx + list * s.idx_list;
    // the lane's own entry looked up, then handed to those that move its row
    const int64_t j = j0 + lane;
    const int64_t i = j < m.count ? (int64_t)idx[j] : -1;
    uint2 mine = make_uint2(0, 0);
    const bool moves = j < m.count && m.rows(b, s, j, i, mine);
    const int64_t from0 = l * s.from.s_layer + g * s.from.s_head, to0 = l * s.to.s_layer + g * s.to.s_head;
    const uint8_t* code = s.from.code[kv] + from0 * (D / 2) + p * 16;
    uint8_t* code_to = s.to.code[kv] + to0 * (D / 2) + p * 16;
    const uint32_t all = __ballot_sync(0xFFFFFFFFu, moves);
    uint4 x[P];
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const int r = lane / P + k * (32 / P);
        const uint32_t row = __shfl_sync(0xFFFFFFFFu, mine.x, r);
        if (all >> r & 1u) x[k] = ld16(code + (uint64_t)row * (D / 2));
    }
    uint2 scale = make_uint2(0, 0);
    uint32_t weight = 0;
    const bool weigh = kv == 0 && s.w && moves;
    if (moves) {
        const uint8_t* from = reinterpret_cast<const uint8_t*>(s.from.scale[kv]) + (from0 + mine.x) * (D / 16);
        if (D == 128) scale = ld8(from);
        else scale.x = ld4(from);
    }
    if (weigh) weight = ld4(s.w + l * s.w_layer + g * s.w_head + m.base + i);
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const int r = lane / P + k * (32 / P);
        const uint32_t row = __shfl_sync(0xFFFFFFFFu, mine.y, r);
        if (all >> r & 1u) *reinterpret_cast<uint4*>(code_to + (uint64_t)row * (D / 2)) = x[k];
    }
    if (moves) {
        uint8_t* to = reinterpret_cast<uint8_t*>(s.to.scale[kv]) + (to0 + mine.y) * (D / 16);
        if (D == 128) *reinterpret_cast<uint2*>(to) = scale;
        else *reinterpret_cast<uint32_t*>(to) = scale.x;
    }
    if (weigh) reinterpret_cast<uint32_t*>(s.w_to)[l * s.t_layer + g * s.t_head + m.base + j] = weight;
}

// 2048 of 16384 rows in place, 36 layers x 8 heads of 128: 44 us, 4.3 TB/s (k_move_into 34): a step's reads wait for memory, then all
// of the block for its slowest thread.
// A group of threads moves the rows of K or of V of one list, a row a thread a step: GROUP = 32, a warp; else a block, or
// the blocks of a cluster together.  In place a row's source is never before its place, so what a step writes is
// read by no later one; within a step every group reads before any writes (a barrier), and the next step's rows are on
// their way by then, as are the entries of the one after it.
template <int D, int GROUP>
__global__ void __launch_bounds__(256, 3) k_move(const __grid_constant__ MoveBatch b, int blocks, int clustered) {
    constexpr int P = D / 32;                 // pieces of a row's codes
    constexpr int N = GROUP / P;              // rows that a piece a thread covers
    __shared__ uint2 where[2][256];           // rows of the cache: from, to
    const MoveSeq& s = b.s[blockIdx.z];
    const int lists = b.n_layers * b.n_kv_heads;
    const int t = threadIdx.x % GROUP;
    const int group = GROUP == 32 ? blockIdx.x * (256 / 32) + threadIdx.x / 32 : blockIdx.x;
    const int unit = group / blocks, part = group % blocks;
    const Moving m(b, s, group == 0 && t == 0);
    if (unit >= 2 * lists) return;            // (a whole group)
    const int64_t base = m.base, count = m.count;
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

    // the thread's entry of the step at j0 (-1: none), and its rows
    auto entry = [&](int64_t j0) { return j0 + t < count ? (int64_t)idx[j0 + t] : -1; };
    auto look_up = [&](int64_t j0, int64_t i, uint2* to) {
        uint2 r = make_uint2(kNone, kNone);
        const bool moves = j0 + t < count && m.rows(b, s, j0 + t, i, r);
        to[t] = r;
        return moves ? i : -1;
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
    int64_t ahead = entry(j0);
    int64_t i = look_up(j0, ahead, rows);
    ahead = entry(j0 + step);
    meet();
    Held<D> h;
    load(rows, i, h);
    for (int64_t n = 0; n < steps; ++n, j0 += step) {
        uint2* here = rows + (n & 1) * 256;
        uint2* next = rows + (~n & 1) * 256;
        const int64_t i1 = look_up(j0 + step, ahead, next);
        ahead = entry(j0 + 2 * step);
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
    if (most <= 32) {
        int C = 1;
        while (C < most) C *= 2;
        k_move_few<D><<<dim3((units * C + 255) / 256, 1, b.n), 256, 0, st>>>(b, C);
        return cudaGetLastError();
    }
    if (!in_place) {
        const int blocks = (int)((most + 255) / 256);
        k_move_into<D><<<dim3((unsigned)(units * blocks), 1, b.n), 256, 0, st>>>(b, blocks);
        return cudaGetLastError();
    }
    // A warp a list, for up to 64 rows, and up to 128 where lists are many: 65 rows of 32 x 288 lists 48 us and with a block a list 108,
    // 128 rows 69 and 115; 128 rows of 288 lists 13 and 13, of 80 lists 13 and 9; 200 rows of 288 lists 18 and 13.  (Graphs, of
    // which 7 us are not the kernel's.)
    if (most <= 64 || (most <= 128 && (int64_t)units * b.n >= 3 * num_sms)) {
        k_move<D, 32><<<dim3((units + 7) / 8, 1, b.n), 256, 0, st>>>(b, 1, 0);
        return cudaGetLastError();
    }
    // A block a list, or more while there are fewer than SMs, a step's rows each at least: 1024 rows of 4 lists 13 us with one block a
    // list of K or V, 9 with four; of 64 lists 15.5 and 13.4 with two; of 152 lists 17.5 and 19.6 with two; 2048 rows of 288 lists
    // 44 with one or two, 56 with eight.
    int blocks = 1;
    while (blocks < 8 && (int64_t)units * b.n * blocks < num_sms && most > 256 * blocks) blocks *= 2;
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

template <int C, bool HELD>
cudaError_t launch_rank_by(const RankBatch& b, int64_t slice, cudaStream_t st) {
    static std::atomic<bool> set[64];     // (the attribute belongs to the device's function)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !set[dev]) {
        e = cudaFuncSetAttribute(k_rank<C, HELD>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRankKeys * 4);
        if (e != cudaSuccess) return e;
        if (dev < 64) set[dev] = true;
    }
    const uint32_t held = (uint32_t)(slice < kRankKeys ? slice : kRankKeys);
    const dim3 grid(b.n_layers * b.n_kv_heads * C, b.n);
    if (C == 1) {
        k_rank<C, HELD><<<grid, kRankThreads, held * 4, st>>>(b, held);
        return cudaGetLastError();
    }
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = C;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = dim3(kRankThreads);
    config.dynamicSmemBytes = held * 4;
    config.stream = st;
    config.attrs = &cluster;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, k_rank<C, HELD>, b, held);
}

}  // namespace

RankPlan rank_plan(const RankBatch& b) {
    int64_t most = 0;
    for (int i = 0; i < b.n; ++i) most = b.s[i].T > most ? b.s[i].T : most;
    // As few blocks of a list as hold it, however few lists there are: 2 lists of 16384 rows 16 us with one block each, 18 with
    // four, 20 with eight; 288 lists 21, 60 and 169 (the cluster's barriers and histograms that are joined in one block's memory);
    // 288 lists of 65536 rows 85 with four, 187 with eight.  (Calls that keep 32 rows, about 7 us of them not the ranking's.)
    RankPlan p{1, (most + 3) & ~(int64_t)3};
    while (p.blocks < kRankCluster && p.slice > kRankKeys) {
        p.blocks *= 2;
        p.slice = ((most + p.blocks - 1) / p.blocks + 3) & ~(int64_t)3;
    }
    p.held = p.slice <= kRankKeys;
    return p;
}

cudaError_t launch_rank(const RankBatch& b, cudaStream_t st) {
    const RankPlan p = rank_plan(b);
    if (!p.held) return launch_rank_by<kRankCluster, false>(b, p.slice, st);
    return p.blocks == 1 ? launch_rank_by<1, true>(b, p.slice, st) : p.blocks == 2 ? launch_rank_by<2, true>(b, p.slice, st)
         : p.blocks == 4 ? launch_rank_by<4, true>(b, p.slice, st) : launch_rank_by<8, true>(b, p.slice, st);
}

cudaError_t launch_move(const MoveBatch& b, int head_dim, cudaStream_t st, int num_sms) {
    int64_t most = 0;
    bool in_place = false;
    for (int i = 0; i < b.n; ++i) {
        most = b.s[i].count > most ? b.s[i].count : most;
        in_place |= b.s[i].in_place != 0;
    }
    // (no rows: lengths to write, and caches that may have fewer rows than `drafted`)
    bool says = false;
    for (int i = 0; i < b.n; ++i) says |= (b.s[i].left && !b.s[i].left_later) || (b.s[i].drafted > 0 && b.s[i].length);
    if (most == 0 && !says) return cudaSuccess;
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
