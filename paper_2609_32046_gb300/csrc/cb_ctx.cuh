// The context behind the C-ABI's opaque handle, and what the host side of every entry point uses.
#pragma once

#include <algorithm>
#include <cstdint>
#include <string>
#include <vector>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "cacheback.h"
#include "cb_receiver.cuh"

namespace cbk {
constexpr int64_t kDefaultWaitNs = 1000000000;   // 1 s
}

namespace cbk {
// The last cb_rope of a context as the kernel takes it.
struct RopeTable {
    cb_rope key{};
    int32_t dims = 0;               // 0: none yet
    float gain = 1.f;
    uint64_t turns[64] = {};
};
}  // namespace cbk

struct cb_ctx {
    cb_config cfg;
    int device = 0;
    int num_sms = 0;
    int G = 1;
    bool use_tc = false;
    bool tc_stage_must = false;     // paged senders must be staged (the shapes score_kernel = 2 takes)
    float scale = 0.f;
    float* scratch = nullptr;       // per sender: pass-1 partials, then pass-2 partials in their place
    float* offs = nullptr;
    uint16_t* ext = nullptr;        // tcgen05 passes: per-row offset terms [S][nS][R_pad][16] bf16
    uint16_t* ones = nullptr;       // tcgen05 passes: [128][16] bf16 block of ones columns
    float* span_keys = nullptr;
    uint16_t* stage = nullptr;      // tcgen05 passes: contiguous copies of paged senders' K (on demand)
    int64_t stage_elems = 0;
    bool stage_captured = false;    // a captured cb_score uses `stage`: a graph holds its address
    std::vector<uint16_t*> old_stages;   // outgrown buffers that graphs may still use, until cb_destroy
    uint32_t* err = nullptr;
    int64_t keys_per_sender = 0;
    int64_t scratch_bytes = 0;
    int32_t score_path = 0;         // kernels of the last cb_score: 2 tcgen05, 1 mma.sync, 0 none yet
    int64_t wait_ns = cbk::kDefaultWaitNs;   // limit of one bounded device wait (tcgen05 passes)
    int32_t stall_next = 0;         // failure-detection test: stall the next cb_score once
    int32_t stall_attend = 0;       // the same for the next cb_attend on the tcgen05 kernel
    int32_t stall_weigh = 0;        // and for the next cb_weigh on its
    int32_t score_sms = 0;          // SMs of the persistent score kernels (0: all)
    bool receiver = false;          // no scratch for cb_score and cb_select
    float* attend_part = nullptr;   // cb_attend: partial results (outputs; maxima and sums)
    float2* attend_ml = nullptr;
    int32_t* attend_tickets = nullptr;   // zero between calls
    cbk::AttendCut* attend_cuts = nullptr;    // and its records of items that several blocks share
    cbk::RopeTable rope;
    cbk::StageTimer* timer = nullptr;
    std::string last_error;
};

namespace cbk {

// Records the text of cb_last_error and returns st (ctx == nullptr: the text of cb_last_error(NULL)).
cb_status fail(cb_ctx* ctx, cb_status st, const char* fmt, ...);

// Device (or managed) memory on ctx's device; device memory or mapped pinned host memory (*dev: the
// address to use on the device).
cb_status check_device_ptr(cb_ctx* ctx, const void* p, const char* what, int i, int align = 16);
cb_status check_source_ptr(cb_ctx* ctx, const void* p, const char* what, int i, int align, const void** dev);

// check_device_ptr for the many pointers of one call: allocations that one of them was found in are known for the
// others (a query of the driver takes longer than all the rest of a pointer's check).
class DevicePtrs {
public:
    explicit DevicePtrs(cb_ctx* ctx) : ctx_(ctx) {}
    cb_status check(const void* p, const char* what, int i, int align = 16);

private:
    cb_ctx* ctx_;
    uintptr_t lo_[8] = {}, hi_[8] = {};
    int n_ = 0;
};

// cb_attend's room for partial results, allocated by the first call that needs it.
cb_status attend_scratch(cb_ctx* ctx, cudaStream_t st);

// Makes ctx's device current for the duration of a call, restoring the caller's device after.
struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
        if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

// Memory that one part of a call writes; dense: every byte of it.
struct Written {
    uintptr_t lo, hi;
    bool dense;
};
// Two parts write the same place: they begin there both, or both are dense and overlap.  (Parts that lie between
// one another's rows, as the slices of a wider array do, are let pass.)  Sorts `w` unless it is in order and apart.
inline bool written_twice(std::vector<Written>& w) {
    bool apart = true;
    for (size_t i = 1; i < w.size() && apart; ++i) apart = w[i - 1].hi <= w[i].lo;
    if (apart) return false;
    std::sort(w.begin(), w.end(), [](const Written& a, const Written& b) { return a.lo < b.lo; });
    uintptr_t end = 0;
    for (size_t i = 0; i < w.size(); ++i) {
        if (i && w[i].lo == w[i - 1].lo) return true;
        if (!w[i].dense) continue;
        if (w[i].lo < end) return true;
        end = w[i].hi;
    }
    return false;
}

// A part reads what another part writes: they begin there both, or both are dense and overlap.  `reads` and `writes` name their
// parts by `of`; no two writes clash (written_twice).
struct PartOf {
    Written at;
    int32_t of;
};
inline bool read_and_written(const std::vector<PartOf>& reads, std::vector<PartOf> writes) {
    if (writes.empty()) return false;
    auto by_lo = [](const PartOf& a, const PartOf& b) { return a.at.lo < b.at.lo; };
    if (!std::is_sorted(writes.begin(), writes.end(), by_lo)) std::sort(writes.begin(), writes.end(), by_lo);
    for (const PartOf& r : reads) {
        const auto same = std::lower_bound(writes.begin(), writes.end(), r, by_lo);
        if (same != writes.end() && same->at.lo == r.at.lo && same->of != r.of) return true;
    }
    writes.erase(std::remove_if(writes.begin(), writes.end(), [](const PartOf& w) { return !w.at.dense; }), writes.end());
    for (const PartOf& r : reads) {
        if (!r.at.dense) continue;
        // (dense writes lie apart, in order: those that overlap are the last ones that begin before the end)
        auto w = std::lower_bound(writes.begin(), writes.end(), r.at.hi, [](const PartOf& a, uintptr_t hi) { return a.at.lo < hi; });
        while (w != writes.begin() && (--w)->at.hi > r.at.lo)
            if (w->of != r.of) return true;
    }
    return false;
}

inline bool stride_ok(int64_t s) { return s > 0 && (s % 8) == 0; }

// An NVTX range over one call of the C-ABI (header-only NVTX: free unless a profiler listens).
struct NvtxRange {
    explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
};

}  // namespace cbk
