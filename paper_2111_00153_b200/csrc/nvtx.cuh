#pragma once
#include <nvtx3/nvToolsExt.h>

// A named NVTX range around every call that queues GPU work: a profiler's timeline shows which API call a
// kernel belongs to.  Without a tool attached the two calls return at once.
struct NvtxRange {
    explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
    NvtxRange(const NvtxRange&) = delete;
    NvtxRange& operator=(const NvtxRange&) = delete;
};
