// What the translation units of entry points share: a profiler range around every call and the
// checks of arguments that recur.
#pragma once

#include <nvtx3/nvToolsExt.h>

#include "sp_internal.h"

namespace sp {

// NVTX range around one entry point: shows up in a timeline profile under the call's name;
// costs a function-pointer test when no profiler is attached.
class CallRange {
   public:
    explicit CallRange(const char *name) { nvtxRangePushA(name); }
    ~CallRange() { nvtxRangePop(); }
    CallRange(const CallRange &) = delete;
    CallRange &operator=(const CallRange &) = delete;
};
#define SP_CALL_RANGE() CallRange sp_call_range__(__func__)

inline bool valid_dtype(sp_dtype d) { return d == SP_F16 || d == SP_BF16; }

}  // namespace sp
