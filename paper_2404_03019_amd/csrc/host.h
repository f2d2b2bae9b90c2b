// Host-side services of the library's entry points that live in another file than api.hip: the
// calling thread's error detail and the temporary memory of a call.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <memory>

#include "../../include/geot.h"

namespace geot {

void detail_clear();
geot_status_t detail_fail(geot_status_t st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
geot_status_t detail_hip_fail(hipError_t e, const char *what);
bool ranges_overlap(const void *a, size_t na, const void *b, size_t nb);

// Temporary memory of one call on a stream: from the stream's kept buffer up to 64 MB (held until
// this object goes, after the call's last launch), else, and in a captured call, from the
// library's stream-ordered pool.
class CallMemory {
   public:
    explicit CallMemory(hipStream_t st);
    ~CallMemory();
    CallMemory(const CallMemory &) = delete;
    CallMemory &operator=(const CallMemory &) = delete;
    geot_status_t get(size_t bytes, char **p);

   private:
    struct State;
    std::unique_ptr<State> s_;
};

}  // namespace geot
