// What the entry points of libdba share across its source files.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dba {

// The text that dba_last_error(NULL) gives the calling thread; returns `code`.
int set_error(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// A launch that tells how it went, so that of one that failed it is known that no kernel of it is under way: hipGetLastError, behind the <<< >>> form,
// may tell of an earlier call on this thread, of whomever, and takes that error from its owner.  (Nor does this one pass its grid through the runtime first: a step's call takes 2.85 instead of 3.05
// us with one launch and 5.27 instead of 5.65 with two, which is the time of a step where short ones of several decodes alternate.)
template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t stream, const A &...a)
{
    auto with = [&](P... arg) {
        void *args[] = {&arg...};
        return hipLaunchKernel(reinterpret_cast<const void *>(kernel), grid, block, args, lds, stream);
    };
    return with(a...);
}

inline bool format_ok(int format) { return format >= 0 && format <= 2; }
inline unsigned elem_bytes(int format) { return format == 0 ? 4u : 2u; }
inline bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

}  // namespace dba
