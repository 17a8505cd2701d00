// What the entry points of libdba share across its source files.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dba {

// The text that dba_last_error(NULL) gives the calling thread; returns `code`.
int set_error(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

inline bool format_ok(int format) { return format >= 0 && format <= 2; }
inline unsigned elem_bytes(int format) { return format == 0 ? 4u : 2u; }
inline bool misaligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

}  // namespace dba
