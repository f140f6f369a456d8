// Host helpers shared by the entry points (defined in api.hip).
#pragma once
#include "common.h"

namespace pevlm {

// Sets the calling thread's error message and returns `st`.
pevlm_status fail(pevlm_status st, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
pevlm_status hip_fail(hipError_t e, const char *what);
pevlm_status check_heads(const pevlm_heads *h, HeadTable *tab);
float scale_of(const pevlm_heads *h);
int32_t compute_units();

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

}  // namespace pevlm
