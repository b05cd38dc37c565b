// What the host sides of the entry points around the sampler have in common.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/sip.h"

namespace {

inline size_t head_align(size_t x) { return (x + 255) / 256 * 256; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool workspace_ok(const void* p, size_t have, size_t need) {
  return p && (reinterpret_cast<uintptr_t>(p) & 255u) == 0 && have >= need;
}
inline int tiles(long long n, int tile) { return (int)((n + tile - 1) / tile); }
constexpr int kChip = 256;                             // workgroups of a compute unit each
inline bool dtype_ok(sip_dtype t) { return t == SIP_F32 || t == SIP_BF16; }
inline int dtype_bytes(sip_dtype t) { return t == SIP_F32 ? 4 : 2; }
// Rows of `n` elements at `p`, `stride` elements apart, that start at multiples of 16 bytes.
inline bool rows_ok(const void* p, int64_t n, int64_t stride, sip_dtype t) {
  return p && aligned16(p) && stride >= n && stride % (16 / dtype_bytes(t)) == 0;
}

inline sip_status launched() { return hipGetLastError() == hipSuccess ? SIP_OK : SIP_ERR_HIP; }

}  // namespace
