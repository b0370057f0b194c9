// eqb_checks.h -- argument checks shared by the files of the exported ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "eqb.h"
#include "eqb_internal.h"

namespace {

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Sizes the library supports (the paper allows 1 <= K < E).
inline eqb_status check_shape(int64_t T, int32_t E, int32_t K, bool need_k) {
  if (T < 0 || E < 2) return EQB_ERR_INVALID_ARG;
  if (need_k && (K < 1 || K >= E)) return EQB_ERR_INVALID_ARG;
  if (E > eqb::kMaxE || (E % 8) != 0) return EQB_ERR_UNSUPPORTED;
  if (need_k && K + 1 > 32) return EQB_ERR_UNSUPPORTED;
  // 32-bit token loop indices need headroom above T.
  if (T > (int64_t(1) << 31) - (int64_t(1) << 24)) return EQB_ERR_UNSUPPORTED;
  return EQB_OK;
}

inline cudaStream_t as_stream(void* s) { return reinterpret_cast<cudaStream_t>(s); }

inline eqb_status to_status(int rc) { return static_cast<eqb_status>(rc); }

}  // namespace
