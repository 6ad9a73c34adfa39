// Host-side pieces shared by the entry points: error message of the calling thread, tensor-map encoder, workspace
// check, optional per-kernel timing.
#pragma once

#include "../../include/tkphi.h"
#include "common.cuh"

#include <vector>

namespace tkphi {

void clear_error();
// Sets the calling thread's error message (tkphi_last_error) and returns st.
tkphi_status fail(tkphi_status st, const char* fmt, ...);
tkphi_status cuda_fail(cudaError_t e, const char* what);
tkphi_status check_ws(void* ws, size_t have, size_t need);
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn();

struct TimedSpan { cudaEvent_t a, b; int kind; };
extern bool g_timing;
extern std::vector<TimedSpan> g_spans;
// Brackets the launches made during its life with events while timing is on.
struct ScopedSpan {
  cudaStream_t st; int kind; cudaEvent_t a = nullptr, b = nullptr;
  ScopedSpan(cudaStream_t s, int k);
  ~ScopedSpan();
};

}  // namespace tkphi
