// What the host files of the library share: argument checks, launches with optional timing, HIP errors.
#pragma once

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/efsparse.h"

namespace efs {

constexpr size_t kAlign = 256;

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline hipStream_t S(void* s) { return reinterpret_cast<hipStream_t>(s); }

// EF_OK, or EF_EHIP with the error kept for the calling thread.
int hip_status(hipError_t e);
inline int launched() { return hip_status(hipGetLastError()); }

// While timing is on, a launch gets a start and a stop event that the runtime ties to the kernel's
// own dispatch (hipExtLaunchKernelGGL), so the elapsed time is the kernel's execution alone.
bool timing_slot(const char* name, hipEvent_t* a, hipEvent_t* b);

}  // namespace efs

// Every launch goes through this macro: the kernel is named after its expression, or NAME (static storage).
#define EF_LAUNCH(KERNEL, GRID, BLOCK, SHM, ST, ...) EF_LAUNCH_AS(#KERNEL, KERNEL, GRID, BLOCK, SHM, ST, __VA_ARGS__)
#define EF_LAUNCH_AS(NAME, KERNEL, GRID, BLOCK, SHM, ST, ...)                          \
  do {                                                                                 \
    hipEvent_t _ea = nullptr, _eb = nullptr;                                           \
    if (efs::timing_slot(NAME, &_ea, &_eb))                                            \
      hipExtLaunchKernelGGL(KERNEL, GRID, BLOCK, SHM, ST, _ea, _eb, 0u, __VA_ARGS__); \
    else                                                                               \
      hipLaunchKernelGGL(KERNEL, GRID, BLOCK, SHM, ST, __VA_ARGS__);                  \
  } while (0)

#define EF_TRY(x)              \
  do {                         \
    const int _rc = (x);       \
    if (_rc != EF_OK) return _rc; \
  } while (0)
