// Argument checks and conversions shared by the files that implement the C ABI.
#pragma once
#include "../../include/lattice.h"
#include "common.h"

#define FAIL(code, ...)         \
  do {                          \
    ::lat::set_error(__VA_ARGS__); \
    return code;                \
  } while (0)
#define REQUIRE(cond, ...) \
  do {                     \
    if (!(cond)) FAIL(LATTICE_ERR_INVALID_ARG, __VA_ARGS__); \
  } while (0)
#define HIPRET(expr)                                  \
  do {                                                \
    hipError_t e__ = (expr);                          \
    if (e__ != hipSuccess) return LATTICE_ERR_HIP;    \
  } while (0)

namespace lat {
static inline DType dt_of(lattice_dtype d) { return d == LATTICE_BF16 ? DT_BF16 : DT_F32; }
static inline size_t esize(lattice_dtype d) { return d == LATTICE_BF16 ? 2 : 4; }
static inline hipStream_t strm(void* s) { return reinterpret_cast<hipStream_t>(s); }
static inline size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }
}  // namespace lat
