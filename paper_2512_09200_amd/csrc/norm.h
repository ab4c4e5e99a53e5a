// Internal interface of the residual norm and of dropout (namespace lat).
// Launchers enqueue on the given stream and return the first HIP error.
#pragma once
#include "common.h"
#include "dropout.h"

namespace lat {

constexpr int NORM_MAX_COLS = 16384;

// [rows, cols] with a row stride in elements
struct RowTensor {
  void* p = nullptr;
  int64_t ld = 0;
};

struct NormArgs {
  DType dt = DT_BF16;
  int64_t rows = 0;
  int cols = 0;
  float eps = 0.f;
  const float* gain = nullptr;
  DropArgs drop;
  RowTensor x, r, h, y;               // forward; y: null where only codes are asked for
  uint8_t* q = nullptr;
  int64_t ldq = 0;
  float* scales = nullptr;
  RowTensor dy, dh, dr, dx;           // backward, with h
  float* dgain = nullptr;
};
hipError_t add_rmsnorm_fwd(const NormArgs& a, hipStream_t s);
size_t add_rmsnorm_bwd_workspace(int64_t rows, int cols);
hipError_t add_rmsnorm_bwd(const NormArgs& a, void* ws, hipStream_t s);

hipError_t dropout(DType dt, int64_t rows, int cols, const DropArgs& d, RowTensor x, RowTensor out, hipStream_t s);

// floor(n / d) for n < 2^31, 1 <= d < 2^31, by a product: with 2^(l-1) < d <= 2^l and
// m = floor(2^(31+l) / d) + 1 < 2^32, n m / 2^(31+l) exceeds n / d by less than
// n / 2^(31+l) <= 2^-l <= 1 / d, so the floors agree.  (d = 1: l = 0, m = 2^31 + 1.)
struct FastDiv {
  uint32_t m;
  int shift;                          // of the 64-bit product
  explicit FastDiv(uint32_t d) {
    int l = 0;
    while ((1ull << l) < d) ++l;
    shift = 31 + l;
    m = (uint32_t)((1ull << shift) / d + 1);
  }
  __host__ __device__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> shift); }
};

}  // namespace lat
