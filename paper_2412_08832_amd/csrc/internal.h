// internal.h -- what the source files of libhadacore share; not part of the ABI.
#ifndef HADACORE_INTERNAL_H
#define HADACORE_INTERNAL_H

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "hadacore.h"

#pragma GCC visibility push(hidden)

namespace hadacore {

// HADACORE_SUCCESS where the current device is a gfx950, else the error.
hadacore_status check_device();

// Compute units of the current device.
int device_cus();

// Byte range of `rows` rows of `width` elements of `size` bytes, `pitch` elements apart.
struct Span {
  uintptr_t lo, hi;
};

inline Span span(const void *p, int64_t rows, int64_t pitch, int64_t width, int64_t size) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  if (rows <= 0 || width <= 0) return {lo, lo};
  return {lo, lo + (uintptr_t)(((rows - 1) * pitch + width) * size)};
}

inline bool spans_overlap(Span x, Span y) { return x.lo < y.hi && y.lo < x.hi; }

// fp8_blocks.hip: rows of `k` values rotated by 2^L = 1..64 of them, e4m3 codes and a
// scale for each 128 values of a row.  Arguments are checked by the caller.
hipError_t launch_short_rotations(const uint16_t *in, int64_t in_stride, uint8_t *codes,
                                  int64_t codes_stride, float *scales, int64_t scales_stride,
                                  int64_t m, int k, int L, hadacore_dtype dtype, float scale,
                                  hipStream_t stream);

}  // namespace hadacore

#pragma GCC visibility pop

#endif  // HADACORE_INTERNAL_H
