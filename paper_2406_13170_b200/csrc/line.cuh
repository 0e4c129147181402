// Arithmetic of work that is a line of units spread over blocks; also compiled for the host, where it is tested.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define AMPH_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define AMPH_HOST_DEVICE inline
#endif

namespace amph {

// a * b / d, of which the product mostly has 32 bits (a 64-bit division is about 100 instructions)
AMPH_HOST_DEVICE long long mul_div(long long a, int b, long long d) {
  const unsigned long long x = (unsigned long long)a * (unsigned)b;
  return ((x | (unsigned long long)d) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)d) : (long long)(x / (unsigned long long)d);
}

// The block that holds unit u when `total` units are spread over n blocks (block c begins at total * c / n).
AMPH_HOST_DEVICE int block_of(long long u, long long total, int n) {
  const unsigned long long x = (unsigned long long)(u + 1) * (unsigned)n - 1;
  return (int)(((x | (unsigned long long)total) >> 32) == 0 ? (uint32_t)x / (uint32_t)total : x / (unsigned long long)total);
}

}  // namespace amph
