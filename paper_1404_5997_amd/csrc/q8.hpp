// Rows of 8-bit values.
#pragma once
#include <stddef.h>

namespace owt {

constexpr int kQ8Align = 128;               // they start at multiples of this many bytes, zeros behind their values
inline __host__ __device__ size_t q8_pitch(int cols) { return ((size_t)cols + kQ8Align - 1) / kQ8Align * kQ8Align; }

}  // namespace owt
