// Layout of the microscaled 4-bit format (cwac.h) and its limits.
#pragma once

#include <stdint.h>

namespace cwac {

constexpr int kMx4Block = 32;    // values that share a scale
constexpr int kMx4Panel = 256;   // values of a row whose eight scale bytes lie together: 128 bytes of codes, one K step of the product
constexpr int32_t kMx4MaxK = 1 << 18;
constexpr int64_t kMx4MaxRows = (int64_t)1 << 31;
constexpr int64_t kMx4MaxPitch = (int64_t)1 << 24;  // of the product's operands: 64 rows x pitch stays in 32 bits

}  // namespace cwac
