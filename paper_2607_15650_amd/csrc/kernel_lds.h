// kernel_lds.h - dynamic LDS of a kernel beyond the default.
#pragma once

#include "internal.h"

namespace ditango {

// Dynamic LDS of a kernel, set once on every device.
template <auto KERNEL, int BYTES>
inline hipError_t set_kernel_lds(int dev) {
  static OncePerDevice once;
  return once.run(dev, [] {
    return hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, BYTES);
  });
}

}  // namespace ditango
