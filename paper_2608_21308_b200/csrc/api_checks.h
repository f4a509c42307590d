// Argument checks that the entry points share.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/e2ttt.h"

namespace e2ttt {

// Every workspace starts with a status block: word 0 is the device status of the last launch that used it.
constexpr size_t kStatusBytes = 256;

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_device();  // api.cu

}  // namespace e2ttt
