// Shared by the token-sequence operators: status reporting of the C ABI, argument blocks,
// launcher declarations.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "dendsn.h"

namespace dendsn {

// The calling thread's error message and the launch counter live in dendsn_capi.cu.
dendsn_status seq_fail(dendsn_status st, const char *fmt, ...);
void seq_count_launches(int n);

inline bool seq_aligned(const void *p, size_t a) {
    return (reinterpret_cast<uintptr_t>(p) % a) == 0;
}

}  // namespace dendsn
