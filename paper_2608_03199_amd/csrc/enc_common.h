// enc_common.h -- value types and small helpers shared by the text-encoder
// operators (norm.hip, attn_*.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sieve_internal.h"

namespace sieve {

typedef uint32_t enc_u32x4 __attribute__((ext_vector_type(4)));

constexpr int enc_size(int dtype) { return dtype == SIEVE_F32 ? 4 : 2; }

inline bool enc_dtype_ok(int dtype) {
  return dtype == SIEVE_F32 || dtype == SIEVE_F16 || dtype == SIEVE_BF16;
}

#define ENC_HIP_TRY(expr)                                                                    \
  do {                                                                                       \
    hipError_t e_ = (expr);                                                                  \
    if (e_ != hipSuccess)                                                                    \
      return set_error(e_ == hipErrorOutOfMemory ? SIEVE_ENOMEM : SIEVE_EDEVICE, "%s: %s (%s)", \
                       #expr, hipGetErrorString(e_), __func__);                              \
  } while (0)

// E consecutive values of T, moved in 16-byte pieces.
template <typename T, int E>
struct EncVec {
  T v[E];
};

// Aligned move of E values (E * sizeof(T) is a multiple of 16).
template <typename T, int E>
__device__ __forceinline__ EncVec<T, E> enc_load(const T* p) {
  constexpr int kPieces = E * (int)sizeof(T) / 16;
  EncVec<T, E> r;
  enc_u32x4 q[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) q[i] = ((const enc_u32x4*)p)[i];
  __builtin_memcpy(&r, q, sizeof(r));
  return r;
}
template <typename T, int E>
__device__ __forceinline__ void enc_store(T* p, const EncVec<T, E>& r) {
  constexpr int kPieces = E * (int)sizeof(T) / 16;
  enc_u32x4 q[kPieces];
  __builtin_memcpy(q, &r, sizeof(r));
#pragma unroll
  for (int i = 0; i < kPieces; ++i) ((enc_u32x4*)p)[i] = q[i];
}

}  // namespace sieve
