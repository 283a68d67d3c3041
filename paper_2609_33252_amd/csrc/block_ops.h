// Device and host helpers shared by the operators around the routed experts
// (norm, gate, dispatch, sort, dense feed-forward).  Internal to libcep.
#pragma once

#include "cep.h"
#include "common.h"
#include "profile.h"

#include <hip/hip_bf16.h>

#include <cstdarg>
#include <cstdio>

namespace cep {

// largest row count of the operators' descriptors (a launch holds fewer than
// 2^32 threads, and a row takes up to 1024)
constexpr int kMaxOpRows = 1 << 21;

// Records the message of a refused or failed call (cep_last_error(NULL)).
__attribute__((format(printf, 2, 3))) inline int refuse(int code, const char *fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return set_global_error(code, buf);
}

inline int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CEP_OK : refuse(CEP_EHIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool is_float_dtype(int t) { return t == CEP_F32 || t == CEP_BF16; }
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
inline size_t dtype_bytes(int t) { return t == CEP_F32 ? 4 : 2; }

// 16 bytes at an address of any alignment (one global access either way).
typedef uint32_t Vec16 __attribute__((ext_vector_type(4)));
typedef Vec16 Any16 __attribute__((aligned(1)));

// Eight consecutive values of a float32 or bf16 row, n of them inside it (the
// others read as zero and are not stored).
__device__ inline void load8(const void *row, int dtype, int64_t at, int n, float v[8]) {
  if (n >= 8) {
    if (dtype == CEP_BF16) {
      const Vec16 u = *(const Any16 *)((const char *)row + at * 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(u[j] << 16);
        v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
      }
    } else {
      const Vec16 lo = *(const Any16 *)((const char *)row + at * 4);
      const Vec16 hi = *(const Any16 *)((const char *)row + at * 4 + 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = __uint_as_float(lo[j]);
        v[4 + j] = __uint_as_float(hi[j]);
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = 0.f;
    if (j < n)
      v[j] = dtype == CEP_BF16 ? (float)((const __bf16 *)row)[at + j] : ((const float *)row)[at + j];
  }
}

__device__ inline uint32_t bf16_pair(float a, float b) {
  union { __bf16 h[2]; uint32_t u; } o;
  o.h[0] = (__bf16)a;  // to nearest even
  o.h[1] = (__bf16)b;
  return o.u;
}

__device__ inline void store8(void *row, int dtype, int64_t at, int n, const float v[8]) {
  if (n >= 8) {
    Vec16 u;
    if (dtype == CEP_BF16) {
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = bf16_pair(v[2 * j], v[2 * j + 1]);
      *(Any16 *)((char *)row + at * 2) = u;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = __float_as_uint(v[4 * h + j]);
        *(Any16 *)((char *)row + at * 4 + 16 * h) = u;
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) {
      if (dtype == CEP_BF16) ((__bf16 *)row)[at + j] = (__bf16)v[j];
      else ((float *)row)[at + j] = v[j];
    }
}

// Sum over the 64 lanes of a wave, in every lane.
__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

}  // namespace cep
