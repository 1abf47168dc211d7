// What the kernels over the 8-bit cache share.
#pragma once
#include "mfma_common.h"

constexpr int BYTE_BLOCK = PD_BYTE_BLOCK;

struct ByteCache {
  int8_t *k, *v;
  float *k_scale, *v_scale;
  void *k_tail, *v_tail;
  int n_req, n_kv_head, n_block;
};

// 8 consecutive values; WIDE: they lie at a multiple of 16 bytes
template <typename T, bool WIDE>
__device__ __forceinline__ void load8(const T *p, float x[8]) {
  if constexpr (!WIDE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = ld_f32(p, j);
  } else if constexpr (sizeof(T) == 4) {
    const float4 a = ((const float4 *)p)[0], b = ((const float4 *)p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    union { uint4 q; T h[8]; } u;
    u.q = *(const uint4 *)p;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = ld_f32(u.h, j);
  }
}

// as the output's type, to nearest (halves: beyond their range infinite, as a conversion is)
__device__ __forceinline__ void store8(float *p, const float y[8]) {
  ((float4 *)p)[0] = make_float4(y[0], y[1], y[2], y[3]);
  ((float4 *)p)[1] = make_float4(y[4], y[5], y[6], y[7]);
}
__device__ __forceinline__ void store8(bf16_t *p, const float y[8]) {
  *(uint4 *)p = make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
}
__device__ __forceinline__ void store8(f16_t *p, const float y[8]) {
  f16x8 h;
#pragma unroll
  for (int j = 0; j < 8; ++j) h[j] = (f16_t)y[j];
  *(f16x8 *)p = h;
}
__device__ __forceinline__ void store4(float *p, floatx4 y) { *(floatx4 *)p = y; }
__device__ __forceinline__ void store4(bf16_t *p, floatx4 y) { *(uint2 *)p = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3])); }
__device__ __forceinline__ void store4(f16_t *p, floatx4 y) {
  union { f16_t h[4]; uint2 u; } o;
#pragma unroll
  for (int j = 0; j < 4; ++j) o.h[j] = (f16_t)y[j];
  *(uint2 *)p = o.u;
}
