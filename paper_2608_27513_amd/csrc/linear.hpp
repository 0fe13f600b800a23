// Operands shared by the linear-attention kernels (damp_serving.h).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "internal.hpp"

namespace damp {

struct LinearParams {
  uint8_t* layer_base;
  uint64_t slot_stride;  // bytes
  uint64_t tile_stride;  // bytes
  const int32_t* slot_in;
  const int32_t* slot_out;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const float* g;
  void* o;
  int64_t q_stride, k_stride, v_stride, g_stride;  // elements between tokens
  float scale;
  int32_t num_slots;
  int32_t HK, HV;
  int32_t dk, dv;
  int32_t o_bf16;
};

// Checks what both entry points share and fills `p`. `rows` is the number of
// tokens that the operands hold; nothing is checked of operands when it is 0.
damp_status linear_params(const char* name, const damp_pool* pool, int32_t layer,
                          const int32_t* slot_in, const int32_t* slot_out, int32_t B, int64_t rows,
                          int32_t num_k_heads, const uint16_t* q, int64_t q_stride,
                          const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                          const float* g, int64_t g_stride, float scale, void* o, int32_t o_dtype,
                          hipStream_t stream, LinearParams* p);

}  // namespace damp
