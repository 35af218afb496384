// Shared by the kernels of exactmoe_serving.h: the 16-bit and 8-bit element
// types and the tickets of outputs that several workgroups share.
#pragma once

#include "common.h"
#include "exactmoe_serving.h"

namespace emoe {

struct Bf16 {
  static constexpr int kType = EMOE_BF16;
  __device__ static __forceinline__ float up(uint32_t bits) { return bf16_to_f32(bits); }
  __device__ static __forceinline__ uint32_t down(float x) { return f32_to_bf16_rne(x); }
};
struct Fp16 {
  static constexpr int kType = EMOE_F16;
  __device__ static __forceinline__ float up(uint32_t bits) { return half_bits_to_f32((uint16_t)bits); }
  __device__ static __forceinline__ uint32_t down(float x) {
    return __builtin_bit_cast(uint16_t, (_Float16)x);
  }
};

// Eight 16-bit elements of a 16-byte chunk, up to fp32 and back.
template <class T>
__device__ __forceinline__ void up8(const uint4& c, float (&v)[8]) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    v[2 * p] = T::up(w[p] & 0xffffu);
    v[2 * p + 1] = T::up(w[p] >> 16);
  }
}
template <class T>
__device__ __forceinline__ uint4 down8(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) w[p] = T::down(v[2 * p]) | (T::down(v[2 * p + 1]) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight values as E4M3: nearest even, saturated (the conversion alone would
// make NaN of what lies above 448); NaN stays NaN.
__device__ __forceinline__ uint2 down8_e4m3(const float (&v)[8]) {
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = v[i] != v[i] ? v[i] : fminf(fmaxf(v[i], -448.f), 448.f);
  uint2 w;
  w.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
  w.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], (int)w.x, true);
  w.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[4], c[5], 0, false);
  w.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[6], c[7], (int)w.y, true);
  return w;
}

// Tickets, each in a line of its own: device-coherent atomics
// on one line come one after the other, whatever the word (19 rows' tickets in
// one line kept a launch busy for 10 us).
constexpr int kTicketLine = 128, kTicketStride = kTicketLine / 4;
constexpr int kTickets = EMOE_SERVING_TICKET_BYTES / kTicketLine;

// The argument checks of emoe_process_logits.
int32_t check_process_logits(const emoe_logits_args& args, const void* workspace,
                             size_t workspace_bytes);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace emoe
