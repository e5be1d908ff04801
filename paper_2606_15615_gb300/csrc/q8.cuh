// 8-bit rows (include/moeca_q8.h): block scales, encoding and decoding.
//
// The scale of a block of 128 values is a power of two, so dividing by it is
// exact and the only rounding is the one to the 8-bit format: any order of
// evaluation, and the tensor core's own scaling, gives the same value.  A
// power of two costs no precision against a free fp32 scale, since the values
// themselves are floating point; at most one binade of range at the top stays
// unused.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "moeca_q8.h"

namespace moeca {

constexpr int kQ8Block = 128;
constexpr int kQ8TileRows = 224, kQ8TileCols = 256;  // a tile of q8_matmul.cu: token rows, weight rows

// What the launches of q8.cu and q8_matmul.cu take (checked by their C calls).
struct Q8Rows {
  uint8_t* q;
  uint8_t* scale;
  int64_t rows, q_stride, scale_stride;
  int width;
};

// Bits of |x|; infinities and NaN are those from kNonFinite on.
constexpr uint32_t kNonFinite = 0x7f800000u;
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale byte of a block whose largest finite magnitude has the bits `a`.
// MAX is 1.75 x 2^8 (e4m3) or 1.75 x 2^15 (e5m2): the scale's exponent is a's
// less 8 or 15, one more where a's significand exceeds 1.75.
template <bool E5>
__device__ __forceinline__ int scale_byte(uint32_t a) {
  const int e = static_cast<int>(a >> 23) - (E5 ? 15 : 8) + ((a & 0x7fffffu) > 0x600000u);
  return a == 0 ? 127 : max(e, 0);
}
// 1 / scale: 2^(127 - byte), byte <= 247 as written by scale_byte.
__device__ __forceinline__ float scale_inverse(int byte) { return __uint_as_float(static_cast<uint32_t>(254 - byte) << 23); }
// The scale: 2^(byte - 127); 2^-127 is subnormal, 255 is NaN.
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(max(byte << 23, 0x400000u) + (byte == 255));
}

// Two values (already divided by the scale) in 8 bits, the first in the low byte.
// NaN becomes NaN.  An infinity is taken for the largest value, 0x7b in e5m2 (one
// below infinity) and 0x7e in e4m3 (one below NaN): a caller that may have met
// one adds 1 to its byte, which is right in both.
template <bool E5>
__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, E5 ? __NV_E5M2 : __NV_E4M3);
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return r;
}

// Two bytes as two floats (every e4m3 / e5m2 value is an fp16 value).
template <bool E5>
__device__ __forceinline__ float2 decode2(uint32_t pair) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(pair), E5 ? __NV_E5M2 : __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// The 16 bytes from byte `m` (a multiple of the type's size, below 16) of two
// consecutive 16-byte pieces.
template <typename TI>
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, uint32_t m) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = m & 8 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = m & 4 ? w[i + 1] : w[i];
  if (sizeof(TI) == 2) {
    const uint32_t sel = m & 2 ? 0x5432 : 0x3210;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __byte_perm(w[i], w[i + 1], sel);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// How long a kernel's bounded waits last, and the one that is to run out (tests;
// see moeca_probe_q8_stall): a barrier of that kind is set up for one arrival
// more than comes.
struct Q8Waits {
  unsigned long long ns;
  int stall;  // moeca_probe_q8_barrier, 0: none
};
Q8Waits q8_waits();  // of the calling host thread

// Whether 16-byte accesses can take rows of this base and stride.
inline bool q8_aligned16(const void* p, int64_t stride_bytes) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride_bytes % 16 == 0;
}

struct Q8WriteArgs {
  Q8Rows c;
  const void* x;
  int64_t x_rows, x_stride;
  int n;
  const int32_t *src, *dst, *count;
};
cudaError_t launch_q8_write(const Q8WriteArgs& a, bool bf16, bool e5, cudaStream_t s);

struct Q8CombineArgs {
  Q8Rows c;
  const int32_t* rows;   // null: slot row = token (one slot)
  const float* weights;
  const void* x;
  int64_t x_stride;
  const float* gate;
  int64_t gate_stride;
  void* out;
  int64_t out_stride;
  float* norms;
  int32_t* status;
  int T, k, seq;
  Q8Waits waits;
  bool vec, gate_vec;  // set at the launch: 16-byte accesses of x and out, of the gate
};
// Whether a launch takes the staged form on a device of `sms` SMs.
bool q8_combine_is_staged_bf16(const Q8CombineArgs& a, int sms);
bool q8_combine_is_staged_f32(const Q8CombineArgs& a, int sms);
cudaError_t launch_q8_combine_bf16(const Q8CombineArgs& a, bool e5, cudaStream_t s);
cudaError_t launch_q8_combine_f32(const Q8CombineArgs& a, bool e5, cudaStream_t s);

struct Q8MatmulArgs {
  Q8Rows a, b, out;
  bool a_e5, b_e5;
  int out_format, act, n_groups, n_cols;
  const int32_t *offsets, *dst;
  const float* bias;
  int32_t* status;
  Q8Waits waits;
};
cudaError_t launch_q8_matmul(const Q8MatmulArgs& a, cudaStream_t s);

}  // namespace moeca
