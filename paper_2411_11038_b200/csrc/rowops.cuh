// Element access and 8-bit checkpoint arithmetic shared by the row kernels (ckpt.cu, norm.cu).
//
// A checkpoint keeps 128 consecutive elements of a row as 8-bit codes of one scale.  Sixteen
// neighbouring lanes hold a group, 8 elements each: its largest magnitude is a maximum over
// 8 registers and 4 shuffles, its codes leave as one 8-byte store per lane.
#pragma once
#include "internal.h"

namespace efqat {

static const int CKPT_GROUP = 128;

__host__ __device__ inline int64_t ckpt_groups(int64_t C) { return ceil_div(C, CKPT_GROUP); }

// 8 consecutive elements <-> fp32 registers (16-byte accesses).
template <typename T>
struct Vec8;
template <>
struct Vec8<bf16> {
  uint4 r;
  __device__ __forceinline__ void load(const bf16* p) { r = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { r = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
template <>
struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// Scale and multiplier of the group that this lane's 16-lane half of the warp holds.  The largest
// magnitude is taken over the bit patterns, where infinity and NaN rank above every finite value.
// Every lane of the warp has to take part.
struct GroupScale {
  float scale, factor;     // value of one code step; multiplier that decides the codes
};
__device__ __forceinline__ GroupScale ckpt_group_scale(const float (&v)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float a = __uint_as_float(top);
  GroupScale g;
  if (top >= 0x7f800000u) {
    g.scale = __uint_as_float(0x7fffffffu);
    g.factor = 0.f;
  } else if (a < 7.888609052210118e-31f) {     // 2^-100: 127 / a would leave the range of fp32 further down
    g.scale = 0.f;
    g.factor = 0.f;
  } else {
    g.scale = __fdiv_rn(a, 127.f);
    g.factor = __fdiv_rn(127.f, a);
  }
  return g;
}

// The 8 codes of a lane as two words.  Adding 1.5 * 2^23 rounds to nearest-even and leaves the code
// in the low byte of the sum's bit pattern (two's complement), so no conversion instruction is used.
__device__ __forceinline__ uint2 ckpt_codes(const float (&v)[8], const GroupScale& g) {
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(__fadd_rn(__fmul_rn(v[i], g.factor), 12582912.f));
  uint2 w;
  w.x = __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
  w.y = __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410);
  if (g.factor == 0.f) w = make_uint2(0u, 0u);     // zeros, or a non-finite group (infinity * 0 is no code)
  return w;
}

// The values that 8 codes stand for.  A code byte with its top bit flipped, placed in the mantissa
// of 2^23, is 2^23 + 128 + code: one subtraction instead of an integer conversion.
__device__ __forceinline__ void ckpt_values(uint2 w, float scale, float (&v)[8]) {
  const uint32_t x[2] = {w.x ^ 0x80808080u, w.y ^ 0x80808080u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    v[i] = __fmul_rn(__uint_as_float(__byte_perm(x[i >> 2], 0x4b000000u, 0x7440 | (i & 3))) - 8388736.f, scale);
}

}  // namespace efqat
