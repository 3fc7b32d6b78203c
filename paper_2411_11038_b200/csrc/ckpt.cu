// 8-bit activation checkpoints and the GELU that uses them: one streaming pass each.
//
//   store      x -> (codes, scales)             load       (codes, scales) -> x~
//   gelu fwd   x -> y [, (codes, scales)]       recompute  (codes, scales) -> gelu(x~)
//   gelu bwd   dY, x or (codes, scales) -> dX
//
// GELU: 1 - Phi(|x|) = P(t) t e / 2 with e = exp(-x^2 / 2), t = 1 / (1 + p |x| / sqrt 2) and the
// degree-4 polynomial P of Abramowitz & Stegun, Handbook of Mathematical Functions, 7.1.26 (absolute
// error of erf at most 1.5e-7).  The slope Phi(x) + x e / sqrt(2 pi) needs the same exponential, so
// either direction costs two special-function operations per element (a reciprocal and a power of
// two); the rest goes through the packed fp32 instructions, two elements to an issue slot.
#include "rowops.cuh"

namespace efqat {

namespace {

enum { ACT_NONE = 0, ACT_GELU = 1, ACT_GELU_BWD = 2 };

__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float ex2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// For two values: Phi(|x|) - 1/2 = 1/2 - P(t) t e / 2, and e = exp(-x^2 / 2) on the side.
__device__ __forceinline__ pair_t normal_half(pair_t x, pair_t& e) {
  const float c = 0.3275911f * 0.70710678118654752f;
  const float2 v = halves(x), z = halves(mul2(mul2(x, both(-0.5f * 1.4426950408889634f)), x));
  const pair_t t = pair_of(rcp_approx(fmaf(fabsf(v.x), c, 1.f)), rcp_approx(fmaf(fabsf(v.y), c, 1.f)));
  e = pair_of(ex2_approx(z.x), ex2_approx(z.y));
  pair_t p = fma2(both(-0.5f * 1.061405429f), t, both(0.5f * 1.453152027f));
  p = fma2(p, t, both(-0.5f * 1.421413741f));
  p = fma2(p, t, both(0.5f * 0.284496736f));
  p = fma2(p, t, both(-0.5f * 0.254829592f));
  return fma2(mul2(p, t), e, both(0.5f));
}
__device__ __forceinline__ pair_t with_signs(pair_t v, pair_t of) { return v | (of & 0x8000000080000000ull); }

// x Phi(x) with Phi(x) = 1/2 + sign(x) (Phi(|x|) - 1/2)
__device__ __forceinline__ pair_t gelu2(pair_t x) {
  pair_t e;
  const pair_t h = normal_half(x, e);
  return mul2(x, add2(with_signs(h, x), both(0.5f)));
}

// Phi(x) + x phi(x)
__device__ __forceinline__ pair_t gelu_slope2(pair_t x) {
  pair_t e;
  const pair_t h = normal_half(x, e);
  return add2(fma2(mul2(x, both(0.3989422804014327f)), e, both(0.5f)), with_signs(h, x));
}

struct RowArgs {
  const void* x; const int8_t* codes_in; const float* scales_in;
  const void* dy;
  void* y; int8_t* codes_out; float* scales_out;
  uint32_t C, G, groups;    // row length, groups per row, groups in all
};

// One warp per pair of groups (16 lanes a group), UNROLL pairs in flight.  SRC: 0 x itself, 1 its
// checkpoint.  HBM-bound: every tensor is touched once, with 16-byte (codes: 8-byte) accesses.
template <typename T, int SRC, int ACT, int SAVE>
__global__ void __launch_bounds__(256) ckpt_kernel(RowArgs a) {
  constexpr int UNROLL = 2;
  pdl_trigger();
  pdl_wait();
  const uint32_t half = (blockIdx.x * 256u + threadIdx.x) >> 4;     // half-warps: one group each
  const uint32_t halves = gridDim.x * 16u;
  const int l16 = threadIdx.x & 15;
  const bool ragged = (a.C % CKPT_GROUP) != 0;
  // (whole warps stay in the loop together: the group maximum is a shuffle over the warp)
  for (uint32_t g0 = half & ~1u; g0 < a.groups; g0 += halves * UNROLL) {
    Vec8<T> xv[UNROLL], dv[UNROLL];
    uint2 cv[UNROLL];
    float sc[UNROLL];
    int64_t at[UNROLL];
    bool ok[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const uint32_t g = g0 + (half & 1u) + u * halves;
      ok[u] = g < a.groups;
      if (ragged) {
        const uint32_t row = g / a.G, col = (g - row * a.G) * CKPT_GROUP + l16 * 8;
        ok[u] = ok[u] && col < a.C;
        at[u] = static_cast<int64_t>(row) * a.C + col;
      } else {
        at[u] = static_cast<int64_t>(g) * CKPT_GROUP + l16 * 8;
      }
      xv[u].zero();
      if (SRC == 0) {
        if (ok[u]) xv[u].load(static_cast<const T*>(a.x) + at[u]);
      } else {
        cv[u] = make_uint2(0u, 0u);
        sc[u] = 0.f;
        if (ok[u]) {
          cv[u] = *reinterpret_cast<const uint2*>(a.codes_in + at[u]);
          sc[u] = a.scales_in[g];
        }
      }
      if (ACT == ACT_GELU_BWD) {
        dv[u].zero();
        if (ok[u]) dv[u].load(static_cast<const T*>(a.dy) + at[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const uint32_t g = g0 + (half & 1u) + u * halves;
      pair_t v[4];
      if (SRC == 0) xv[u].get(v); else ckpt_values(cv[u], sc[u], v);
      if (SAVE) {
        const GroupScale gs = ckpt_group_scale(v);
        if (ok[u]) {
          *reinterpret_cast<uint2*>(a.codes_out + at[u]) = ckpt_codes(v, gs);
          if (l16 == 0) a.scales_out[g] = gs.scale;
        }
      }
      if (SAVE && ACT == ACT_NONE) continue;
      pair_t o[4];
      if (ACT == ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = v[i];
      } else if (ACT == ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = gelu2(v[i]);
      } else {
        pair_t d[4];
        dv[u].get(d);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = mul2(d[i], gelu_slope2(v[i]));
      }
      if (ok[u]) store8(static_cast<T*>(a.y) + at[u], o);
    }
  }
}

template <typename T, int SRC, int ACT, int SAVE>
void launch(const RowArgs& a, int sm_count, cudaStream_t st) {
  const int64_t blocks = ceil_div(a.groups, 16);
  const int64_t cap = static_cast<int64_t>(sm_count) * 8;
  count_launches(1);
  launch_dependent(ckpt_kernel<T, SRC, ACT, SAVE>, static_cast<unsigned>(blocks < cap ? blocks : cap), 256, 0, st, 1, a);
}

template <typename T>
void dispatch(const RowArgs& a, int act, int sm_count, cudaStream_t st) {
  const bool src = a.codes_in != nullptr, save = a.codes_out != nullptr;
  if (act == ACT_GELU_BWD) {
    if (src) launch<T, 1, ACT_GELU_BWD, 0>(a, sm_count, st); else launch<T, 0, ACT_GELU_BWD, 0>(a, sm_count, st);
  } else if (act == ACT_GELU) {
    if (src) launch<T, 1, ACT_GELU, 0>(a, sm_count, st);
    else if (save) launch<T, 0, ACT_GELU, 1>(a, sm_count, st);
    else launch<T, 0, ACT_GELU, 0>(a, sm_count, st);
  } else {
    if (src) launch<T, 1, ACT_NONE, 0>(a, sm_count, st); else launch<T, 0, ACT_NONE, 1>(a, sm_count, st);
  }
}

}  // namespace

void launch_ckpt(int dtype, int act, const void* x, const efqat_ckpt* in, const void* dy, int64_t M, int64_t C,
                 void* y, const efqat_ckpt* out, int sm_count, cudaStream_t st) {
  RowArgs a = {};
  a.x = x; a.dy = dy; a.y = y;
  if (in) { a.codes_in = in->codes; a.scales_in = in->scales; }
  if (out) { a.codes_out = out->codes; a.scales_out = out->scales; }
  a.C = static_cast<uint32_t>(C);
  a.G = static_cast<uint32_t>(ckpt_groups(C));
  a.groups = static_cast<uint32_t>(M * ckpt_groups(C));
  if (dtype == EFQAT_BF16) dispatch<bf16>(a, act, sm_count, st); else dispatch<float>(a, act, sm_count, st);
}

}  // namespace efqat
