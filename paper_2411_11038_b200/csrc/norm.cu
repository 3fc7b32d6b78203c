// Layer norm over the rows of a dense matrix: forward, backward with the reduction of the
// parameters' gradients, and the forward again from an 8-bit checkpoint.
//
//   y  = (x - mean) rstd gamma + beta
//   g  = dY gamma,  xh = (x - mean) rstd,  dX = rstd (g - mean_c(g) - xh mean_c(g xh))
//   dgamma = sum_m dY xh,  dbeta = sum_m dY
//
// A row belongs to a team of `team` warps, each lane holding NV vectors of 8 columns in registers,
// so every tensor is read and written once.  Rows of up to a warp's reach need shuffles only;
// wider ones exchange one partial sum per warp through shared memory.  The variance is formed from
// the centred values (no cancellation for rows far from zero).
#include "rowops.cuh"

namespace efqat {

namespace {

static const int NORM_THREADS = 512;    // most threads of a block

struct NormArgs {
  const void* x; const int8_t* codes_in; const float* scales_in;
  const void* dy; const float* gamma; const float* beta; float eps;
  void* y; float* mean; float* rstd;                      // y: dX in the backward
  int8_t* codes_out; float* scales_out;
  float* part;                                            // backward: [gridDim.x][2][C] partial dgamma, dbeta
  int64_t M;
  int C, G, team;                                         // columns, checkpoint groups per row, warps per row
};

// Sum of two values over a team.  Teams of one warp: shuffles.  Larger teams are whole blocks.
// `slot` alternates so that one barrier per exchange is enough.
__device__ __forceinline__ float2 team_sum(float2 v, int team, float2* s_red, int& slot) {
  v.x = warp_sum(v.x);
  v.y = warp_sum(v.y);
  if (team == 1) return v;
  float2* red = s_red + slot * 32;
  slot ^= 1;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float2 t = make_float2(0.f, 0.f);
  for (int w = 0; w < team; ++w) {
    const float2 o = red[w];
    t.x += o.x;
    t.y += o.y;
  }
  return t;
}

template <typename T, int NV, int SRC, int SAVE>
__global__ void __launch_bounds__(NORM_THREADS) norm_fwd_kernel(NormArgs a) {
  __shared__ float2 s_red[64];
  pdl_trigger();
  pdl_wait();
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int teams = warps / a.team;                     // 1 when a team has several warps
  const int tl = a.team == 1 ? lane : threadIdx.x;      // lane within the team
  const int stride = a.team * 32 * 8;
  int slot = 0;
  const float inv_c = 1.f / static_cast<float>(a.C);
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * teams + (a.team == 1 ? warp : 0); row < a.M;
       row += static_cast<int64_t>(gridDim.x) * teams) {
    float v[NV][8];
    const int64_t base = row * a.C;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = tl * 8 + j * stride;
      if (SRC == 0) {
        Vec8<T> r;
        r.zero();
        if (c < a.C) r.load(static_cast<const T*>(a.x) + base + c);
        r.get(v[j]);
      } else {
        uint2 w = make_uint2(0u, 0u);
        float s = 0.f;
        if (c < a.C) {
          w = *reinterpret_cast<const uint2*>(a.codes_in + base + c);
          s = a.scales_in[row * a.G + c / CKPT_GROUP];
        }
        ckpt_values(w, s, v[j]);
      }
    }
    float mean, rstd;
    if (SRC == 0) {
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) s.x += v[j][i];
      mean = team_sum(s, a.team, s_red, slot).x * inv_c;
      s = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        if (tl * 8 + j * stride < a.C) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float d = v[j][i] - mean;
            s.x = fmaf(d, d, s.x);
          }
        }
      }
      const float var = team_sum(s, a.team, s_red, slot).x * inv_c;
      rstd = 1.f / sqrtf(var + a.eps);
      if (tl == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
      }
    } else {
      mean = a.mean[row];
      rstd = a.rstd[row];
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = tl * 8 + j * stride;
      if (SAVE) {
        const GroupScale gs = ckpt_group_scale(v[j]);
        if (c < a.C) {
          *reinterpret_cast<uint2*>(a.codes_out + base + c) = ckpt_codes(v[j], gs);
          if ((tl & 15) == 0) a.scales_out[row * a.G + c / CKPT_GROUP] = gs.scale;
        }
      }
      if (c < a.C) {
        float o[8], gm[8], bt[8];
        Vec8<float> p;
        p.load(a.gamma + c);
        p.get(gm);
        if (a.beta) p.load(a.beta + c); else p.zero();
        p.get(bt);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = fmaf((v[j][i] - mean) * rstd, gm[i], bt[i]);
        store8(static_cast<T*>(a.y) + base + c, o);
      }
    }
  }
}

// Backward.  A block keeps the running dgamma / dbeta of its rows in registers (each lane owns the
// same columns in every row) and writes one partial row of each at the end.
template <typename T, int NV, int SRC>
__global__ void __launch_bounds__(NORM_THREADS) norm_bwd_kernel(NormArgs a) {
  __shared__ float2 s_red[64];
  extern __shared__ float s_part[];      // teams > 1: [teams][2][C]
  pdl_trigger();
  pdl_wait();
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int teams = warps / a.team;
  const int tl = a.team == 1 ? lane : threadIdx.x;
  const int stride = a.team * 32 * 8;
  int slot = 0;
  const float inv_c = 1.f / static_cast<float>(a.C);
  float dg[NV][8], db[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[j][i] = db[j][i] = 0.f;
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * teams + (a.team == 1 ? warp : 0); row < a.M;
       row += static_cast<int64_t>(gridDim.x) * teams) {
    const int64_t base = row * a.C;
    float xh[NV][8], d[NV][8];
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = tl * 8 + j * stride;
      Vec8<T> r;
      r.zero();
      if (c < a.C) r.load(static_cast<const T*>(a.dy) + base + c);
      r.get(d[j]);
      if (SRC == 0) {
        r.zero();
        if (c < a.C) r.load(static_cast<const T*>(a.x) + base + c);
        r.get(xh[j]);
      } else {
        uint2 w = make_uint2(0u, 0u);
        float s = 0.f;
        if (c < a.C) {
          w = *reinterpret_cast<const uint2*>(a.codes_in + base + c);
          s = a.scales_in[row * a.G + c / CKPT_GROUP];
        }
        ckpt_values(w, s, xh[j]);
      }
    }
    float2 s = make_float2(0.f, 0.f);      // sums of g and g xh
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = tl * 8 + j * stride;
      if (c < a.C) {
        float gm[8];
        Vec8<float> p;
        p.load(a.gamma + c);
        p.get(gm);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          xh[j][i] = (xh[j][i] - mean) * rstd;
          dg[j][i] = fmaf(d[j][i], xh[j][i], dg[j][i]);
          db[j][i] += d[j][i];
          d[j][i] *= gm[i];
          s.x += d[j][i];
          s.y = fmaf(d[j][i], xh[j][i], s.y);
        }
      }
    }
    s = team_sum(s, a.team, s_red, slot);
    const float c1 = s.x * inv_c, c2 = s.y * inv_c;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = tl * 8 + j * stride;
      if (c < a.C) {
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = rstd * (d[j][i] - fmaf(xh[j][i], c2, c1));
        store8(static_cast<T*>(a.y) + base + c, o);
      }
    }
  }
  float* out = a.part + static_cast<int64_t>(blockIdx.x) * 2 * a.C;
  if (teams == 1) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = tl * 8 + j * stride;
      if (c < a.C) {
        store8(out + c, dg[j]);
        store8(out + a.C + c, db[j]);
      }
    }
    return;
  }
  float* mine = s_part + static_cast<int64_t>(warp) * 2 * a.C;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = tl * 8 + j * stride;
    if (c < a.C) {
      store8(mine + c, dg[j]);
      store8(mine + a.C + c, db[j]);
    }
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * a.C; c += blockDim.x) {
    float t = 0.f;
    for (int w = 0; w < teams; ++w) t += s_part[static_cast<int64_t>(w) * 2 * a.C + c];
    out[c] = t;
  }
}

// dgamma / dbeta: columns of the [parts][2 C] partial sums.  8 threads per column, fixed order.
__global__ void __launch_bounds__(256) norm_reduce_kernel(const float* __restrict__ part, int parts, int C,
                                                          float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float s[8][33];
  pdl_trigger();
  pdl_wait();
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + cx;
  float t = 0.f;
  if (c < 2 * C)
    for (int r = ry; r < parts; r += 8) t += part[static_cast<int64_t>(r) * 2 * C + c];
  s[ry][cx] = t;
  __syncthreads();
  if (ry == 0 && c < 2 * C) {
    for (int r = 1; r < 8; ++r) t += s[r][cx];
    if (c < C) dgamma[c] = t; else dbeta[c - C] = t;
  }
}

// Warps per row and vectors per lane for a reach of `most` vectors.
struct Shape {
  int team, nv;
};
Shape row_shape(int64_t C, int most) {
  Shape s;
  s.team = static_cast<int>(ceil_div(C, 256 * most));
  s.nv = static_cast<int>(ceil_div(C, 256 * s.team));
  return s;
}

static const int FWD_NV = 4, BWD_NV = 4;

template <typename T, int NV>
void fwd_nv(const NormArgs& a, unsigned grid, unsigned block, cudaStream_t st) {
  count_launches(1);
  if (a.codes_in) launch_dependent(norm_fwd_kernel<T, NV, 1, 0>, grid, block, 0, st, 1, a);
  else if (a.codes_out) launch_dependent(norm_fwd_kernel<T, NV, 0, 1>, grid, block, 0, st, 1, a);
  else launch_dependent(norm_fwd_kernel<T, NV, 0, 0>, grid, block, 0, st, 1, a);
}

template <typename T>
void fwd_t(const NormArgs& a, int nv, unsigned grid, unsigned block, cudaStream_t st) {
  switch (nv) {
    case 1: fwd_nv<T, 1>(a, grid, block, st); break;
    case 2: fwd_nv<T, 2>(a, grid, block, st); break;
    case 3: fwd_nv<T, 3>(a, grid, block, st); break;
    default: fwd_nv<T, 4>(a, grid, block, st); break;
  }
}

template <typename T, int NV>
void bwd_nv(const NormArgs& a, unsigned grid, unsigned block, size_t smem, cudaStream_t st) {
  count_launches(1);
  if (a.codes_in) launch_dependent(norm_bwd_kernel<T, NV, 1>, grid, block, smem, st, 1, a);
  else launch_dependent(norm_bwd_kernel<T, NV, 0>, grid, block, smem, st, 1, a);
}

template <typename T>
void bwd_t(const NormArgs& a, int nv, unsigned grid, unsigned block, size_t smem, cudaStream_t st) {
  switch (nv) {
    case 1: bwd_nv<T, 1>(a, grid, block, smem, st); break;
    case 2: bwd_nv<T, 2>(a, grid, block, smem, st); break;
    case 3: bwd_nv<T, 3>(a, grid, block, smem, st); break;
    default: bwd_nv<T, 4>(a, grid, block, smem, st); break;
  }
}

struct BwdPlan {
  int team, nv, warps, grid;
};
BwdPlan bwd_plan(int64_t M, int64_t C, int sm_count) {
  const Shape s = row_shape(C, BWD_NV);
  BwdPlan p;
  p.team = s.team; p.nv = s.nv;
  p.warps = s.team == 1 ? 4 : s.team;
  const int64_t teams = s.team == 1 ? 4 : 1;
  const int64_t need = ceil_div(M, teams), cap = static_cast<int64_t>(sm_count) * (s.team <= 4 ? 2 : 1);
  p.grid = static_cast<int>(need < cap ? need : cap);
  return p;
}

NormArgs norm_args(const void* x, const efqat_ckpt* in, int64_t M, int64_t C, int team) {
  NormArgs a = {};
  a.x = x;
  if (in) { a.codes_in = in->codes; a.scales_in = in->scales; }
  a.M = M;
  a.C = static_cast<int>(C);
  a.G = static_cast<int>(ckpt_groups(C));
  a.team = team;
  return a;
}

}  // namespace

size_t layer_norm_workspace_bytes(int64_t M, int64_t C, int sm_count) {
  return M > 0 ? static_cast<size_t>(bwd_plan(M, C, sm_count).grid) * 2 * C * 4 : 0;
}

void launch_norm_fwd(int dtype, const void* x, const efqat_ckpt* in, int64_t M, int64_t C, const float* gamma,
                     const float* beta, float eps, void* y, float* mean, float* rstd, const efqat_ckpt* out,
                     int sm_count, cudaStream_t st) {
  const Shape s = row_shape(C, FWD_NV);
  NormArgs a = norm_args(x, in, M, C, s.team);
  a.gamma = gamma; a.beta = beta; a.eps = eps;
  a.y = y; a.mean = mean; a.rstd = rstd;
  if (out) { a.codes_out = out->codes; a.scales_out = out->scales; }
  const int warps = s.team == 1 ? 4 : s.team;
  const int64_t need = ceil_div(M, s.team == 1 ? 4 : 1);
  const int64_t cap = static_cast<int64_t>(sm_count) * (32 / warps > 0 ? 32 / warps : 1);
  const unsigned grid = static_cast<unsigned>(need < cap ? need : cap);
  if (dtype == EFQAT_BF16) fwd_t<bf16>(a, s.nv, grid, warps * 32, st);
  else fwd_t<float>(a, s.nv, grid, warps * 32, st);
}

void launch_norm_bwd(int dtype, const void* dy, const void* x, const efqat_ckpt* in, int64_t M, int64_t C,
                     const float* gamma, const float* mean, const float* rstd, void* dx, float* dgamma, float* dbeta,
                     float* part, int sm_count, cudaStream_t st) {
  const BwdPlan p = bwd_plan(M, C, sm_count);
  NormArgs a = norm_args(x, in, M, C, p.team);
  a.dy = dy; a.gamma = gamma;
  a.y = dx; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.part = part;
  const size_t smem = p.team == 1 ? static_cast<size_t>(p.warps) * 2 * C * 4 : 0;     // at most 4 * 2 * 1024 * 4 = 32 KB
  if (dtype == EFQAT_BF16) bwd_t<bf16>(a, p.nv, p.grid, p.warps * 32, smem, st);
  else bwd_t<float>(a, p.nv, p.grid, p.warps * 32, smem, st);
  count_launches(1);
  launch_dependent(norm_reduce_kernel, static_cast<unsigned>(ceil_div(2 * C, 32)), 256, 0, st, 1,
                   static_cast<const float*>(part), p.grid, static_cast<int>(C), dgamma, dbeta);
}

}  // namespace efqat
