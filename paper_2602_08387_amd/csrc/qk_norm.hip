// RMS norm of every query and key head and the rotary embedding in one pass, and its gradient.
//
//   forward   z = x rstd gamma,  rstd = (mean x^2 + eps)^(-1/2) over the head's dh values;  y = R(p) z
//   backward  dz = R(-p) dy;  dgamma = sum dz x rstd;  dxh = dz gamma;  dx = rstd (dxh - x rstd mean(dxh x rstd))
//
// Both are bound by HBM: 4 bytes an element forward, 6 backward; 16384 tokens of 32 and 8 heads of 128 in 70 us (0.34 GB, 4.8 TB/s) and 102 (0.51 GB, 5.1 TB/s
// in the kernel's 98, and the gains' sums), one token in 3.3, the launch.  A head's row is dh / 8 lanes of 16 bytes, so a wave holds
// 4 to 16 rows and everything a row needs stays within 4 to 16 lanes: the mean and, for split pairs, the other member of a
// pair come from lane exchanges in the register file (DPP), not through LDS.  A wave takes a token (or, of few tokens, a part of its
// heads), so that the token's angles are evaluated once: in fp64, one pair a lane, handed to the lanes that need them through LDS as fp32.
#include "common.h"
#include "kernels.h"

namespace dl {

constexpr int kQkWaves = 4;   // waves of a workgroup

// x of lane l ^ M, within 16 lanes
template <int M>
__device__ __forceinline__ int lane_xor(int x) {
  if constexpr (M == 1) return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true);        // quad_perm 1, 0, 3, 2
  else if constexpr (M == 2) return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true);   // quad_perm 2, 3, 0, 1
  else if constexpr (M == 4) return __builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);   // mirrored in 8 lanes, then in 4
  else return __builtin_amdgcn_mov_dpp(x, 0x128, 0xf, 0xf, true);                        // rotated by 8 of 16
}
template <int M>
__device__ __forceinline__ float lane_xor(float x) { return __int_as_float(lane_xor<M>(__float_as_int(x))); }
template <int M>
__device__ __forceinline__ bf16x8 lane_xor(const bf16x8& v) {
  const u32x4 u = __builtin_bit_cast(u32x4, v);
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)lane_xor<M>((int)u[i]);
  return __builtin_bit_cast(bf16x8, r);
}
// sum over the LPR lanes of a row, in every lane of it
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
  x += lane_xor<1>(x);
  x += lane_xor<2>(x);
  if constexpr (LPR >= 8) x += lane_xor<4>(x);
  if constexpr (LPR >= 16) x += lane_xor<8>(x);
  return x;
}

struct QkNormArgs {
  const bf16_t *x[2];            // q, k [tokens][heads][DH]
  const bf16_t *gamma[2];
  const bf16_t *dy[2];           // backward
  bf16_t *out[2];                // q_out, k_out, or dq, dk
  float *rstd[2];                // written by the forward (may be null), read by the backward
  float *partial[2];             // backward: a row of DH sums for every workgroup
  const int64_t *start, *lengths;
  int64_t tokens;
  int seq, heads[2], groups[2];  // groups: of 64 / LPR rows
  int parts, per_part;           // a token's groups are dealt to `parts` waves
  double log2_base;
  float eps;
  int layout;
};

// What a lane keeps of its token's angles: y[e] = x[e] c[e] + partner[e] s[e] for its 8 elements (partner: the other member of
// the element's pair), with the sign of the rotation and its direction in s.
template <int DH>
__device__ __forceinline__ void load_angles(const float* cs, const float* sn, int layout, bool inverse, int lr, float (&c)[8], float (&s)[8]) {
  const bool second = layout == 0 && lr >= DH / 16;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = layout == 0 ? (lr * 8 + e) & (DH / 2 - 1) : lr * 4 + (e >> 1);
    c[e] = cs[i];
    const bool minus = (layout == 0 ? !second : !(e & 1)) != inverse;
    s[e] = minus ? -sn[i] : sn[i];
  }
}

template <int DH, bool BWD>
__global__ __launch_bounds__(64 * kQkWaves) void qk_norm_kernel(const QkNormArgs a) {
  constexpr int LPR = DH / 8, RPW = 64 / LPR;
  __shared__ float angle[kQkWaves][2][DH / 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane % LPR, row = lane / LPR;
  float* cs = angle[wave][0];
  float* sn = angle[wave][1];
  const double theta = lane < DH / 2 ? exp2(-2.0 * (double)lane / (double)DH * a.log2_base) : 0.0;
  float g[2][8];
#pragma unroll
  for (int w = 0; w < 2; ++w) unpack8(*reinterpret_cast<const bf16x8*>(a.gamma[w] + lr * 8), g[w]);
  float dg[2][8] = {};

  const int64_t tasks = a.tokens * a.parts, stride = (int64_t)gridDim.x * kQkWaves;
  for (int64_t task = (int64_t)blockIdx.x * kQkWaves + wave; task < tasks; task += stride) {
    const int64_t tok = task / a.parts;
    const int part = (int)(task % a.parts);
    const int64_t b = tok / a.seq;
    const int t = (int)(tok % a.seq);
    const bool valid = !a.lengths || t < a.lengths[b];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the lanes are done with the angles of the token before
    if (valid && lane < DH / 2) {
      const double p = (double)(t + (a.start ? a.start[b] : 0));
      double s, c;
      sincos(p * theta, &s, &c);
      cs[lane] = (float)c;
      sn[lane] = (float)s;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float c[8], s[8];
    load_angles<DH>(cs, sn, a.layout, BWD, lr, c, s);
    const int g0 = part * a.per_part, g1 = min(g0 + a.per_part, a.groups[0] + a.groups[1]);
    for (int gi = g0; gi < g1; ++gi) {
      const int w = gi >= a.groups[0];
      const int head = (gi - (w ? a.groups[0] : 0)) * RPW + row;
      const int nh = w ? a.heads[1] : a.heads[0];
      if (head >= nh) continue;
      const int64_t r = tok * nh + head, at = r * DH + lr * 8;
      bf16_t* out = (w ? a.out[1] : a.out[0]) + at;
      float* rstd = w ? a.rstd[1] : a.rstd[0];
      float y[8];
      if (!valid) {
        const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
        *reinterpret_cast<bf16x8*>(out) = zero;
        if (!BWD && rstd && lr == 0) rstd[r] = 0.f;
        continue;
      }
      const bf16x8 xv = *reinterpret_cast<const bf16x8*>((w ? a.x[1] : a.x[0]) + at);
      float x[8];
      unpack8(xv, x);
      if constexpr (!BWD) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += x[e] * x[e];
        const float rs = 1.0f / sqrtf(row_sum<LPR>(ss) / (float)DH + a.eps);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = x[e] * rs * (w ? g[1][e] : g[0][e]);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = z[e] * c[e] + (a.layout == 0 ? lane_xor<LPR / 2>(z[e]) : z[e ^ 1]) * s[e];
        if (rstd && lr == 0) rstd[r] = rs;
      } else {
        const bf16x8 dv = *reinterpret_cast<const bf16x8*>((w ? a.dy[1] : a.dy[0]) + at);
        const float rs = rstd[r];
        float d[8], o[8], dxh[8], m = 0.f;
        unpack8(dv, d);
        if (a.layout == 0) unpack8(lane_xor<LPR / 2>(dv), o);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = d[e ^ 1];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float dz = d[e] * c[e] + o[e] * s[e];
          x[e] *= rs;
          if (w) dg[1][e] += dz * x[e];
          else dg[0][e] += dz * x[e];
          dxh[e] = dz * (w ? g[1][e] : g[0][e]);
          m += dxh[e] * x[e];
        }
        m = row_sum<LPR>(m) / (float)DH;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = rs * (dxh[e] - x[e] * m);
      }
      *reinterpret_cast<bf16x8*>(out) = pack8(y);
    }
  }
  if constexpr (BWD) {
    // a workgroup's partial row: the rows of a wave by lane exchanges, then the waves in order
    __shared__ float red[kQkWaves][2][DH];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = dg[w][e];
#pragma unroll
        for (int o = LPR; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
        if (row == 0) red[wave][w][lr * 8 + e] = v;
      }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * DH; i += 64 * kQkWaves) {
      const int w = i / DH, col = i % DH;
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < kQkWaves; ++k) v += red[k][w][col];
      (w ? a.partial[1] : a.partial[0])[(int64_t)blockIdx.x * DH + col] = v;
    }
  }
}

// Workgroups, and waves to a token: a wave a token where there are tokens enough for kQkMostBlocks workgroups; of fewer tokens the heads
// are dealt out, one group of rows a wave at the least.
constexpr int kQkMostBlocks = 1024;
struct QkPlan { int groups[2], parts, per_part, blocks; };
static QkPlan qk_plan(int64_t tokens, int64_t Hq, int64_t Hkv, int64_t dh) {
  QkPlan p;
  const int64_t rows = 512 / dh;
  p.groups[0] = (int)((Hq + rows - 1) / rows);
  p.groups[1] = (int)((Hkv + rows - 1) / rows);
  const int64_t groups = p.groups[0] + p.groups[1], waves = (int64_t)kQkMostBlocks * kQkWaves;
  int64_t parts = tokens >= waves ? 1 : waves / tokens;
  if (parts > groups) parts = groups;
  p.per_part = (int)((groups + parts - 1) / parts);
  p.parts = (int)((groups + p.per_part - 1) / p.per_part);
  const int64_t blocks = (tokens * p.parts + kQkWaves - 1) / kQkWaves;
  p.blocks = (int)(blocks < kQkMostBlocks ? blocks : kQkMostBlocks);
  return p;
}

static QkNormArgs qk_args(const QkNormCall& c, const QkPlan& p) {
  QkNormArgs a{};
  a.x[0] = (const bf16_t*)c.q; a.x[1] = (const bf16_t*)c.k;
  a.gamma[0] = (const bf16_t*)c.gamma_q; a.gamma[1] = (const bf16_t*)c.gamma_k;
  a.rstd[0] = c.rstd_q; a.rstd[1] = c.rstd_k;
  a.start = c.start; a.lengths = c.lengths;
  a.tokens = c.batch * c.seq; a.seq = (int)c.seq;
  a.heads[0] = (int)c.Hq; a.heads[1] = (int)c.Hkv;
  a.groups[0] = p.groups[0]; a.groups[1] = p.groups[1];
  a.parts = p.parts; a.per_part = p.per_part;
  a.log2_base = log2((double)c.base);
  a.layout = c.layout;
  return a;
}

int launch_qk_norm_rope_fwd(const QkNormCall& c, float eps, void* q_out, void* k_out, hipStream_t st) {
  const QkPlan p = qk_plan(c.batch * c.seq, c.Hq, c.Hkv, c.dh);
  QkNormArgs a = qk_args(c, p);
  a.out[0] = (bf16_t*)q_out; a.out[1] = (bf16_t*)k_out;
  a.eps = eps;
  const dim3 grid((unsigned)p.blocks), block(64 * kQkWaves);
  if (c.dh == 128) hipLaunchKernelGGL((qk_norm_kernel<128, false>), grid, block, 0, st, a);
  else if (c.dh == 64) hipLaunchKernelGGL((qk_norm_kernel<64, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((qk_norm_kernel<32, false>), grid, block, 0, st, a);
  return check_launch("qk_norm_rope_forward");
}

// the most that a plan of so many tokens, or fewer, has: a size that does not fall as the call grows
size_t qk_norm_rope_bwd_workspace(int64_t tokens, int64_t Hq, int64_t Hkv, int64_t dh) {
  const QkPlan p = qk_plan(1, Hq, Hkv, dh);
  const int64_t waves = tokens * (p.groups[0] + p.groups[1]), blocks = (waves + kQkWaves - 1) / kQkWaves;
  return (size_t)(blocks < kQkMostBlocks ? blocks : kQkMostBlocks) * 2 * dh * sizeof(float);
}

int launch_qk_norm_rope_bwd(const QkNormCall& c, const void* dq_out, const void* dk_out, void* dq, void* dk, void* dgamma_q,
                            void* dgamma_k, int accumulate, void* workspace, hipStream_t st) {
  const QkPlan p = qk_plan(c.batch * c.seq, c.Hq, c.Hkv, c.dh);
  QkNormArgs a = qk_args(c, p);
  a.dy[0] = (const bf16_t*)dq_out; a.dy[1] = (const bf16_t*)dk_out;
  a.out[0] = (bf16_t*)dq; a.out[1] = (bf16_t*)dk;
  a.partial[0] = (float*)workspace; a.partial[1] = (float*)workspace + (int64_t)p.blocks * c.dh;
  const dim3 grid((unsigned)p.blocks), block(64 * kQkWaves);
  if (c.dh == 128) hipLaunchKernelGGL((qk_norm_kernel<128, true>), grid, block, 0, st, a);
  else if (c.dh == 64) hipLaunchKernelGGL((qk_norm_kernel<64, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((qk_norm_kernel<32, true>), grid, block, 0, st, a);
  if (int rc = check_launch("qk_norm_rope_backward")) return rc;
  return launch_gain_sums(GainSums{a.partial[0], a.partial[1], dgamma_q, dgamma_k, p.blocks, (int)c.dh, accumulate}, st);
}

}  // namespace dl
