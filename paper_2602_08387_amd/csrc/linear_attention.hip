// Linear attention with a decay for each KV head: S_t = lambda S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t, and its gradient.
#include "common.h"
#include "kernels.h"

namespace dl {

// The logarithm of a decay, minus infinity (no memory at all) made finite: times no token it is to give 0, not NaN.
__device__ __forceinline__ double decay_log(float g) { return g < -1e30f ? -1e30 : (double)g; }
// The decay of one token as the sum of two fp32: rounded to one, a state of n tokens' memory would be off by up to 6e-8 n.
struct Decay { float hi, lo; };
__device__ __forceinline__ Decay decay_of(float g) {
  const double d = exp(decay_log(g));
  const float hi = (float)d;
  return Decay{hi, (float)(d - (double)hi)};
}
// lambda s + x
__device__ __forceinline__ float decayed(const Decay& l, float s, float x) { return __builtin_fmaf(s, l.hi, __builtin_fmaf(s, l.lo, x)); }

// One token after the other.  Workgroup: 16 columns of the state of one (batch row, KV head); thread: one of them in D / 16 rows.
//   forward   S = lambda S + a b^T;                out_h = mult S^T x_h for the group's heads h
//   REVERSE   R = lambda R + mult sum_h x_h y_h^T, from the last token to the first; out = R^T a
// with b and y of the workgroup's 16 columns.  s_in is transposed if `flip`.
struct RecurrentArgs {
  const bf16_t *a, *b, *x, *y;
  bf16_t* out;
  const float *log_decay, *s_in;
  float* s_out;
  const int64_t* lengths;
  int seq, Hq, Hkv, flip;
  float mult;
};
template <int D, bool REVERSE>
__global__ __launch_bounds__(256) void linear_recurrent_kernel(const RecurrentArgs p) {
  constexpr int R = D / 16;
  __shared__ float red[4][16];
  const int pair = blockIdx.x, b = pair / p.Hkv, j = pair % p.Hkv, G = p.Hq / p.Hkv, col = (int)blockIdx.y * 16;
  const int c = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const Decay lam = decay_of(p.log_decay[j]);
  int64_t len = p.lengths ? p.lengths[b] : p.seq;
  len = len < 0 ? 0 : len > p.seq ? p.seq : len;
  float s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = i * 16 + rg;
    s[i] = !p.s_in ? 0.f : p.s_in[(int64_t)pair * D * D + (p.flip ? (col + c) * D + row : row * D + col + c)];
  }
  auto reduce = [&](float v) {
    v += __shfl_xor(v, 16, 64);
    v += __shfl_xor(v, 32, 64);
    __syncthreads();
    if ((threadIdx.x & 63) < 16) red[wave][c] = v;
    __syncthreads();
    return (red[0][c] + red[1][c]) + (red[2][c] + red[3][c]);
  };
  for (int n = 0; n < p.seq; ++n) {
    const int t = REVERSE ? p.seq - 1 - n : n;
    const int64_t kv = (((int64_t)b * p.seq + t) * p.Hkv + j) * D, q = (((int64_t)b * p.seq + t) * p.Hq + (int64_t)j * G) * D;
    if (t >= len) {
      if (rg == 0) {
        if (REVERSE) p.out[kv + col + c] = (bf16_t)0.f;
        else for (int h = 0; h < G; ++h) p.out[q + (int64_t)h * D + col + c] = (bf16_t)0.f;
      }
      continue;
    }
    if constexpr (!REVERSE) {
      const float bv = (float)p.b[kv + col + c];
#pragma unroll
      for (int i = 0; i < R; ++i) s[i] = decayed(lam, s[i], (float)p.a[kv + i * 16 + rg] * bv);
      for (int h = 0; h < G; ++h) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) v += s[i] * (float)p.x[q + (int64_t)h * D + i * 16 + rg];
        v = reduce(v);
        if (rg == 0) p.out[q + (int64_t)h * D + col + c] = (bf16_t)(v * p.mult);
      }
    } else {
      if (t < len - 1)
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = decayed(lam, s[i], 0.f);
      for (int h = 0; h < G; ++h) {
        const float y = (float)p.y[q + (int64_t)h * D + col + c] * p.mult;
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] += (float)p.x[q + (int64_t)h * D + i * 16 + rg] * y;
      }
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < R; ++i) v += s[i] * (float)p.a[kv + i * 16 + rg];
      v = reduce(v);
      if (rg == 0) p.out[kv + col + c] = (bf16_t)v;
    }
  }
  if (p.s_out)
#pragma unroll
    for (int i = 0; i < R; ++i) p.s_out[(int64_t)pair * D * D + (i * 16 + rg) * D + col + c] = REVERSE && len > 0 ? decayed(lam, s[i], 0.f) : s[i];
}

template <bool REVERSE>
static int launch_recurrent(const RecurrentArgs& a, int64_t pairs, int64_t dh, hipStream_t st) {
  const dim3 grid((unsigned)pairs, (unsigned)(dh / 16)), block(256);
  if (dh == 128) hipLaunchKernelGGL((linear_recurrent_kernel<128, REVERSE>), grid, block, 0, st, a);
  else if (dh == 64) hipLaunchKernelGGL((linear_recurrent_kernel<64, REVERSE>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((linear_recurrent_kernel<32, REVERSE>), grid, block, 0, st, a);
  return check_launch("linear attention");
}

size_t linear_attention_fwd_workspace(int64_t B, int64_t S, int64_t Hq, int64_t Hkv, int64_t dh) { return 256; }
size_t linear_attention_bwd_workspace(int64_t B, int64_t S, int64_t Hq, int64_t Hkv, int64_t dh) { return 256; }

int launch_linear_attention_fwd(const LinearCall& c, const float* s_in, void* o, float* s_out, void* workspace, hipStream_t st) {
  RecurrentArgs a{};
  a.a = (const bf16_t*)c.k; a.b = (const bf16_t*)c.v; a.x = (const bf16_t*)c.q; a.out = (bf16_t*)o;
  a.log_decay = c.log_decay; a.s_in = s_in; a.s_out = s_out; a.lengths = c.lengths;
  a.seq = (int)c.S; a.Hq = (int)c.Hq; a.Hkv = (int)c.Hkv; a.mult = c.scale;
  return launch_recurrent<false>(a, c.B * c.Hkv, c.dh, st);
}

int launch_linear_attention_bwd(const LinearCall& c, const float* s_in, const void* d_o, const float* ds_out, void* dq, void* dk, void* dv,
                                float* ds_in, void* workspace, hipStream_t st) {
  RecurrentArgs a{};
  a.log_decay = c.log_decay; a.lengths = c.lengths;
  a.seq = (int)c.S; a.Hq = (int)c.Hq; a.Hkv = (int)c.Hkv; a.mult = c.scale;
  a.a = (const bf16_t*)c.v; a.b = (const bf16_t*)c.k; a.x = (const bf16_t*)d_o; a.out = (bf16_t*)dq; a.s_in = s_in; a.flip = 1;
  if (int rc = launch_recurrent<false>(a, c.B * c.Hkv, c.dh, st)) return rc;
  a.x = (const bf16_t*)d_o; a.y = (const bf16_t*)c.q; a.out = (bf16_t*)dk; a.s_in = ds_out;
  if (int rc = launch_recurrent<true>(a, c.B * c.Hkv, c.dh, st)) return rc;
  a.a = (const bf16_t*)c.k; a.x = (const bf16_t*)c.q; a.y = (const bf16_t*)d_o; a.out = (bf16_t*)dv; a.s_out = ds_in; a.flip = 0;
  return launch_recurrent<true>(a, c.B * c.Hkv, c.dh, st);
}

// ------------------------------------------------------------------------------------------
// One token for every batch row.  Bound by HBM: the state is read and written once, 8 bytes an element.  Workgroup: COLS columns of
// one state; a thread holds four columns of every RG-th row, so that the state stays in registers between its update and the products
// with the group's queries.
// ------------------------------------------------------------------------------------------
template <int D, int COLS>
__global__ __launch_bounds__(256) void linear_step_kernel(const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v,
                                                          const float* __restrict__ log_decay, const int64_t* __restrict__ lengths,
                                                          float* __restrict__ state, int Hq, int Hkv, float scale, bf16_t* __restrict__ o) {
  constexpr int CV = COLS / 4, RG = 256 / CV, R = (D + RG - 1) / RG;
  __shared__ f32x4 red[4][CV];
  const int pair = blockIdx.x, b = pair / Hkv, j = pair % Hkv, G = Hq / Hkv, col = (int)blockIdx.y * COLS;
  const int cv = threadIdx.x % CV, rg = threadIdx.x / CV, wave = threadIdx.x >> 6, c = col + cv * 4;
  const bf16_t* qp = q + ((int64_t)b * Hq + (int64_t)j * G) * D;
  bf16_t* op = o + ((int64_t)b * Hq + (int64_t)j * G) * D;
  if (lengths && lengths[b] <= 0) {
    const bf16x4 zero = {0, 0, 0, 0};
    if (rg == 0)
      for (int h = 0; h < G; ++h) *reinterpret_cast<bf16x4*>(op + (int64_t)h * D + c) = zero;
    return;
  }
  const Decay lam = decay_of(log_decay[j]);
  const bf16_t* kp = k + (int64_t)pair * D;
  const bf16x4 vv = *reinterpret_cast<const bf16x4*>(v + (int64_t)pair * D + c);
  float* sp = state + (int64_t)pair * D * D + c;
  f32x4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (D % RG == 0 || i * RG + rg < D) s[i] = *reinterpret_cast<const f32x4*>(sp + (i * RG + rg) * D);
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (D % RG == 0 || i * RG + rg < D) {
      const float kk = (float)kp[i * RG + rg];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = decayed(lam, s[i][e], kk * (float)vv[e]);
      *reinterpret_cast<f32x4*>(sp + (i * RG + rg) * D) = s[i];
    }
  for (int h = 0; h < G; ++h) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (D % RG == 0 || i * RG + rg < D) acc += s[i] * (float)qp[(int64_t)h * D + i * RG + rg];
#pragma unroll
    for (int off = CV; off < 64; off <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) < CV) red[wave][cv] = acc;
    __syncthreads();
    if (threadIdx.x < CV) {
      const f32x4 t = ((red[0][cv] + red[1][cv]) + (red[2][cv] + red[3][cv])) * scale;
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (bf16_t)t[e];
      *reinterpret_cast<bf16x4*>(op + (int64_t)h * D + c) = w;
    }
  }
}

int launch_linear_attention_step(const LinearCall& c, float* state, void* o, hipStream_t st) {
  const int64_t pairs = c.B * c.Hkv;
#define STEP(D, COLS)                                                                                                          \
  hipLaunchKernelGGL((linear_step_kernel<D, COLS>), dim3((unsigned)pairs, D / COLS), dim3(256), 0, st, (const bf16_t*)c.q,      \
                     (const bf16_t*)c.k, (const bf16_t*)c.v, c.log_decay, c.lengths, state, (int)c.Hq, (int)c.Hkv, c.scale, (bf16_t*)o)
  if (c.dh == 128) STEP(128, 32);
  else if (c.dh == 64) STEP(64, 32);
  else STEP(32, 32);
#undef STEP
  return check_launch("linear_attention_step");
}

}  // namespace dl
