// The paged cache of keys and values: new tokens into their pages, rotated and quantised on the way, and back out of them.
//
//   append   k~ = R(p) k, q~ = R(p) q (optional), v;  bf16: rounded.  e4m3: 2^-e x rounded, with the smallest e that brings the vector's largest
//            magnitude within 448
//   read     2^e times what is held, in bf16: exact
//
// Both move bytes and little else: two prompts of 8192 tokens (32 and 8 heads of 128, rotated) into an e4m3 cache in 92 us (0.37 GB, 4.0 TB/s), into a bf16
// one in 91 (4.4), back from e4m3 in 25 (0.10 GB, 4.0); one token in 3.6, the launch.  Two groups of vectors under way at a time take 92 us, one 94.5, four
// 92; in one loop over all groups, whose kind decides what is read from the kernel's arguments, it was 126.  A head's vector is dh / 8 lanes of 16 bytes, so
// a wave holds 4 to 16 vectors and the vector's largest magnitude and, for split pairs, the other member of a pair come from lane exchanges (DPP).  A wave
// takes a token's heads (or, of few tokens, a part of them), so that its angles are evaluated once: in fp64, one pair a lane, handed on through LDS as fp32.
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "lane_exchange.h"
#include "paged_cache.h"

namespace dl {

constexpr int kCacheWaves = 4;        // waves of a workgroup
constexpr int kAhead = 2;                 // groups of vectors that a wave has under way

// the largest over the LPR lanes of a vector, in every lane of it
template <int LPR>
__device__ __forceinline__ float vector_max(float x) {
  x = fmaxf(x, lane_xor<1>(x));
  x = fmaxf(x, lane_xor<2>(x));
  if constexpr (LPR >= 8) x = fmaxf(x, lane_xor<4>(x));
  if constexpr (LPR >= 16) x = fmaxf(x, lane_xor<8>(x));
  return x;
}

struct AppendArgs {
  PagedCache cache;
  const bf16_t* x[3];            // q (or null), k, v: [tokens][heads][DH]
  bf16_t* q_out;
  const int64_t *start, *lengths;
  int64_t tokens;
  int seq, heads[3], first[4];   // groups of 64 / LPR vectors: those of q from first[0], k, v, and their end
  int parts, per_part;           // a token's groups are dealt to `parts` waves
  double log2_base;
  int layout;                    // of the rotation's pairs, -1: no rotation
};

template <int DH, bool E4M3>
__global__ __launch_bounds__(64 * kCacheWaves) void append_kernel(const AppendArgs a) {
  constexpr int LPR = DH / 8, RPW = 64 / LPR;
  __shared__ float angle[kCacheWaves][2][DH / 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane % LPR, row = lane / LPR;
  const double theta = lane < DH / 2 ? exp2(-2.0 * (double)lane / (double)DH * a.log2_base) : 0.0;

  const int64_t tasks = a.tokens * a.parts, stride = (int64_t)gridDim.x * kCacheWaves;
  for (int64_t task = (int64_t)blockIdx.x * kCacheWaves + wave; task < tasks; task += stride) {
    const int64_t tok = task / a.parts;
    const int part = (int)(task % a.parts);
    const int64_t b = tok / a.seq;
    const int t = (int)(tok % a.seq);
    const bool valid = t < row_length(a.lengths, b, a.seq);
    const int64_t p = row_start(a.start, b) + t;
    const int page = valid ? page_of(a.cache, b, p) : -1;
    const int g0 = part * a.per_part, g1 = min(g0 + a.per_part, a.first[3]);
    float cs[8] = {}, sn[8] = {};
    if (valid && a.layout >= 0 && g0 < a.first[2]) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // the lanes are done with the angles of the token before
      if (lane < DH / 2) {
        double s, c;
        sincos((double)p * theta, &s, &c);
        angle[wave][0][lane] = (float)c;
        angle[wave][1][lane] = (float)s;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      // y[e] = x[e] cs[e] + partner[e] sn[e], with the sign of the rotation in sn
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = a.layout == 0 ? (lr * 8 + e) & (DH / 2 - 1) : lr * 4 + (e >> 1);
        const bool minus = a.layout == 0 ? lr < LPR / 2 : !(e & 1);
        cs[e] = angle[wave][0][i];
        sn[e] = minus ? -angle[wave][1][i] : angle[wave][1][i];
      }
    }
    // the groups of q (W 0), k and v, some of which are under way together
    const auto vectors = [&](auto WHICH, const bf16_t* x, int nh, int first, int last) {
      constexpr int W = decltype(WHICH)::value;
      for (int gi = max(g0, first); gi < min(g1, last); gi += kAhead) {
        bf16x8 xv[kAhead];
        int head[kAhead];
        int64_t at[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          head[i] = (gi + i - first) * RPW + row;
          at[i] = (tok * nh + head[i]) * DH + lr * 8;
          if (gi + i < min(g1, last) && head[i] < nh && valid && (W == 0 || page >= 0)) xv[i] = *reinterpret_cast<const bf16x8*>(x + at[i]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (gi + i >= min(g1, last) || head[i] >= nh) continue;
          if (!valid || (W > 0 && page < 0)) {
            const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
            if (W == 0) *reinterpret_cast<bf16x8*>(a.q_out + at[i]) = zero;
            continue;
          }
          float y[8];
          unpack8(xv[i], y);
          if (W < 2 && a.layout >= 0) {
            // each product rounded on its own: a fused multiply-add would round the two members of a pair differently, and the largest magnitude of
            // a vector decides its exponent
#pragma clang fp contract(off)
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (a.layout == 0 ? lane_xor<LPR / 2>(y[e]) : y[e ^ 1]) * sn[e];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = y[e] * cs[e] + z[e];
          }
          if constexpr (W == 0) {
            *reinterpret_cast<bf16x8*>(a.q_out + at[i]) = pack8(y);
          } else {
            const int64_t vec = vector_of(a.cache, page, head[i], p);
            char* out = a.cache.x[W - 1];
            if constexpr (!E4M3) {
              *reinterpret_cast<bf16x8*>(out + vec * DH * 2 + lr * 16) = pack8(y);
            } else {
              float amax = 0.f;
#pragma unroll
              for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(y[e]) < INFINITY ? fabsf(y[e]) : 0.f);
              const int ex = e4m3_exponent(vector_max<LPR>(amax));
              const float inv = power_of_two(-ex);
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] *= inv;
              if (ex >= kScaleMost)          // 256 * 2^120 is above the range of bf16
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fabsf(y[e]) < INFINITY ? fminf(fmaxf(y[e], -240.f), 240.f) : y[e];
              const u32x2 u = {pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7])};
              *reinterpret_cast<u32x2*>(out + vec * DH + lr * 8) = u;
              if (lr == 0) a.cache.scale[W - 1][vec] = (uint8_t)(ex + kScaleBias);
            }
          }
        }
      }
    };
    vectors(std::integral_constant<int, 0>{}, a.x[0], a.heads[0], 0, a.first[1]);
    vectors(std::integral_constant<int, 1>{}, a.x[1], a.heads[1], a.first[1], a.first[2]);
    vectors(std::integral_constant<int, 2>{}, a.x[2], a.heads[1], a.first[2], a.first[3]);
  }
}

// Workgroups, and waves to a token: a wave a token where there are tokens enough; of fewer, the heads are dealt out, one group of vectors a wave at the least.
constexpr int kCacheMostBlocks = 2048;
static void plan_token_parts(int64_t tokens, int groups, int& parts, int& per_part, int& blocks) {
  const int64_t waves = (int64_t)kCacheMostBlocks * kCacheWaves;
  int64_t n = tokens >= waves ? 1 : waves / tokens;
  if (n > groups) n = groups;
  per_part = (int)((groups + n - 1) / n);
  parts = (groups + per_part - 1) / per_part;
  const int64_t want = (tokens * parts + kCacheWaves - 1) / kCacheWaves;
  blocks = (int)(want < kCacheMostBlocks ? want : kCacheMostBlocks);
}

int launch_kv_cache_append(const CacheCall& c, const void* q, const void* k, const void* v, int64_t seq, int64_t Hq, float base, int layout,
                           void* q_out, hipStream_t st) {
  AppendArgs a{};
  a.cache = paged_cache(c);
  a.x[0] = (const bf16_t*)q; a.x[1] = (const bf16_t*)k; a.x[2] = (const bf16_t*)v;
  a.q_out = (bf16_t*)q_out;
  a.start = c.start; a.lengths = c.lengths;
  a.tokens = c.batch * seq; a.seq = (int)seq;
  a.heads[0] = q ? (int)Hq : 0; a.heads[1] = a.heads[2] = (int)c.heads;
  const int rows = 512 / (int)c.dh;
  for (int w = 0; w < 3; ++w) a.first[w + 1] = a.first[w] + (a.heads[w] + rows - 1) / rows;
  int blocks;
  plan_token_parts(a.tokens, a.first[3], a.parts, a.per_part, blocks);
  a.log2_base = base > 0.f ? log2((double)base) : 0.0;
  a.layout = base > 0.f ? layout : -1;
  const dim3 grid((unsigned)blocks), block(64 * kCacheWaves);
  if (c.e4m3) {
    if (c.dh == 128) hipLaunchKernelGGL((append_kernel<128, true>), grid, block, 0, st, a);
    else if (c.dh == 64) hipLaunchKernelGGL((append_kernel<64, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((append_kernel<32, true>), grid, block, 0, st, a);
  } else {
    if (c.dh == 128) hipLaunchKernelGGL((append_kernel<128, false>), grid, block, 0, st, a);
    else if (c.dh == 64) hipLaunchKernelGGL((append_kernel<64, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((append_kernel<32, false>), grid, block, 0, st, a);
  }
  return check_launch("kv_cache_append");
}

struct ReadArgs {
  PagedCache cache;
  bf16_t* out[2];                // k, v: [tokens][heads][DH]
  const int64_t *start, *lengths;
  int64_t vectors;               // tokens * heads
  int seq;
};

template <int DH, bool E4M3>
__global__ __launch_bounds__(64 * kCacheWaves) void read_kernel(const ReadArgs a) {
  constexpr int LPR = DH / 8;
  const int lr = threadIdx.x % LPR;
  const int64_t stride = (int64_t)gridDim.x * (64 * kCacheWaves / LPR);
  for (int64_t i = (int64_t)blockIdx.x * (64 * kCacheWaves / LPR) + threadIdx.x / LPR; i < a.vectors; i += stride) {
    const int64_t tok = i / a.cache.heads, b = tok / a.seq;
    const int head = (int)(i % a.cache.heads), t = (int)(tok % a.seq);
    const int64_t p = row_start(a.start, b) + t;
    const int page = t < row_length(a.lengths, b, a.seq) ? page_of(a.cache, b, p) : -1;
    bf16x8 y[2] = {};
    if (page >= 0) {
      const int64_t vec = vector_of(a.cache, page, head, p);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if constexpr (E4M3)
          y[w] = unpack_e4m3(*reinterpret_cast<const u32x2*>(a.cache.x[w] + vec * DH + lr * 8), power_of_two((int)a.cache.scale[w][vec] - kScaleBias));
        else y[w] = *reinterpret_cast<const bf16x8*>(a.cache.x[w] + (vec * DH + lr * 8) * 2);
      }
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) *reinterpret_cast<bf16x8*>(a.out[w] + i * DH + lr * 8) = y[w];
  }
}

int launch_kv_cache_read(const CacheCall& c, int64_t seq, void* k, void* v, hipStream_t st) {
  ReadArgs a{};
  a.cache = paged_cache(c);
  a.out[0] = (bf16_t*)k; a.out[1] = (bf16_t*)v;
  a.start = c.start; a.lengths = c.lengths;
  a.seq = (int)seq;
  a.vectors = c.batch * seq * c.heads;
  const int64_t per = 64 * kCacheWaves / (c.dh / 8), want = (a.vectors + per - 1) / per;
  const dim3 grid((unsigned)(want < kCacheMostBlocks ? want : kCacheMostBlocks)), block(64 * kCacheWaves);
  if (c.e4m3) {
    if (c.dh == 128) hipLaunchKernelGGL((read_kernel<128, true>), grid, block, 0, st, a);
    else if (c.dh == 64) hipLaunchKernelGGL((read_kernel<64, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((read_kernel<32, true>), grid, block, 0, st, a);
  } else {
    if (c.dh == 128) hipLaunchKernelGGL((read_kernel<128, false>), grid, block, 0, st, a);
    else if (c.dh == 64) hipLaunchKernelGGL((read_kernel<64, false>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((read_kernel<32, false>), grid, block, 0, st, a);
  }
  return check_launch("kv_cache_read");
}

}  // namespace dl
