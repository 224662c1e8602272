// Log-probabilities of given tokens under rows of bf16 logits, with each row's entropy and its likeliest tokens; and the gradient.
//
//   z = x / temperature, M = max z, S = sum exp(z - M), U = sum exp(z - M) (z - M):
//   lse = M + ln S;  logp(v) = (z_v - M) - ln S;  entropy = ln S - U / S                          (no difference of large numbers)
//   dx_v = ([v = target] dlp - p_v (dlp + dH (logp_v + entropy))) / temperature
//
// Forward: one pass, bound by the reading of the logits (2 bytes each; some 11 issue slots of the vector units an element, of which the exponential takes four). A thread
// keeps S and U relative to its own running maximum, which it raises once in 32 elements.  Exponents are formed as (x - max) times a constant: of a row that
// is all but certain S is then 1 and a little, exactly, where one FMA against the rounded product max * constant would be off by that rounding (and infinite
// for a row masked with the type's lowest value).
//
// The likeliest tokens: a wave keeps a list of 64 sorted over its lanes.  An element has to pass the list's n-th, and a bound that the workgroup's waves
// share: at first the n-th largest of the threads' maxima over their first 32 elements, then the least of what the waves have as their (n / 4)-th.  The few
// that pass go to a buffer in LDS and from there into the list, one by one or sorted 64 at a time.  An order without ties: a 64-bit key of the logit's bits
// as a whole number of the same order, then the lower index.
//
// Few rows are cut into parts, joined by a second kernel.
//
// Measured, 128256 tokens a row: 4096 rows 186 us without the likeliest (1.05 GB, 5.6 TB/s: memory), 216 with 5, 250 with 20, 292 with 64 (vector
// instructions); one row 13.7 with 20 (two launches, 8.4 and 5.4 us: loads, exchanges and barriers one after the other).  The gradient of 4096 rows 395 us
// (2.1 GB, 5.3 TB/s: memory).
#include "common.h"
#include "kernels.h"
#include "lane_exchange.h"

namespace dl {

constexpr int kLpGradThreads = 256, kLpUnroll = 4;
constexpr int kLpBuffer = 64 + 512;      // candidates of a wave: those that wait, and a whole vector from every lane
constexpr int kLpSingly = 24;           // candidates that go into the list one by one (11 instructions each; sorting 64 takes some 300)
constexpr float kLpLn2 = 0.6931471805599453f;

struct LogprobsArgs {
  const bf16_t* logits;
  const int64_t* targets;                // null: every row counts
  int64_t ld;
  int V, parts, per_part, n_top;         // per_part: vectors of 8
  float inverse, inverse_log2e;
  float *logprobs, *entropy, *lse, *top_logprobs;   // each may be null
  int64_t* top_ids;
  float* part_sums;                      // [row][part][4]: maximum (of x), S, U (in log2 units)
  uint64_t* part_top;                    // [row][part][n_top]
};

__device__ __forceinline__ bool row_counts(const LogprobsArgs& a, int64_t row) {
  if (!a.targets) return true;
  const int64_t t = a.targets[row];
  return t >= 0 && t < a.V;
}

// The logit of a row's target; asked for early, since it takes two loads one after the other.
__device__ __forceinline__ float scored_logit(const LogprobsArgs& a, int64_t row) {
  return a.logprobs ? (float)a.logits[row * a.ld + a.targets[row]] : 0.f;
}

// Keys: larger for a larger logit, for equal ones for the lower index; 0 is below every key.  -0 and 0 are equal.
__device__ __forceinline__ uint64_t key_of(uint32_t bits, int index) {
  const int s = (int)(int16_t)bits, order = s >= 0 ? s : -32768 - s;
  return (uint64_t)(uint32_t)(order + 65536) << 32 | (0xffffffffu - (uint32_t)index);
}
__device__ __forceinline__ int key_index(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }
__device__ __forceinline__ float key_logit(uint64_t key) {
  const int order = (int)(key >> 32) - 65536;
  return __uint_as_float((uint32_t)(uint16_t)(order >= 0 ? order : -32768 - order) << 16);
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

// One step of a bitonic sort: of lanes l and l ^ J the larger in the lane without J's bit; turned round where `turned`.
template <int J, typename T>
__device__ __forceinline__ T sort_step(T k, int lane, bool turned) {
  const T o = lane_xor<J>(k);
  return (o > k) == (((lane & J) != 0) != turned) ? k : o;
}
// A bitonic sequence over N lanes into order.
template <int N, typename T>
__device__ __forceinline__ T merge_step(T k, int lane, bool turned) {
  k = sort_step<N / 2>(k, lane, turned);
  if constexpr (N > 2) k = merge_step<N / 2>(k, lane, turned);
  return k;
}
// 64 lanes into descending order: keys, or floats that are not NaN.
template <typename T>
__device__ __forceinline__ T sort_descending(T k, int lane) {
  k = merge_step<2>(k, lane, (lane & 2) != 0);
  k = merge_step<4>(k, lane, (lane & 4) != 0);
  k = merge_step<8>(k, lane, (lane & 8) != 0);
  k = merge_step<16>(k, lane, (lane & 16) != 0);
  k = merge_step<32>(k, lane, (lane & 32) != 0);
  return merge_step<64>(k, lane, false);
}
// The 64 largest of two descending sequences, descending.
__device__ __forceinline__ uint64_t join_descending(uint64_t a, uint64_t b, int lane) {
  return merge_step<64>(max64(a, __shfl(b, 63 - lane, 64)), lane, false);
}

struct Sums { float m, s, u; };          // maximum of x, S and U relative to it; m = -inf: nothing but -inf so far

// Sums relative to another maximum.
__device__ __forceinline__ Sums relative_to(const Sums& v, float top, float inverse_log2e) {
  if (v.m == -INFINITY) return {top, v.s, v.u};        // zeros, or NaN
  const float d = fmaxf((v.m - top) * inverse_log2e, -1e4f);
  const float f = __builtin_amdgcn_exp2f(d);
  return {top, f * v.s, f * (v.u + d * v.s)};
}

// A row's results from its sums; scored: its target's logit; list: its likeliest, one a lane of the calling wave.
__device__ __forceinline__ void finish_row(const LogprobsArgs& a, int64_t row, float scored, const Sums& v, uint64_t list, int lane) {
  const bool empty = v.m == -INFINITY && v.s == 0.f;    // nothing but -inf
  const float log_s = empty ? 0.f : logf(v.s);
  const auto logp = [&](float x) { return x == -INFINITY ? (v.s == v.s ? -INFINITY : v.s) : (x - v.m) * a.inverse - log_s; };
  if (lane == 0) {
    if (a.logprobs) a.logprobs[row] = logp(scored);
    if (a.entropy) a.entropy[row] = empty ? 0.f : log_s - kLpLn2 * (v.u / v.s);
    if (a.lse) a.lse[row] = empty ? -INFINITY : v.m * a.inverse + log_s;
  }
  if (lane < a.n_top) {
    if (a.top_ids) a.top_ids[row * a.n_top + lane] = list ? key_index(list) : -1;
    if (a.top_logprobs) a.top_logprobs[row * a.n_top + lane] = list ? logp(key_logit(list)) : NAN;
  }
}
__device__ __forceinline__ void finish_uncounted(const LogprobsArgs& a, int64_t row) {
  if (threadIdx.x == 0) {
    if (a.logprobs) a.logprobs[row] = 0.f;
    if (a.entropy) a.entropy[row] = 0.f;
    if (a.lse) a.lse[row] = 0.f;
  }
  if ((int)threadIdx.x < a.n_top) {
    if (a.top_ids) a.top_ids[row * a.n_top + threadIdx.x] = -1;
    if (a.top_logprobs) a.top_logprobs[row * a.n_top + threadIdx.x] = 0.f;
  }
}

// A float that is not NaN as a whole number of the same order, and back.
__device__ __forceinline__ int ordered(float x) { const int i = (int)__float_as_uint(x); return i ^ ((i >> 31) & 0x7fffffff); }
__device__ __forceinline__ float from_ordered(int i) { return __uint_as_float((uint32_t)(i ^ ((i >> 31) & 0x7fffffff))); }

// A wave's list of the likeliest, with the buffer in front of it.
struct TopList {
  uint64_t list = 0;                     // descending over the lanes
  uint64_t* buffer;
  int held = 0;                          // in the buffer
  bool full = false;                     // whether the list has n
  float last = -INFINITY;                // its n-th
  float least = -INFINITY;               // what an element has to be to enter

  // An element equal to the list's n-th comes behind it, since a wave's indices ascend.  bound: n elements of the row's part are not below it; one that is equal may
  // be among them.
  __device__ __forceinline__ void raise(float bound) { least = full ? fmaxf(bound, from_ordered(ordered(last) + 1)) : bound; }
  __device__ __forceinline__ void push(bool take, uint32_t bits, int index, int lane) {
    const uint64_t who = __builtin_amdgcn_ballot_w64(take);
    if (who == 0) return;
    if (take) buffer[held + __popcll(who & ((1ull << lane) - 1))] = key_of(bits, index);
    held += __popcll(who);
  }
  __device__ __forceinline__ void drain(int lane, int n_top) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
    for (int i = 0; i < held; i += 64) {
      const int n = min(held - i, 64);
      const uint64_t key = lane < n ? buffer[i + lane] : 0;
      if (n > kLpSingly) {
        list = join_descending(list, sort_descending(key, lane), lane);
      } else {
        // one after the other: the smaller ones move up a lane, the key takes the place of the first of them
        for (int k = 0; k < n; ++k) {
          const uint64_t one = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), k) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)key, k);
          const uint64_t up = (uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(0, (int)(list >> 32), 0x138, 0xf, 0xf, false) << 32 |
                              (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)list, 0x138, 0xf, 0xf, false);
          const uint64_t above = __builtin_amdgcn_ballot_w64(list > one);
          list = list > one ? list : lane == __popcll(above) ? one : up;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    held = 0;
    const uint64_t nth = __shfl(list, n_top - 1, 64);
    full = nth != 0;
    if (full) last = key_logit(nth);
  }
};

// WAVES: of a workgroup.  One wave takes a short part alone, without waiting for others and without joining their lists (64 rows of 32000, 20 likeliest: 13.8
// us, 16.7 with four); of longer parts, or with many likeliest to sort, four share the work and their bounds.  Registers for five waves a SIMD: for six
// some go to memory (4096 rows of 128256, 5 likeliest 4 % slower; 64 likeliest 3 % faster).
template <bool TOP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 5) void logprobs_kernel(const LogprobsArgs a) {
  constexpr int kLpWaves = WAVES, kLpThreads = 64 * WAVES;
  __shared__ float red[kLpWaves][4];
  __shared__ int bound, quarter[kLpWaves];   // the largest of the waves' n-th, and the (n / 4)-th of each
  __shared__ float maxima[TOP ? kLpWaves : 1][64];
  __shared__ uint64_t lists[TOP ? kLpWaves : 1][64];
  __shared__ uint64_t buffer[TOP ? kLpWaves : 1][TOP ? kLpBuffer : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x / a.parts;
  const int part = (int)(blockIdx.x % a.parts);
  if (!row_counts(a, row)) {
    if (a.parts == 1) finish_uncounted(a, row);
    return;
  }
  const u32x4* in = reinterpret_cast<const u32x4*>(a.logits + row * a.ld);
  const int whole = a.V >> 3, vectors = (a.V + 7) >> 3;          // the last vector may hold columns behind the vocabulary
  const int first = part * a.per_part, end = min(vectors, first + a.per_part);
  Sums v{-INFINITY, 0.f, 0.f};
  TopList top;
  top.buffer = buffer[TOP ? wave : 0];
  bool begun = false;
  const int few = WAVES == 1 ? 64 : a.n_top >> 1;    // candidates that wait for others
  const bool all_begin = first + (kLpWaves - 1) * 64 < end;
  if constexpr (TOP) {
    if (threadIdx.x == 0) bound = ordered(-INFINITY);
    if (threadIdx.x < kLpWaves) quarter[threadIdx.x] = ordered(-INFINITY);
    __syncthreads();
  }

  for (int c0 = first + wave * 64; c0 < end; c0 += kLpThreads * kLpUnroll) {
    u32x4 w[kLpUnroll];
#pragma unroll
    for (int i = 0; i < kLpUnroll; ++i) {
      const int c = c0 + i * kLpThreads + lane;
      w[i] = c < end ? in[c] : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};      // -inf
      if (c == whole) {                  // columns behind the vocabulary
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c * 8 + e >= a.V) w[i][e >> 1] = (e & 1) ? (w[i][e >> 1] & 0xffffu) | 0xff800000u : (w[i][e >> 1] & 0xffff0000u) | 0xff80u;
      }
    }
    const auto logit = [&](int i, int e) { return __uint_as_float((e & 1) ? w[i][e >> 1] & 0xffff0000u : w[i][e >> 1] << 16); };
    // the largest, one instruction for two elements, which lets NaN through; a wave that has one looks again without
    float vmax[kLpUnroll], mx;
#pragma unroll
    for (int i = 0; i < kLpUnroll; ++i) {
      vmax[i] = logit(i, 0);
#pragma unroll
      for (int e = 1; e < 8; ++e) vmax[i] = __builtin_elementwise_maximum(vmax[i], logit(i, e));
      mx = i ? __builtin_elementwise_maximum(mx, vmax[i]) : vmax[i];
    }
    if (__builtin_amdgcn_ballot_w64(mx != mx)) {
#pragma unroll
      for (int i = 0; i < kLpUnroll; ++i) {
        vmax[i] = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) vmax[i] = fmaxf(vmax[i], logit(i, e));
        mx = i ? fmaxf(mx, vmax[i]) : vmax[i];
      }
    }
    if (mx > v.m) v = relative_to(v, mx, a.inverse_log2e);
    const float ref = v.m == -INFINITY ? 0.f : v.m;
    // S in parts: every addition to a sum loses up to 2^-24 of it (rows of 128256, a spread of 4: entropies off by 0.9e-6 at the most, 2.4e-6 one by one)
    float part_s;
#pragma unroll
    for (int i = 0; i < kLpUnroll; ++i)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float t0 = (logit(i, e) - ref) * a.inverse_log2e, p0 = __builtin_amdgcn_exp2f(t0);
        const float t1 = (logit(i, e + 1) - ref) * a.inverse_log2e, p1 = __builtin_amdgcn_exp2f(t1);
        part_s = i + e == 0 ? p0 + p1 : part_s + (p0 + p1);
        v.u = __builtin_fmaf(p0, fmaxf(t0, -1e4f), v.u);         // t may be -inf where p is 0
        v.u = __builtin_fmaf(p1, fmaxf(t1, -1e4f), v.u);
      }
    v.s += part_s;
    if constexpr (TOP) {
      // the first bound: the n-th largest of the threads' largest, or, of a part too short for all waves, of the wave's lanes'.  A wave's bounds hold for all
      if (!begun) {
        float largest = sort_descending(mx, lane);
        if (WAVES > 1 && all_begin) {
          maxima[wave][lane] = largest;
          __syncthreads();
#pragma unroll
          for (int i = 1; i < kLpWaves; ++i) largest = merge_step<64>(fmaxf(largest, maxima[(wave + i) % kLpWaves][63 - lane]), lane, false);
        }
        const float nth = __shfl(largest, a.n_top - 1, 64);
        if (lane == 0) __hip_atomic_fetch_max(&bound, ordered(nth), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        begun = true;
      }
      // n elements are not below what one wave has as its n-th, nor below the least of what the four have as their (n / 4)-th
      int known = __hip_atomic_load(&quarter[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
#pragma unroll
      for (int i = 1; i < kLpWaves; ++i) known = min(known, __hip_atomic_load(&quarter[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP));
      top.raise(from_ordered(max(known, __hip_atomic_load(&bound, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP))));
      if (__builtin_amdgcn_ballot_w64(mx >= top.least)) {
        static_assert(kLpUnroll == 4, "vectors in turn");
        u32x4 x = w[0], x1 = w[1], x2 = w[2], x3 = w[3];
        float m0 = vmax[0], m1 = vmax[1], m2 = vmax[2], m3 = vmax[3];
#pragma unroll 1
        for (int c = c0 + lane; c < c0 + lane + kLpUnroll * kLpThreads; c += kLpThreads) {       // a loop: one copy of the code
          if (__builtin_amdgcn_ballot_w64(m0 >= top.least)) {
            const int left = c < end ? a.V - c * 8 : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t bits = (x[e >> 1] >> ((e & 1) * 16)) & 0xffffu;
              top.push(__uint_as_float(bits << 16) >= top.least && e < left, bits, c * 8 + e, lane);
            }
            if (top.held > few) {
              top.drain(lane, a.n_top);
              const uint64_t part = __shfl(top.list, (a.n_top - 1) / kLpWaves, 64);
              if (part != 0 && lane == 0) __hip_atomic_store(&quarter[wave], ordered(key_logit(part)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
              if (top.full) {
                top.raise(top.least);
                if (lane == 0) __hip_atomic_fetch_max(&bound, ordered(top.last), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
              }
            }
          }
          x = x1; x1 = x2; x2 = x3;
          m0 = m1; m1 = m2; m2 = m3;
        }
      }
    }
  }
  // the waves' sums and lists, joined by the first wave
  const float mw = wave_max(v.m);
  Sums r = relative_to(v, mw, a.inverse_log2e);
  r.s = wave_sum(r.s);
  r.u = wave_sum(r.u);
  if (lane == 0) { red[wave][0] = mw; red[wave][1] = r.s; red[wave][2] = r.u; }
  if constexpr (TOP) {
    if (top.held > 0) top.drain(lane, a.n_top);
    lists[wave][lane] = top.list;
  }
  __syncthreads();
  if (wave != 0) return;
  float m = red[0][0];
#pragma unroll
  for (int i = 1; i < kLpWaves; ++i) m = fmaxf(m, red[i][0]);
  Sums sum{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kLpWaves; ++i) {
    const Sums o{red[i][0], red[i][1], red[i][2]}, p = relative_to(o, m, a.inverse_log2e);
    sum.s += p.s;
    sum.u += p.u;
  }
  uint64_t list = 0;
  if constexpr (TOP) {
    list = top.list;
#pragma unroll
    for (int i = 1; i < kLpWaves; ++i) list = join_descending(list, lists[i][lane], lane);
  }
  if (a.parts == 1) {
    finish_row(a, row, scored_logit(a, row), sum, list, lane);
  } else {
    const int64_t at = row * a.parts + part;
    if (lane == 0) *reinterpret_cast<f32x4*>(a.part_sums + at * 4) = f32x4{sum.m, sum.s, sum.u, 0.f};
    if (TOP && lane < a.n_top) a.part_top[at * a.n_top + lane] = list;
  }
}

// Joins the parts of a row: a workgroup a row, whose waves take some lists each and then halve their number; the last wave joins the sums.  What can be asked
// for without knowing more is asked for first: the time is that of loads and exchanges one after the other.
constexpr int kLpJoinWaves = 16;
template <bool TOP>
__global__ __launch_bounds__(64 * kLpJoinWaves) void logprobs_join_kernel(const LogprobsArgs a) {
  __shared__ uint64_t lists[TOP ? kLpJoinWaves / 2 : 1][64];
  __shared__ float joined[3];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int64_t row = blockIdx.x;
  uint64_t some[4];
  const uint64_t* from = a.part_top + row * a.parts * a.n_top + lane;
  const auto load = [&](int i0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) some[k] = lane < a.n_top && i0 + k * waves < a.parts ? from[(int64_t)(i0 + k * waves) * a.n_top] : 0;
  };
  if constexpr (TOP) load(wave);
  const f32x4* parts = reinterpret_cast<const f32x4*>(a.part_sums) + row * a.parts;
  const f32x4 own = wave == waves - 1 && lane < a.parts ? parts[lane] : f32x4{-INFINITY, 0.f, 0.f, 0.f};
  if (!row_counts(a, row)) {
    finish_uncounted(a, row);
    return;
  }
  const float scored = wave == 0 ? scored_logit(a, row) : 0.f;
  if (wave == waves - 1) {
    float m = own[0];
    for (int i = lane + 64; i < a.parts; i += 64) m = fmaxf(m, parts[i][0]);
    m = wave_max(m);
    Sums sum = relative_to(Sums{own[0], own[1], own[2]}, m, a.inverse_log2e);
    for (int i = lane + 64; i < a.parts; i += 64) {
      const Sums p = relative_to(Sums{parts[i][0], parts[i][1], parts[i][2]}, m, a.inverse_log2e);
      sum.s += p.s;
      sum.u += p.u;
    }
    sum.s = wave_sum(sum.s);
    sum.u = wave_sum(sum.u);
    if (lane == 0) { joined[0] = m; joined[1] = sum.s; joined[2] = sum.u; }
  }
  uint64_t list = 0;
  if constexpr (TOP) {
    for (int i0 = wave; i0 < a.parts; i0 += 4 * waves) {
      if (i0 != wave) load(i0);
#pragma unroll
      for (int k = 0; k < 4; ++k) list = join_descending(list, some[k], lane);
    }
    for (int half = waves / 2; half > 0; half /= 2) {
      if (wave >= half && wave < 2 * half) lists[wave - half][lane] = list;
      __syncthreads();
      if (wave < half) list = join_descending(list, lists[wave][lane], lane);
      __syncthreads();
    }
  } else {
    __syncthreads();
  }
  if (wave == 0) finish_row(a, row, scored, Sums{joined[0], joined[1], joined[2]}, list, lane);
}

// Parts of a row: where there are fewer rows than fill the chip, of no less than four vectors a lane of a wave.
constexpr int64_t kLpWorkgroups = 1024;
static int64_t lp_most_parts(int64_t V) { return (V + 2047) / 2048; }

// sums and lists of the parts; rows * parts is within kLpWorkgroups wherever there are parts
static int64_t lp_parts_held(int64_t T, int64_t V) {
  const int64_t n = T < kLpWorkgroups ? T * lp_most_parts(V) : kLpWorkgroups;
  return n < kLpWorkgroups ? n : kLpWorkgroups;
}
size_t token_logprobs_workspace(int64_t T, int64_t V, int64_t n_top) { return (size_t)lp_parts_held(T, V) * (16 + 8 * (size_t)n_top); }

int launch_token_logprobs_fwd(const LogprobsCall& c, int n_top, float* logprobs, float* entropy, float* lse, int64_t* top_ids, float* top_logprobs,
                              void* workspace, hipStream_t st) {
  LogprobsArgs a{};
  a.logits = (const bf16_t*)c.logits;
  a.targets = c.targets;
  a.ld = c.ld;
  a.V = (int)c.V;
  a.inverse = c.inverse_temperature;
  a.inverse_log2e = (float)((double)c.inverse_temperature * 1.4426950408889634);
  a.logprobs = logprobs; a.entropy = entropy; a.lse = lse;
  a.top_ids = top_ids; a.top_logprobs = top_logprobs;
  a.n_top = n_top;
  const int64_t most = lp_most_parts(c.V), wanted = kLpWorkgroups / c.T, vectors = (c.V + 7) / 8;
  const int64_t parts = wanted < 1 ? 1 : wanted < most ? wanted : most;
  a.per_part = (int)((vectors + parts - 1) / parts);
  a.parts = (int)((vectors + a.per_part - 1) / a.per_part);
  a.part_sums = (float*)workspace;
  a.part_top = (uint64_t*)((char*)workspace + 16 * lp_parts_held(c.T, c.V));
  const dim3 grid((unsigned)(c.T * a.parts));
  const bool alone = a.per_part <= 512 && n_top <= 32;            // vectors: two batches of a wave
  if (n_top && alone) hipLaunchKernelGGL((logprobs_kernel<true, 1>), grid, dim3(64), 0, st, a);
  else if (n_top) hipLaunchKernelGGL((logprobs_kernel<true, 4>), grid, dim3(256), 0, st, a);
  else if (alone) hipLaunchKernelGGL((logprobs_kernel<false, 1>), grid, dim3(64), 0, st, a);
  else hipLaunchKernelGGL((logprobs_kernel<false, 4>), grid, dim3(256), 0, st, a);
  if (int rc = check_launch("token_logprobs_forward")) return rc;
  if (a.parts == 1) return 0;
  const dim3 joining(!n_top ? 64 : a.parts > 16 ? 64 * kLpJoinWaves : 256);
  if (n_top) hipLaunchKernelGGL((logprobs_join_kernel<true>), dim3((unsigned)c.T), joining, 0, st, a);
  else hipLaunchKernelGGL((logprobs_join_kernel<false>), dim3((unsigned)c.T), joining, 0, st, a);
  return check_launch("token_logprobs_forward, joining parts");
}

struct LogprobsGradArgs {
  const bf16_t* logits;
  bf16_t* dlogits;                       // may be logits: a vector is read by the thread that writes it, before it does
  const int64_t* targets;
  const float *lse, *entropy, *d_logprobs, *d_entropy;   // the last two: one may be null
  int64_t ld;
  int V, blocks;                         // workgroups of a row
  float inverse;
};
constexpr float kLpNothing = -1e30f;     // the lse of a row of which a mask (-infinity, or the type's lowest value) has left nothing

__global__ __launch_bounds__(kLpGradThreads) void logprobs_grad_kernel(const LogprobsGradArgs a) {
  const int64_t row = blockIdx.x / a.blocks;
  const int c0 = (int)(blockIdx.x % a.blocks) * (kLpGradThreads * kLpUnroll) + threadIdx.x;
  const int64_t tgt = a.targets ? a.targets[row] : 0;
  const float lse = a.lse[row];
  const bool counts = tgt >= 0 && tgt < a.V && !(lse <= kLpNothing);
  const float dlp = a.d_logprobs ? a.d_logprobs[row] : 0.f, dh = a.d_entropy ? a.d_entropy[row] : 0.f;
  // dx = p (A + B t), t = log p, and for the target dlp / temperature more
  const float A = -(dlp + (a.d_entropy ? dh * a.entropy[row] : 0.f)) * a.inverse, B = -dh * a.inverse;
  const u32x4* in = reinterpret_cast<const u32x4*>(a.logits + row * a.ld);
  u32x4* out = reinterpret_cast<u32x4*>(a.dlogits + row * a.ld);
  const int vectors = (int)(a.ld >> 3);
  u32x4 w[kLpUnroll];
#pragma unroll
  for (int i = 0; i < kLpUnroll; ++i) {
    const int c = c0 + i * kLpGradThreads;
    if (counts && c < vectors && c * 8 < a.V) w[i] = in[c];
  }
#pragma unroll
  for (int i = 0; i < kLpUnroll; ++i) {
    const int c = c0 + i * kLpGradThreads;
    if (c >= vectors) continue;
    bf16x8 y = {0, 0, 0, 0, 0, 0, 0, 0};
    if (counts && c * 8 < a.V) {
      float d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __uint_as_float((e & 1) ? w[i][e >> 1] & 0xffff0000u : w[i][e >> 1] << 16);
        const float t = __builtin_fmaf(x, a.inverse, -lse), p = __builtin_amdgcn_exp2f(t * kLog2e);
        d[e] = p * __builtin_fmaf(B, fmaxf(t, -1e4f), A);
      }
      if (a.d_logprobs && c == (int)(tgt >> 3))
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] += e == (int)(tgt & 7) ? dlp * a.inverse : 0.f;
      if (c * 8 + 8 > a.V)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = c * 8 + e < a.V ? d[e] : 0.f;
      y = pack8(d);
    }
    out[c] = __builtin_bit_cast(u32x4, y);
  }
}

int launch_token_logprobs_bwd(const LogprobsCall& c, const float* lse, const float* entropy, const float* d_logprobs, const float* d_entropy,
                              void* dlogits, hipStream_t st) {
  LogprobsGradArgs a{};
  a.logits = (const bf16_t*)c.logits;
  a.dlogits = (bf16_t*)dlogits;
  a.targets = c.targets;
  a.lse = lse; a.entropy = entropy; a.d_logprobs = d_logprobs; a.d_entropy = d_entropy;
  a.ld = c.ld;
  a.V = (int)c.V;
  a.inverse = c.inverse_temperature;
  a.blocks = (int)((c.ld / 8 + kLpGradThreads * kLpUnroll - 1) / (kLpGradThreads * kLpUnroll));
  hipLaunchKernelGGL(logprobs_grad_kernel, dim3((unsigned)(c.T * a.blocks)), dim3(kLpGradThreads), 0, st, a);
  return check_launch("token_logprobs_backward");
}

}  // namespace dl
