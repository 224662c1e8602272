// Linear attention with a decay for each KV head, and its gradient.  For one batch row and KV head, state S [dh, dh]:
//
//   S_t = lambda S_(t-1) + k_t v_t^T,   o_t = scale S_t^T q_t                                       (forward)
//   dq_t = scale S_t do_t;   R_t = lambda R_(t+1) + scale sum_h q_t^h do_t^hT,  dk_t = R_t v_t,  dv_t = R_t^T k_t
//
// Over chunks of 64 tokens these are matrix products.  With i, j a token's place in its chunk and S the state before the chunk,
//   o_i = scale (sum over j <= i of lambda^(i-j) (q_i . k_j) v_j + lambda^(i+1) S^T q_i),   S' = lambda^64 S + sum_j (lambda^(63-j) k_j) v_j^T
// The gradient of q is the same with (do, v, k) in the place of (q, k, v) and the state transposed; those of k and v walk the chunks from
// the last to the first with the state's gradient E, that of the state a chunk ends with:
//   dv_j = scale sum over i >= j, h of lambda^(i-j) (q_i . k_j) do_i + lambda^(63-j) E^T k_j,   dk_j = ... (do_i . v_j) q_i + lambda^(63-j) E v_j
//   E' = lambda^64 E + scale sum_i (lambda^(i+1) q_i) do_i^T
// A chain of 64-token steps is long, so a sequence is cut into segments (linear_plan) that run side by side: a first kernel forms
// what each segment adds to the state, a second adds these up from segment to segment, and the third does the chunks of a segment, starting
// from the state it begins (ends) with.  16384 tokens of 32 and 8 heads of 128 take 138 us, and 0.54 GB move (one pass over the data: 0.34 GB, 70 us at a
// copy's 4.76 TB/s; the rest is k and v read twice and the states between the kernels); backward 309 us and 1.24 GB (0.54 GB, 113 us).  Nothing is at its
// limit alone.  The sums over segments wait for their loads (3.8 to 4.5 TB/s; as long without their products); the kernels that do the chunks move 3.1 to
// 3.4 TB/s, and the vector units issue in 56 to 69 % of the cycles beside 15 to 32 % of the matrix units'.
//
// Precision.  States are fp32, in the accumulators and in memory; as operands they are the sum of two fp16, scaled by a power of two: 22 bits, and queries,
// scaled too, are exact in fp16.  Keys and values that have means make a state a large rank-one part and, in front of it, what tells tokens apart, which is all that
// a query orthogonal to the keys' mean sees.  In one fp16 results would be off by 2e-4 without means, 8e-3 at means of one deviation and 4e-2 at four, where
// their own rounding to bf16 is 1.7e-3; in two, by 4e-8, 2e-6 and 8e-6 (2-norms, emulated in fp64 for 4096 tokens of heads of 128).  The decayed keys
// (queries) whose products with the values (do) a state sums are split into three bf16 terms, which is exact up to fp32.  Where a state serves only results
// rounded to bf16, two terms do (2e-6, 3e-6 and 1e-5), and its decay from chunk to chunk is one fp32 (2e-7, 3e-6 and 2e-5).  Weighted scores are two terms (4e-7
// whatever the means); sums of few heads or keys cancel, and a score rounded to bf16 then shows (gradients 4e-2 off in single elements).  Decays of many tokens
// are evaluated as powers (exp2 of a multiple of the logarithm), the factor between chunks of a state that leaves as the sum of two fp32, so that no
// rounding of lambda is repeated.
//
// Layout.  All products are v_mfma_f32_16x16x32_bf16, D[row][col] += A[row][k] B[k][col]: lane (g = lane / 16, r = lane % 16) holds row r of A and
// column r of B, 8 of 32 k each, and rows 4 g .. 4 g + 3 of column r of D.  Scores are formed as S^T[j][i] = K Q^T, so that a lane
// owns one query and its scores come out as the B operand of O^T[d][i] += V^T P^T: k-slot (g, e) is token 4 g + e of the first 16 for e < 4, and of
// the second 16 otherwise, and the transposing reads of V take the same tokens.
#include "common.h"
#include "kernels.h"

namespace dl {

constexpr int kChunk = 64;
constexpr int kLinWaves = 8;   // waves of a workgroup: a state of 128 x 128 is 32 registers in each, and 16 of them fit a compute unit

// The logarithm of a decay, minus infinity (no memory at all) made finite: times no token it is to give 0, not NaN.
__device__ __forceinline__ double decay_log(float g) { return g < -1e30f ? -1e30 : (double)g; }
// A decay as the sum of two fp32: rounded to one, the state after n of them would be off by up to 6e-8 n.
struct Decay { float hi, lo; };
__device__ __forceinline__ Decay decay_of(float g, int tokens) {
  const double d = exp(decay_log(g) * tokens);
  const float hi = (float)d;
  return Decay{hi, (float)(d - (double)hi)};
}
// lambda s + x
__device__ __forceinline__ float decayed(const Decay& l, float s, float x) { return __builtin_fmaf(s, l.hi, __builtin_fmaf(s, l.lo, x)); }
// lambda^n for 0 <= n, log2 = log2(lambda)
__device__ __forceinline__ float power(float log2, int n) { return __builtin_amdgcn_exp2f(log2 * (float)n); }

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A value that the compiler works with from here on only: without this it keeps what it can derive from the lane's number and the decay
// (LDS addresses, powers) for every phase of a loop in registers throughout, a hundred more than there are, and reloads them from scratch
// memory in every iteration.  (Such a register costs bandwidth too: the 8 that linear_out_kernel<128> once spilled in every chunk were half as
// many bytes to HBM as o itself, 403 MB for 268 at 65536 tokens of 16 heads, and 202 us for 185.)
template <typename T>
__device__ __forceinline__ T here(T x) {
  asm volatile("" : "+v"(x));
  return x;
}

// rows * 64 .. of one head: `rows` rows of D at stride ld; a row at or past `rows` reads as zeros and is not written
template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const bf16_t* first, int64_t ld, int rows) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(first), 0, rows > 0 ? (int)(((rows - 1) * ld + D) * 2) : 0, 0x00020000);
}
__device__ __forceinline__ bf16x8 load8(__amdgpu_buffer_rsrc_t rs, uint32_t at) {
  return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)at, 0, 0));
}
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t rs, uint32_t at, const bf16x8& v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), rs, (int)at, 0, 0);
}

// [rows][D] of 16 bits in LDS, 16-byte piece c of row r at piece c ^ swz(r).  The LDS serves 256 bytes a clock, of 8-byte reads 32 lanes in order, of 16-byte
// reads lanes 0-3, 12-15, 20-27, then 4-11, 16-19, 28-31 (and 32 on likewise; timed, with pairs of lanes in one bank).  The pieces are dealt so that
// neither 8 rows of 32 bytes (transposing reads) nor those lanes of an operand along the rows, 8 of one piece and 8 of its neighbour, meet in a bank.
template <int D>
struct Rows {
  static constexpr int BYTES = D * 2, PIECES = D / 8;
  static __device__ __forceinline__ int swz(int r) {
    const int fours = ((((r >> 2) ^ (r >> 3)) & 1) << 1) | ((r >> 3) & 1);   // of rows 0, 4, 8, 12: 0, 2, 3, 1
    return (PIECES == 16 ? (r & 3) << 2 : PIECES == 8 ? ((r >> 1) & 1) << 2 : 0) | fours;
  }
  static __device__ __forceinline__ int at(int r, int piece) { return r * BYTES + ((piece ^ swz(r)) << 4); }
  // Operands, by a lane's LDS address that is the same for all of a kind (of a tile at the start of LDS): everything else is an exclusive or with a
  // constant, and constants added (the tile `t` and its row), which the read itself adds.
  // along: 16 rows from row0, k over step ks of the row
  static __device__ __forceinline__ uint32_t along_lane(uint32_t lds, int lane) { return lds + at(lane & 15, lane >> 4); }
  static __device__ __forceinline__ bf16x8 along(uint32_t along_lane, int t, int row0, int ks) {
    return *(LDS_PTR(const bf16x8))(uintptr_t)((along_lane ^ (uint32_t)(ks << 6)) + (uint32_t)(t + row0 * BYTES));
  }
  // columns: the 16 columns 16 n .. of the tile, k over the 32 rows from row0: slot (g, e) is row 4 g + e, or 12 + 4 g + e for e >= 4; with GAP 4 row 8 g + e
  template <int GAP = 16>
  static __device__ __forceinline__ uint32_t columns_lane(uint32_t lds, int lane) {
    return lds + at((lane >> 4) * (GAP == 16 ? 4 : 8) + ((lane & 15) >> 2), (lane & 3) >> 1) + (lane & 1) * 8;
  }
  template <int GAP = 16>
  static __device__ __forceinline__ bf16x8 columns(uint32_t columns_lane, int t, int n, int row0) {
    // a row further by 4 changes one bit of the swizzle, by 16 none
    const uint32_t lo = columns_lane ^ (uint32_t)(n << 5), hi = GAP == 16 ? lo : columns_lane ^ (uint32_t)((n << 5) ^ (swz(4) << 4));
    bf16x8 v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(lo + (uint32_t)(t + row0 * BYTES)));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(hi + (uint32_t)(t + (row0 + GAP) * BYTES)));
    return v;
  }
};
// where a kernel's LDS begins
__device__ __forceinline__ uint32_t lds_address(char* smem) { return (uint32_t)(uintptr_t)(LDS_PTR(char))smem; }

// A 64-row tile from memory to LDS without a detour through registers: each load of a wave fills 1 KB, lane after lane, so the pieces are
// picked in memory in the order in which they lie in LDS.  Done when vmcnt is 0 and a barrier passed.
template <int D>
__device__ __forceinline__ void tile_to_lds(__amdgpu_buffer_rsrc_t rs, char* t, int64_t ld, int wave, int lane) {
  constexpr int PIECES = Rows<D>::PIECES, RPI = 64 / PIECES, N = kChunk / RPI;
  lane = here(lane);
#pragma unroll
  for (int i = 0; i < (N + kLinWaves - 1) / kLinWaves; ++i) {
    const int j = i * kLinWaves + wave, r = j * RPI + lane / PIECES;
    if (N % kLinWaves == 0 || j < N)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LDS_PTR(void))(t + j * 1024), 16,
                                               (uint32_t)(r * (int)ld * 2 + (((lane % PIECES) ^ Rows<D>::swz(r)) << 4)), 0, 0, 0);
  }
}
// The same through registers, for a kernel that has them: asked for a tile ahead, written to LDS when the one before is done with.
template <int D>
struct Staged {
  static constexpr int TOTAL = kChunk * Rows<D>::PIECES, THREADS = 64 * kLinWaves, N = (TOTAL + THREADS - 1) / THREADS;
  bf16x8 v[N];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, int64_t ld) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = i * THREADS + (int)threadIdx.x;
      if (TOTAL % THREADS == 0 || idx < TOTAL) v[i] = load8(rs, (uint32_t)(idx / Rows<D>::PIECES * (int)ld * 2 + idx % Rows<D>::PIECES * 16));
    }
  }
  __device__ __forceinline__ void store(char* t) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = i * THREADS + (int)threadIdx.x;
      if (TOTAL % THREADS == 0 || idx < TOTAL) *reinterpret_cast<bf16x8*>(t + Rows<D>::at(idx / Rows<D>::PIECES, idx % Rows<D>::PIECES)) = v[i];
    }
  }
};
__device__ __forceinline__ void loads_done() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f32x4 mfma16_f16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Powers of two that take numbers up to some bound into the upper half of fp16's range (below 2^15, so that what is 2^29 times smaller than
// the bound keeps its eleven bits, and what these round off, down to 2^40 times smaller, a second fp16), and back.  exponent: of the bound, as an fp32 has it.
struct Scale {
  float up, down;
  __device__ __forceinline__ explicit Scale(int exponent) {
    const int e = max(exponent, 29);
    up = __int_as_float((268 - e) << 23);
    down = __int_as_float((e - 14) << 23);
  }
};

// An operand of KS steps (a lane's 8 values of 32 each, four lanes a row), in fp16: the rows scaled, exactly, to their largest value.  Two values at a
// time, in integers: of the 15 bits under a bf16's sign the exponent is moved and all are shifted into fp16's place.
template <int KS>
struct ScaledRow {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  f16x8 v[KS];
  float down;   // infinite for a row that is not finite
  __device__ __forceinline__ explicit ScaledRow(const bf16x8 (&x)[KS]) {
    u16x2 top = {0, 0};
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, __builtin_bit_cast(u32x4, x[k])[i] & 0x7fff7fffu));
    uint32_t most = max((uint32_t)top.x, (uint32_t)top.y);
    const auto a = __builtin_amdgcn_permlane16_swap(most, most, false, false);
    most = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(most, most, false, false);
    most = max(b[0], b[1]);
    const uint32_t e = max(most >> 7, 29u);
    down = __int_as_float(e == 255 ? 0x7f800000 : (int)(e - 14) << 23);
    const unsigned short less = (unsigned short)((e - 29) << 7);
#pragma unroll
    for (int k = 0; k < KS; ++k) {
      const u32x4 u = __builtin_bit_cast(u32x4, x[k]);
      u32x4 h;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u16x2 m = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, u[i] & 0x7fff7fffu), u16x2{less, less}) << (unsigned short)3;
        h[i] = (u[i] & 0x80008000u) | __builtin_bit_cast(uint32_t, m);
      }
      v[k] = __builtin_bit_cast(f16x8, h);
    }
  }
};

// Stores NB blocks of 16 values of a lane's row as bf16.  A lane holds values 16 n + 4 g .. + 3 of block n; lanes 16 apart exchange halves of two blocks,
// and each stores 16 bytes of one of them.  all: no lane's row is to be zeros (keep false).
template <int NB>
__device__ __forceinline__ void store_row(__amdgpu_buffer_rsrc_t rs, uint32_t row_at, const f32x4 (&o)[NB], bool all, bool keep, int lane) {
  const int g = lane >> 4;
  row_at += (g & 1) * 32 + (g >> 1) * 16;
#pragma unroll
  for (int n = 0; n < NB; n += 2) {
    u32x2 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (bf16_t)o[n + i][e];
      x[i] = __builtin_bit_cast(u32x2, v);
    }
    const auto a = __builtin_amdgcn_permlane16_swap(x[0].x, x[1].x, false, false), b = __builtin_amdgcn_permlane16_swap(x[0].y, x[1].y, false, false);
    u32x4 w = {a[0], b[0], a[1], b[1]};
    if (!all)
      if (!keep) w = u32x4{0, 0, 0, 0};
    __builtin_amdgcn_raw_buffer_store_b128(w, rs, (int)(row_at + n * 32), 0, 0);
  }
}

__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// Weights of a chunk's tokens, in LDS: on their way into the state after `rows` tokens from the chunk's first, lambda^(rows-1-t), and into the gradient of the
// state `before` tokens before the chunk, mult lambda^(before+t+1).  (Sixteen registers would hold a lane's, and are not there.)
__device__ __forceinline__ void weights_to_end(float* w, float log2, int rows) {
  if (threadIdx.x < kChunk) w[threadIdx.x] = power(log2, max(rows - 1 - (int)threadIdx.x, 0));
}
__device__ __forceinline__ void weights_from_start(float* w, float log2, float mult, int before) {
  if (threadIdx.x < kChunk) w[threadIdx.x] = mult * power(log2, before + (int)threadIdx.x + 1);
}

// Both terms of a state as an operand lie in LDS.  Of a 128 x 128 state, two workgroups' would take 192 of a compute unit's 160 KB: there they take turns in one place.  (One workgroup a
// compute unit, with registers to load the next tiles ahead: 117 us for 110 in the forward's last kernel, 16384 tokens of 32 and 8 heads of 128, 265
// for 246 in the gradients'.)
template <int D> constexpr bool kBothTerms = D < 128;
template <int D> constexpr int kStateLds = (kBothTerms<D> ? 2 : 1) * D * D * 2;

// A state [D along keys][D along values] over the waves: wave -> RB x CB blocks of 16 x 16 (of 32 x 32 elements four waves hold one each).  In
// memory between the kernels it lies as the accumulators do: [wave][block][lane] f32x4.
template <int D>
struct State {
  static constexpr int RB = 1, CB = D == 128 ? 8 : D / 32, N = RB * CB, WAVES = D == 32 ? 4 : kLinWaves;
  f32x4 a[RB][CB];
  static __device__ __forceinline__ int row_block(int wave) { return D == 128 ? wave : wave >> 1; }
  static __device__ __forceinline__ int col_block(int wave) { return D == 128 ? 0 : (wave & 1) * CB; }
  // first of the four rows, and the column, of a lane in block (rb, cb) of the state
  static __device__ __forceinline__ int row(int rb, int lane) { return rb * 16 + ((lane >> 4) << 2); }
  static __device__ __forceinline__ int col(int cb, int lane) { return cb * 16 + (lane & 15); }
  static __device__ __forceinline__ bool holds(int wave) { return WAVES == kLinWaves || wave < WAVES; }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j) a[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // EXACT: with both terms of the decay
  template <bool EXACT>
  __device__ __forceinline__ void decay(const Decay& l) {
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) a[i][j][e] = EXACT ? decayed(l, a[i][j][e], 0.f) : a[i][j][e] * l.hi;
  }
  // element of a [D][D] matrix, transposed if flip
  static __device__ __forceinline__ int element(int row, int col, int flip) { return flip ? col * D + row : row * D + col; }
  __device__ __forceinline__ void load_matrix(const float* s, int flip, int wave, int lane) {
    if (!holds(wave)) return;
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) a[i][j][e] = s[element(row(row_block(wave) + i, lane) + e, col(col_block(wave) + j, lane), flip)];
  }
  __device__ __forceinline__ void store_matrix(float* s, int wave, int lane) const {
    if (!holds(wave)) return;
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[element(row(row_block(wave) + i, lane) + e, col(col_block(wave) + j, lane), 0)] = a[i][j][e];
  }
  __device__ __forceinline__ void load(const float* s, int wave, int lane) {
    if (!holds(wave)) return;
#pragma unroll
    for (int i = 0; i < N; ++i) a[i / CB][i % CB] = reinterpret_cast<const f32x4*>(s)[(wave * N + i) * 64 + lane];
  }
  __device__ __forceinline__ void store(float* s, int wave, int lane) const {
    if (!holds(wave)) return;
#pragma unroll
    for (int i = 0; i < N; ++i) reinterpret_cast<f32x4*>(s)[(wave * N + i) * 64 + lane] = a[i / CB][i % CB];
  }
  // the largest of the wave's elements, those that are no numbers left out
  __device__ __forceinline__ float largest(int wave) const {
    float m = 0.f;
    if (holds(wave)) {
#pragma unroll
      for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(a[i][j][e]));
      if (__builtin_amdgcn_ballot_w64(m > 3e38f) != 0) {
        m = 0.f;
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
          for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) m = fabsf(a[i][j][e]) < INFINITY ? fmaxf(m, fabsf(a[i][j][e])) : m;
      }
    }
    const auto a32 = __builtin_amdgcn_permlane32_swap(__float_as_int(m), __float_as_int(m), false, false);
    m = fmaxf(__int_as_float(a32[0]), __int_as_float(a32[1]));
    const auto a16 = __builtin_amdgcn_permlane16_swap(__float_as_int(m), __float_as_int(m), false, false);
    m = fmaxf(__int_as_float(a16[0]), __int_as_float(a16[1]));
    m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x128, 0xf, 0xf, true)));   // rotations within 16 lanes
    m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x124, 0xf, 0xf, true)));
    m = fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x122, 0xf, 0xf, true)));
    return fmaxf(m, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(m), 0x121, 0xf, 0xf, true)));
  }
  // to LDS [columns][rows]: an operand along either.  The scaled state is the sum of two fp16: its rounding and what that rounds off (at most 8; no
  // number where the first is infinite, which the clamp keeps out of the product).  The second lies behind the first, or low says which is meant.
  __device__ __forceinline__ void to_lds(char* t, float up, bool low, int wave, int lane) const {
    if (!holds(wave)) return;
    lane = here(lane);
    up = here(up);   // no conversion ahead of the barrier in front of this
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
      for (int j = 0; j < CB; ++j) {
        f16x4 v, rest;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = a[i][j][e] * up;
          const _Float16 h = (_Float16)x;
          const float off = __builtin_amdgcn_fmed3f(x - (float)h, -8.f, 8.f);
          if (kBothTerms<D>) {
            v[e] = h;
            rest[e] = (_Float16)off;
          } else {
            v[e] = (_Float16)(low ? off : x);
          }
        }
        const int r = row(row_block(wave) + i, lane), p = (col_block(wave) + j) * 16 + (lane & 15);
        char* at = t + Rows<D>::at(p, r >> 3) + ((r & 7) << 1);
        *reinterpret_cast<f16x4*>(at) = v;
        if (kBothTerms<D>) *reinterpret_cast<f16x4*>(at + D * D * 2) = rest;
      }
  }
  // += sum over a tile's 64 tokens of (w x)^T y, all in LDS (x, y: where); w x as the sum of SPLIT bf16
  template <int SPLIT>
  __device__ __forceinline__ void add(int x, int y, const float* w, int wave, int lane, uint32_t columns_lane) {
    if (!holds(wave)) return;
    lane = here(lane);
    const uint32_t cl = here(columns_lane ^ (uint32_t)(col_block(wave) << 5)), own = here(columns_lane ^ (uint32_t)(row_block(wave) << 5));
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      bf16x8 part[RB][SPLIT];
      const f32x4 w0 = *reinterpret_cast<const f32x4*>(w + p * 32 + ((lane >> 4) << 2)), w1 = *reinterpret_cast<const f32x4*>(w + p * 32 + 16 + ((lane >> 4) << 2));
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        float f[8];
        unpack8(Rows<D>::columns(own, x, i, p * 32), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] *= e < 4 ? w0[e] : w1[e - 4];
#pragma unroll
        for (int k = 0; k < SPLIT; ++k) {
          part[i][k] = pack8(f);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] -= (float)part[i][k][e];
        }
      }
      constexpr int AT_ONCE = CB < 2 ? CB : 2;   // blocks in turn: an MFMA whose sum is the last one's waits for it
#pragma unroll
      for (int j0 = 0; j0 < CB; j0 += AT_ONCE) {
        bf16x8 v[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) v[j] = Rows<D>::columns(cl, y, j0 + j, p * 32);
#pragma unroll
        for (int k = SPLIT - 1; k >= 0; --k)
#pragma unroll
          for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
            for (int i = 0; i < RB; ++i) a[i][j0 + j] = mfma16(part[i][k], v[j], a[i][j0 + j]);
      }
    }
  }
};

// The scale of a state whose waves left their largest elements in LDS.
__device__ __forceinline__ Scale state_scale(const float* largest) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < kLinWaves; ++i) m = fmaxf(m, largest[i]);
  return Scale(__builtin_amdgcn_readfirstlane(__float_as_int(m) >> 23));
}

// A 16 x 16 block of scores, whose lane holds four keys of one query (STEP -1) or four queries of one key (STEP 1), times mult lambda^(place of the query -
// place of the key); what is not causal becomes 0.  blocks: from the key's to the query's, -1 .. 3.  The same work for every block, without branches, so
// that two of them, their reads and products, pass together (times with a state of one term): with branches around what is not causal, and one power of the lane's for the blocks off the
// diagonal, dk, dv and dq of 4096 tokens of 32 heads of 64 on one KV head take 49.6 us for 44.7, the forward's last kernel 80 for 78 (16384 tokens
// of 32 and 8 heads of 128); heads of 64 that share nothing 36.9 for 37.4.
// (Beside a state of 128 x 128 no register is left for what a lane derives from its number and keeps: the caller passes here(lane).)
template <int STEP>
__device__ __forceinline__ void weigh_scores(f32x4& s, float log2, float mult, int blocks, int lane) {
  const int first = blocks * 16 + STEP * (((lane >> 4) << 2) - (lane & 15));   // the lane's four differences: this, and the next three in STEPs
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = first + STEP * e >= 0 ? s[e] * (mult * power(log2, first + STEP * e)) : 0.f;
}

// o[n] += factor times the product of a(n, k) with the scaled row, for NB blocks, four in turn
template <int KS, int NB, typename F>
__device__ __forceinline__ void add_scaled(f32x4 (&o)[NB], const ScaledRow<KS>& x, float factor, F&& a) {
  constexpr int AT_ONCE = NB < 4 ? NB : 4;
#pragma unroll
  for (int n0 = 0; n0 < NB; n0 += AT_ONCE) {
    f32x4 t[AT_ONCE];
#pragma unroll
    for (int n = 0; n < AT_ONCE; ++n) t[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int n = 0; n < AT_ONCE; ++n) t[n] = mfma16_f16(__builtin_bit_cast(f16x8, a(n0 + n, k)), x.v[k], t[n]);
#pragma unroll
    for (int n = 0; n < AT_ONCE; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n0 + n][e] = __builtin_fmaf(t[n][e], factor, o[n0 + n][e]);
  }
}

// Weighted scores of 32 tokens as an operand: the sum of two bf16.
struct Scores {
  bf16x8 hi, lo;
  __device__ __forceinline__ explicit Scores(const f32x4 (&sc)[2]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = (bf16_t)sc[e >> 2][e & 3];
      lo[e] = (bf16_t)(sc[e >> 2][e & 3] - (float)hi[e]);
    }
  }
  // o[n] += a(n) times the scores, for NB blocks, four in turn
  template <int NB, typename F>
  __device__ __forceinline__ void times(f32x4 (&o)[NB], F&& a) const {
    constexpr int AT_ONCE = NB > 4 ? 2 : NB;
#pragma unroll
    for (int n0 = 0; n0 < NB; n0 += AT_ONCE) {
      bf16x8 x[AT_ONCE];
#pragma unroll
      for (int n = 0; n < AT_ONCE; ++n) x[n] = a(n0 + n);
#pragma unroll
      for (int n = 0; n < AT_ONCE; ++n) o[n0 + n] = mfma16(x[n], lo, o[n0 + n]);
#pragma unroll
      for (int n = 0; n < AT_ONCE; ++n) o[n0 + n] = mfma16(x[n], hi, o[n0 + n]);
    }
  }
};

struct LinearArgs {
  const bf16_t *q, *k, *v, *d_o;
  bf16_t *o, *dk, *dv;
  const float* log_decay;
  const int64_t* lengths;
  float* seg;              // [pair][segment] states (gradients) between the kernels; null: there is one segment, which takes s_in itself
  const float* s_in;
  float* s_out;
  int S, Hq, Hkv, flip;    // flip: s_in is read transposed
  int seg_chunks, nseg;
  float scale;
};

// tokens of batch row b
__device__ __forceinline__ int row_length(const LinearArgs& p, int b) {
  const int64_t n = p.lengths ? p.lengths[b] : p.S;
  return (int)(n < 0 ? 0 : n > p.S ? p.S : n);
}
__device__ __forceinline__ float log2_decay(float g) { return (float)(decay_log(g) * 1.4426950408889634); }

// ------------------------------------------------------------------------------------------
// What a segment of m tokens adds to the state that passes through it: sum_t lambda^(m-1-t) k_t v_t^T, from k and v;
// GRADIENT: to the state's gradient, sum over t and the group's heads of scale lambda^(t+1) q_t do_t^T, from q and d_o.
// Bound by its loads: without its products it takes as long.  27 us at 16384 tokens of 8 KV heads of 128 (0.1 GB, 3.8 TB/s), 86 us in their backward with
// 32 heads (0.37 GB, 4.3 TB/s); the gradients' sums dealt to workgroups by heads, so that they end with the states', came to the same, and cost the scan.
// ------------------------------------------------------------------------------------------
template <int D, int SPLIT, bool GRADIENT>
__device__ __forceinline__ void segment_sum(const LinearArgs& p, char* smem) {
  constexpr int xt = 0, yt = kChunk * D * 2;
  float* w = reinterpret_cast<float*>(smem + 2 * kChunk * D * 2);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int pair = blockIdx.x / p.nseg, sg = blockIdx.x % p.nseg, b = pair / p.Hkv, j = pair % p.Hkv;
  const int len = row_length(p, b), t0 = sg * p.seg_chunks * kChunk;
  State<D> s;
  s.clear();
  float* out = p.seg + (int64_t)blockIdx.x * D * D;
  const int m = min(len - t0, p.seg_chunks * kChunk);
  if (m <= 0) {
    s.store(out, wave, lane);
    return;
  }
  const int G = GRADIENT ? p.Hq / p.Hkv : 1, items = (m + kChunk - 1) / kChunk * G;
  const int64_t ld = (int64_t)(GRADIENT ? p.Hq : p.Hkv) * D;
  const bf16_t *x = GRADIENT ? p.q : p.k, *y = GRADIENT ? p.d_o : p.v;
  const int64_t first = ((int64_t)b * p.S + t0) * ld + (int64_t)j * G * D;
  const float log2 = log2_decay(p.log_decay[j]);
  const uint32_t columns_lane = Rows<D>::columns_lane(lds_address(smem), lane);
  Staged<D> xs, ys;
  auto fetch = [&](int it) {
    const int rows = min(m - it / G * kChunk, kChunk);
    const int64_t at = first + (int64_t)(it / G) * kChunk * ld + (int64_t)(it % G) * D;
    xs.load(rows_rsrc<D>(x + at, ld, rows), ld);
    ys.load(rows_rsrc<D>(y + at, ld, rows), ld);
  };
  fetch(0);
  for (int it = 0; it < items; ++it) {
    const int c = it / G;
    __syncthreads();
    xs.store(smem + xt);
    ys.store(smem + yt);
    if (!GRADIENT) weights_to_end(w, log2, m - c * kChunk);
    else if (it % G == 0) weights_from_start(w, log2, p.scale, c * kChunk);
    __syncthreads();
    if (it + 1 < items) fetch(it + 1);
    s.template add<SPLIT>(xt, yt, w, wave, lane, columns_lane);
  }
  s.store(out, wave, lane);
}
// y 0: the states, of `a`; 1: their gradients, of `g`.  What may reach the caller (the forward's states, the backward's gradients) is summed with three
// terms, whether the caller asked for it or not, so that no other result depends on that; the states of a backward serve dq alone.
template <int D, bool BACKWARD>
__global__ __launch_bounds__(64 * kLinWaves, 4) void linear_segment_kernel(const LinearArgs a, const LinearArgs g) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  if (!BACKWARD) segment_sum<D, 3, false>(a, smem);
  else if (blockIdx.y == 0) segment_sum<D, 2, false>(a, smem);
  else segment_sum<D, 3, true>(g, smem);
}

// ------------------------------------------------------------------------------------------
// From segment to segment: what each adds is replaced by the state it begins with; GRADIENT: by the gradient of the state it ends
// with.  A thread holds four elements of a state in fp64 (a decay of many tokens has no second fp32), eight segments ahead in flight.
// 14 us for 512 states of 128 x 128 (67 MB read and written, 4.8 TB/s).
// ------------------------------------------------------------------------------------------
template <int D, bool GRADIENT>
__device__ __forceinline__ void segment_scan(const LinearArgs& p) {
  using St = State<D>;
  constexpr int PARTS = D * D / 1024, AHEAD = 8;
  const int pair = blockIdx.x / PARTS, f = blockIdx.x % PARTS * 256 + threadIdx.x, b = pair / p.Hkv, j = pair % p.Hkv;
  const int lane = f & 63, blk = (f >> 6) % St::N, wave = (f >> 6) / St::N;
  const int row = St::row(St::row_block(wave) + blk / St::CB, lane), col = St::col(St::col_block(wave) + blk % St::CB, lane);
  const int len = row_length(p, b), seg_tokens = p.seg_chunks * kChunk;
  const double log = decay_log(p.log_decay[j]), whole = exp(log * seg_tokens);
  f32x4* at = reinterpret_cast<f32x4*>(p.seg + (int64_t)pair * p.nseg * D * D) + f;
  double s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = p.s_in ? (double)p.s_in[(int64_t)pair * D * D + St::element(row + e, col, p.flip)] : 0.0;
  for (int n0 = 0; n0 < p.nseg; n0 += AHEAD) {
    f32x4 u[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int n = n0 + i;
      if (n < p.nseg) u[i] = at[(int64_t)(GRADIENT ? p.nseg - 1 - n : n) * (D * D / 4)];
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (n0 + i >= p.nseg) break;
      const int n = GRADIENT ? p.nseg - 1 - n0 - i : n0 + i, m = min(max(len - n * seg_tokens, 0), seg_tokens);
      at[(int64_t)n * (D * D / 4)] = f32x4{(float)s[0], (float)s[1], (float)s[2], (float)s[3]};
      if (m == 0) continue;
      const double l = m == seg_tokens ? whole : exp(log * m);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = l * s[e] + (double)u[i][e];
    }
  }
  if (p.s_out)
#pragma unroll
    for (int e = 0; e < 4; ++e) p.s_out[(int64_t)pair * D * D + St::element(row + e, col, 0)] = (float)s[e];
}
template <int D>
__global__ __launch_bounds__(256) void linear_scan_kernel(const LinearArgs a, const LinearArgs g) {
  if (blockIdx.y == 0) segment_scan<D, false>(a);
  else segment_scan<D, true>(g);
}

// ------------------------------------------------------------------------------------------
// o of a segment (dq of one, from d_o, v, k): its chunks from the first to the last, the state in the accumulators and, as an operand, in
// LDS.  Four waves take 16 queries of a head each, the other four those of the next head; an odd last head is shared, half of the columns
// for either.  110 to 120 us at 16384 tokens of 32 and 8 heads of 128 (0.37 GB, 3.1 to 3.4 TB/s), of which the state's second term is 30: 10 its
// products, 12 its conversion, 8 the barriers (each timed without it).
// SPLIT: 3 where the state goes on to the caller, 2 where it serves this kernel's products alone.
// ------------------------------------------------------------------------------------------
// NB blocks of 16 columns from n0 of o for the query that the lane's row is.  some: there is a state, scaled by sc; low: of its terms the second is in LDS,
// where there is but one, and the first afterwards
template <int D, int NB>
__device__ __forceinline__ void out_tile(f32x4 (&o)[NB], const bf16x8 (&qf)[D / 32], const State<D>& s, bool some, const Scale& sc, bool low, char* smem,
                                         int tile, int n0, float log2, float scale, int wave, int lane, uint32_t along_lane, uint32_t columns_lane) {
  constexpr int KS = D / 32, kt = 0, vt = kChunk * D * 2, st = 2 * kChunk * D * 2;
  const uint32_t al = here(along_lane), sl = here(along_lane + (uint32_t)(n0 * 16 * D * 2)), cl = here(columns_lane ^ (uint32_t)(n0 << 5));
  #pragma unroll
  for (int n = 0; n < NB; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int pr = 0; pr < 2; ++pr) {
    if (2 * pr > tile) break;
    f32x4 p[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) p[i] = mfma16(Rows<D>::along(al, kt, (2 * pr + i) * 16, k), qf[k], p[i]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) weigh_scores<-1>(p[i], log2, scale, tile - 2 * pr - i, D == 128 ? here(lane) : lane);
    const Scores pf(p);
    pf.times(o, [&](int n) { return Rows<D>::columns(cl, vt, n, pr * 32); });
  }
  if (some) {   // last, when the queries as they are need no registers any more
    const ScaledRow<KS> qs(qf);
    const float after = power(log2, tile * 16 + (here(lane) & 15) + 1) * scale * sc.down * qs.down;
    const auto add = [&](int t) {
      const uint32_t at = here(sl);
      add_scaled<KS>(o, qs, after, [&](int n, int k) { return Rows<D>::along(at, t, n * 16, k); });
    };
    add(st);
    if constexpr (!kBothTerms<D>) {
      __syncthreads();
      s.to_lds(smem + st, sc.up, !low, wave, lane);
      __syncthreads();
    }
    add(st + kStateLds<D> - D * D * 2);
  }
}

template <int D, int SPLIT>
__device__ __forceinline__ void segment_out(const LinearArgs& p, int id, int part, int parts, char* smem) {
  constexpr int NB = D / 16, KS = D / 32;
  constexpr int kt = 0, vt = kChunk * D * 2, st = 2 * kChunk * D * 2;
  float *largest = reinterpret_cast<float*>(smem + st + kStateLds<D>), *w = largest + kLinWaves;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int pair = id / p.nseg, sg = id % p.nseg, b = pair / p.Hkv, j = pair % p.Hkv, G = p.Hq / p.Hkv;
  const int per = (G + parts - 1) / parts, h0 = part * per, h1 = min(G, h0 + per);
  const int len = row_length(p, b), t0 = sg * p.seg_chunks * kChunk;
  const int rows_all = min(p.S - t0, p.seg_chunks * kChunk), m = max(min(len - t0, rows_all), 0), chunks = (m + kChunk - 1) / kChunk;
  const int64_t ldq = (int64_t)p.Hq * D, ldk = (int64_t)p.Hkv * D, tok0 = (int64_t)b * p.S + t0;
  const int64_t kv0 = tok0 * ldk + (int64_t)j * D, q0 = tok0 * ldq + (int64_t)j * G * D;
  float* s_out = p.seg || part ? nullptr : p.s_out;

  State<D> s;
  if (p.seg) s.load(p.seg + (int64_t)id * D * D, wave, lane);
  else if (p.s_in) s.load_matrix(p.s_in + (int64_t)pair * D * D, p.flip, wave, lane);
  else s.clear();
  bool some = p.s_in != nullptr || sg > 0;   // a state that is not zero
  Scale sc(0);
  if (some) largest[wave] = s.largest(wave);
  const float log2 = uniform(log2_decay(p.log_decay[j]));
  const Decay whole = decay_of(p.log_decay[j], kChunk);
  const uint32_t along_lane = Rows<D>::along_lane(lds_address(smem), lane), columns_lane = Rows<D>::columns_lane(lds_address(smem), lane);

  for (int c = 0; c < chunks; ++c) {
    const int rows = min(m - c * kChunk, kChunk), rows_out = min(rows_all - c * kChunk, kChunk);
    const bool more = c + 1 < chunks;
    const int64_t kc = kv0 + (int64_t)c * kChunk * ldk;
    __syncthreads();
    tile_to_lds<D>(rows_rsrc<D>(p.k + kc, ldk, rows), smem + kt, ldk, wave, lane);
    tile_to_lds<D>(rows_rsrc<D>(p.v + kc, ldk, rows), smem + vt, ldk, wave, lane);
    if (c == 0 || rows < kChunk) weights_to_end(w, log2, rows);
    if (some) {
      sc = state_scale(largest);
      s.to_lds(smem + st, sc.up, false, wave, lane);
    }
    loads_done();
    bool low = false;
    const int64_t qc = q0 + (int64_t)c * kChunk * ldq;
    for (int h = h0; h < h1; h += 2, low = !low) {
      const bool both = h + 1 < h1;
      if (!both && D == 32 && wave >= 4) break;   // 16 columns are not worth sharing
      const int head = both ? h + (wave >> 2) : h, tile = (wave + (h >> 1)) & 3, t = tile * 16 + r;
      const uint32_t at = (uint32_t)(t * (int)ldq * 2);
      const __amdgpu_buffer_rsrc_t rq = rows_rsrc<D>(p.q + qc + (int64_t)head * D, ldq, rows);
      const __amdgpu_buffer_rsrc_t ro = rows_rsrc<D>(p.o + qc + (int64_t)head * D, ldq, rows_out);
      bf16x8 qf[KS];
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[k] = load8(rq, at + k * 64 + g * 16);
      if (both || D == 32) {
        f32x4 o[NB];
        out_tile<D, NB>(o, qf, s, some, sc, low, smem, tile, 0, log2, p.scale, wave, lane, along_lane, columns_lane);
        store_row<NB>(ro, at, o, rows == kChunk, t < rows, lane);
      } else if constexpr (D > 32) {
        const int n0 = wave >= 4 ? NB / 2 : 0;
        f32x4 o[NB / 2];
        out_tile<D, NB / 2>(o, qf, s, some, sc, low, smem, tile, n0, log2, p.scale, wave, lane, along_lane, columns_lane);
        store_row<NB / 2>(ro, at + n0 * 32, o, rows == kChunk, t < rows, lane);
      }
    }
    if (more || s_out) {
      s.template decay<SPLIT == 3>(rows == kChunk ? whole : Decay{power(log2, rows), 0.f});
      s.template add<SPLIT>(kt, vt, w, wave, lane, columns_lane);
      some = true;
      if (more) largest[wave] = s.largest(wave);
    }
  }
  const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int c = chunks; c * kChunk < rows_all; ++c)
    for (int h = h0 + (wave >> 2); h < h1; h += 2) {
      const __amdgpu_buffer_rsrc_t ro = rows_rsrc<D>(p.o + q0 + (int64_t)c * kChunk * ldq + (int64_t)h * D, ldq, min(rows_all - c * kChunk, kChunk));
#pragma unroll
      for (int n = 0; n < NB; n += 2) store8(ro, (uint32_t)(((wave & 3) * 16 + r) * (int)ldq * 2) + n * 32 + g * 16, zero);
    }
  if (s_out) s.store_matrix(s_out + (int64_t)pair * D * D, wave, lane);
}

// workgroup -> segment, and part of the group's heads
template <int D, int SPLIT>
__global__ __launch_bounds__(64 * kLinWaves, 4) void linear_out_kernel(const LinearArgs p, int segments, int parts) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  segment_out<D, SPLIT>(p, blockIdx.x % segments, blockIdx.x / segments, parts, smem);
}

// ------------------------------------------------------------------------------------------
// dk and dv of a segment: its chunks from the last to the first, the gradient E of the state that a chunk ends with in the accumulators
// and, as an operand along either side, in LDS.  The group's heads pass by, their q and do in LDS; four waves form dv of 16 keys each, the
// other four dk, which is the same with q and do, k and v in each other's place and E transposed.
// ------------------------------------------------------------------------------------------
template <int D, int SPLIT>
__device__ __forceinline__ void segment_keys(const LinearArgs& p, int id, char* smem) {
  constexpr int NB = D / 16, KS = D / 32;
  constexpr int qt = 0, dt = kChunk * D * 2, et = 2 * kChunk * D * 2, lt = et + kStateLds<D> - D * D * 2;   // lt: the state's second term
  float *largest = reinterpret_cast<float*>(smem + et + kStateLds<D>), *w = largest + kLinWaves;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int pair = id / p.nseg, sg = id % p.nseg, b = pair / p.Hkv, j = pair % p.Hkv, G = p.Hq / p.Hkv;
  const int len = row_length(p, b), t0 = sg * p.seg_chunks * kChunk;
  const int rows_all = min(p.S - t0, p.seg_chunks * kChunk), m = max(min(len - t0, rows_all), 0), chunks = (m + kChunk - 1) / kChunk;
  const int64_t ldq = (int64_t)p.Hq * D, ldk = (int64_t)p.Hkv * D, tok0 = (int64_t)b * p.S + t0;
  const int64_t kv0 = tok0 * ldk + (int64_t)j * D, q0 = tok0 * ldq + (int64_t)j * G * D;
  const bool dk_role = wave >= 4;
  const int tile = wave & 3, key = tile * 16 + r;
  const uint32_t at = (uint32_t)(key * (int)ldk * 2);
  const bf16_t* own = (dk_role ? p.v : p.k) + kv0;
  bf16_t* out = (dk_role ? p.dk : p.dv) + kv0;
  const uint32_t score_rows = dk_role ? dt : qt, sum_rows = dk_role ? qt : dt;

  State<D> s;
  if (p.seg) s.load(p.seg + (int64_t)id * D * D, wave, lane);
  else if (p.s_in) s.load_matrix(p.s_in + (int64_t)pair * D * D, 0, wave, lane);
  else s.clear();
  // not zero: a gradient comes in, or the row goes on behind this segment
  bool some = p.s_in != nullptr || len > t0 + p.seg_chunks * kChunk;
  Scale sc(0);
  if (some) largest[wave] = s.largest(wave);
  const float log2 = uniform(log2_decay(p.log_decay[j]));
  const Decay whole = decay_of(p.log_decay[j], kChunk);
  weights_from_start(w, log2, p.scale, 0);
  const uint32_t along_lane = Rows<D>::along_lane(lds_address(smem), lane), columns_lane = Rows<D>::columns_lane(lds_address(smem), lane);
  for (int c = chunks - 1; c >= 0; --c) {
    const int rows = min(m - c * kChunk, kChunk);
    const int64_t kc = (int64_t)c * kChunk * ldk;
    const bool more = c > 0 || (!p.seg && p.s_out);
    const bool into = some;
    auto bring = [&](int h) {   // the head's queries and do, once nobody works with what is there
      const int64_t from = q0 + (int64_t)c * kChunk * ldq + (int64_t)h * D;
      __syncthreads();
      tile_to_lds<D>(rows_rsrc<D>(p.q + from, ldq, rows), smem + qt, ldq, wave, lane);
      tile_to_lds<D>(rows_rsrc<D>(p.d_o + from, ldq, rows), smem + dt, ldq, wave, lane);
    };
    bring(0);
    if (into) {
      sc = state_scale(largest);
      s.to_lds(smem + et, sc.up, true, wave, lane);
    }
    const __amdgpu_buffer_rsrc_t rk = rows_rsrc<D>(own + kc, ldk, rows);
    bf16x8 kf[KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) kf[k] = load8(rk, at + k * 64 + g * 16);
    loads_done();
    f32x4 acc[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (into) {
      float down;
      const auto add = [&](int t) {
        bf16x8 kh[KS];   // scaled for each term: beside a state of 128 x 128 there are no registers to keep this and kf, nor for the addresses of more columns
#pragma unroll
        for (int k = 0; k < KS; ++k) kh[k] = D == 128 ? __builtin_bit_cast(bf16x8, here(__builtin_bit_cast(u32x4, kf[k]))) : kf[k];
        const ScaledRow<KS> ks(kh);
        down = ks.down;
        constexpr int AT_ONCE = D == 128 ? 2 : NB;
#pragma unroll
        for (int n0 = 0; n0 < NB; n0 += AT_ONCE) {
          if (!dk_role) {
            const uint32_t al = here(along_lane);
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
              for (int n = n0; n < n0 + AT_ONCE; ++n) acc[n] = mfma16_f16(__builtin_bit_cast(f16x8, Rows<D>::along(al, t, n * 16, k)), ks.v[k], acc[n]);
          } else {
            const uint32_t cl = Rows<D>::template columns_lane<4>(lds_address(smem), here(lane));
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
              for (int n = n0; n < n0 + AT_ONCE; ++n)
                acc[n] = mfma16_f16(__builtin_bit_cast(f16x8, Rows<D>::template columns<4>(cl, t, n, k * 32)), ks.v[k], acc[n]);
          }
        }
      };
      add(lt);
      if constexpr (!kBothTerms<D>) {
        __syncthreads();
        s.to_lds(smem + et, sc.up, false, wave, lane);
        __syncthreads();
      }
      add(et);
      const float left = power(here(log2), max(rows - 1 - key, 0)) * sc.down * down;
#pragma unroll
      for (int n = 0; n < NB; ++n) acc[n] *= left;
    }
    if (more) s.template decay<SPLIT == 3>(rows == kChunk ? whole : Decay{power(log2, rows), 0.f});
    for (int h = 0; h < G; ++h) {
      if (h > 0) {
        bring(h);
        loads_done();
      }
#pragma unroll
      for (int pr = 0; pr < 2; ++pr) {
        if (2 * pr + 1 < tile) continue;
        const uint32_t al = here(along_lane + score_rows), cl = here(columns_lane + sum_rows);
        f32x4 sc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          sc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KS; ++k) sc[i] = mfma16(Rows<D>::along(al, 0, (2 * pr + i) * 16, k), kf[k], sc[i]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) weigh_scores<1>(sc[i], log2, p.scale, 2 * pr + i - tile, D == 128 ? here(lane) : lane);
        const Scores pf(sc);
        pf.times(acc, [&](int n) { return Rows<D>::columns(cl, 0, n, pr * 32); });
      }
      if (more) s.template add<SPLIT>(qt, dt, w, wave, lane, columns_lane);
    }
    some = some || more;
    if (c > 0) largest[wave] = s.largest(wave);
    store_row<NB>(rows_rsrc<D>(out + kc, ldk, min(rows_all - c * kChunk, kChunk)), at, acc, rows == kChunk, key < rows, lane);
  }
  const bf16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int c = chunks; c * kChunk < rows_all; ++c) {
    const __amdgpu_buffer_rsrc_t ro = rows_rsrc<D>(out + (int64_t)c * kChunk * ldk, ldk, min(rows_all - c * kChunk, kChunk));
#pragma unroll
    for (int n = 0; n < NB; n += 2) store8(ro, at + n * 32 + g * 16, zero);
  }
  if (!p.seg && p.s_out) s.store_matrix(p.s_out + (int64_t)pair * D * D, wave, lane);
}

// The three gradients of a call in one launch: first the workgroups for dk and dv of `g`, which take longest, then those for dq of `a`.  233 us at 16384
// tokens of 32 and 8 heads of 128 (0.80 GB, 3.4 TB/s).  (With a state of one term: both kinds alternating by eights, so that a segment's do, k and v would come from memory
// once for both: 256 us when this order took 227.  A head's q and do asked for while the one before is worked on: no change, but for heads of
// 64 of which very many share a KV head, a fifth less at 32 of one.)
template <int D, int SPLIT>
__global__ __launch_bounds__(64 * kLinWaves, 4) void linear_grad_kernel(const LinearArgs a, const LinearArgs g, int segments, int parts) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  int id = blockIdx.x;
  const bool keys = id < segments;
  if (!keys) id -= segments;
  if (keys) segment_keys<D, SPLIT>(g, id, smem);
  else segment_out<D, SPLIT>(a, id % segments, id / segments, parts, smem);
}

// ------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------
constexpr int kMostSegments = 1024;   // of a call that cuts its sequences

// Segments of a sequence, a whole number of chunks each, and the parts into which a group's query heads are dealt where there are few segments.
struct LinearPlan { int seg_chunks, nseg, parts; };

// Time in us of a call whose sequences are cut into n: chains of chunks, or the bytes that move where they take longer.  The constants (us for a chunk, D 128,
// 64, 32: a workgroup of linear_out_kernel with up to two heads, and for a further two; one for dk and dv, and for each head of the group; one tile pair of
// linear_segment_kernel) are 1.3 times what single workgroups took with their inputs in the caches and a state of one term.  Workgroups that share compute
// units take 1.3 (1.6) times as long; 4.3 TB/s.  Over 152 shapes of 128 to 8192 tokens, timed with every power of two, the choice is 1 % slower than the
// best on average, at worst 1.24 times (92 us for 74); one segment throughout would be 3.9 times slower, always the most 1.2 times.
static double linear_time(bool backward, double pairs, int chunks, int G, int64_t D, int n, LinearPlan* plan) {
  static const double kStep[3][5] = {{6.5, 3.3, 4.7, 3.6, 2.9}, {3.5, 1.7, 2.5, 2.2, 1.6}, {2.5, 1.0, 1.7, 1.4, 1.2}};
  const double* c = kStep[D == 128 ? 0 : D == 64 ? 1 : 2];
  const double bytes_us = 4.3e6, tile = 2.0 * kChunk * D / bytes_us, slots = D == 128 ? 512 : 768;
  const int sc = (chunks + n - 1) / n;
  n = (chunks + sc - 1) / sc;
  const double segs = pairs * n, state = n > 1 ? segs * D * D * 4 * (backward ? 2 : 1) / bytes_us : 0.0;
  const double half = backward ? 256 : 512;   // a backward's other workgroups, for dk and dv, fill the rest
  int parts = (int)(segs < half ? (half + segs - 1) / segs : 1);
  if (parts > G) parts = G;
  const int heads = (G + parts - 1) / parts;
  parts = (G + heads - 1) / heads;   // none without a head
  *plan = LinearPlan{sc, n, parts};
  const auto most = [](double a, double b) { return a > b ? a : b; };
  const auto rounds = [](double work, double at_once) { return (double)(int64_t)((work + at_once - 1) / at_once); };
  const auto busy = [](double blocks, double by) { return blocks > 256 ? by : 1.0; };
  double t = 3.0;
  if (n > 1) {
    t += 4.0 + most(sc * c[4] * (backward ? G : 1) * rounds(segs * (backward ? 2 : 1), slots), pairs * chunks * tile * 2 * (backward ? 1 + G : 1) + state);
    t += 4.0 + 1.5 * state + 0.12 * n;   // (states come from caches in part)
  }
  if (!backward)
    t += most(sc * (c[0] + c[1] * ((heads + 1) / 2 - 1)) * rounds(segs * parts, slots) * busy(segs * parts, 1.3), pairs * chunks * tile * (2 * G + 2 * parts) + state);
  else
    t += most(sc * (c[2] + c[3] * G) * rounds(segs, slots / 2) * busy(segs * (1 + parts), 1.6), pairs * chunks * tile * (4 * G + 4 + 2 * parts) + state);
  return t;
}
static LinearPlan linear_plan(bool backward, int64_t pairs, int64_t S, int64_t Hq, int64_t Hkv, int64_t D) {
  const int chunks = (int)((S + kChunk - 1) / kChunk), G = (int)(Hq / Hkv);
  LinearPlan best, p;
  double t = linear_time(backward, (double)pairs, chunks, G, D, 1, &best);
  for (int n = 2; n <= chunks && pairs * n <= kMostSegments; n *= 2) {
    const double u = linear_time(backward, (double)pairs, chunks, G, D, n, &p);
    if (u < t) {
      t = u;
      best = p;
    }
  }
  return best;
}
void query_linear_attention_plan(bool backward, int64_t B, int64_t S, int64_t Hq, int64_t Hkv, int64_t dh, int32_t* plan) {
  const LinearPlan p = linear_plan(backward, B * Hkv, S, Hq, Hkv, dh);
  plan[0] = p.seg_chunks;
  plan[1] = p.nseg;
  plan[2] = p.parts;
}
// room for the states of all segments: a size that does not fall as the call grows
static size_t segment_bytes(int64_t pairs, int64_t S, int64_t dh) {
  const int64_t chunks = (S + kChunk - 1) / kChunk;
  const int64_t n = pairs < kMostSegments && pairs * chunks < kMostSegments ? pairs * chunks : kMostSegments;
  return (size_t)(n * dh * dh) * sizeof(float);
}
size_t linear_attention_fwd_workspace(int64_t B, int64_t S, int64_t Hq, int64_t Hkv, int64_t dh) { return segment_bytes(B * Hkv, S, dh); }
size_t linear_attention_bwd_workspace(int64_t B, int64_t S, int64_t Hq, int64_t Hkv, int64_t dh) { return 2 * segment_bytes(B * Hkv, S, dh); }

static LinearArgs linear_args(const LinearCall& c, const LinearPlan& plan) {
  LinearArgs a{};
  a.q = (const bf16_t*)c.q; a.k = (const bf16_t*)c.k; a.v = (const bf16_t*)c.v;
  a.log_decay = c.log_decay; a.lengths = c.lengths;
  a.S = (int)c.S; a.Hq = (int)c.Hq; a.Hkv = (int)c.Hkv;
  a.seg_chunks = plan.seg_chunks; a.nseg = plan.nseg; a.scale = c.scale;
  return a;
}

// the states (gradients) between segments, in a.seg (and g.seg, if g is given)
template <int D>
static int run_states(const LinearArgs& a, const LinearArgs* g, int64_t pairs, hipStream_t st) {
  const auto segments = g ? linear_segment_kernel<D, true> : linear_segment_kernel<D, false>;
  hipLaunchKernelGGL(segments, dim3((unsigned)(pairs * a.nseg), g ? 2 : 1), dim3(64 * kLinWaves), 2 * kChunk * D * 2 + kChunk * sizeof(float), st,
                     a, g ? *g : a);
  if (int rc = check_launch("linear attention (segments)")) return rc;
  hipLaunchKernelGGL(linear_scan_kernel<D>, dim3((unsigned)(pairs * (D * D / 1024)), g ? 2 : 1), dim3(256), 0, st, a, g ? *g : a);
  return check_launch("linear attention (scan)");
}

template <int D> constexpr size_t kLinearLds = 2 * kChunk * D * 2 + kStateLds<D> + (kLinWaves + kChunk) * sizeof(float);

template <int D, int SPLIT>
static int launch_out(const LinearArgs& a, int64_t segments, int parts, hipStream_t st) {
  static std::atomic<unsigned long long> done;
  if (int rc = reserve_lds(linear_out_kernel<D, SPLIT>, kLinearLds<D>, done, "linear_attention_forward")) return rc;
  hipLaunchKernelGGL((linear_out_kernel<D, SPLIT>), dim3((unsigned)(segments * parts)), dim3(64 * kLinWaves), kLinearLds<D>, st, a, (int)segments, parts);
  return check_launch("linear_attention_forward");
}
template <int D>
static int run_forward(LinearArgs a, int64_t pairs, int parts, float* workspace, hipStream_t st) {
  const int64_t segments = pairs * a.nseg;
  if (a.nseg > 1 || (parts > 1 && a.s_out)) {
    a.seg = workspace;
    if (int rc = run_states<D>(a, nullptr, pairs, st)) return rc;
  }
  return a.nseg > 1 ? launch_out<D, 2>(a, segments, parts, st) : launch_out<D, 3>(a, segments, parts, st);
}

template <int D, int SPLIT>
static int launch_grad(const LinearArgs& a, const LinearArgs& g, int64_t segments, int parts, hipStream_t st) {
  static std::atomic<unsigned long long> done;
  if (int rc = reserve_lds(linear_grad_kernel<D, SPLIT>, kLinearLds<D>, done, "linear_attention_backward")) return rc;
  hipLaunchKernelGGL((linear_grad_kernel<D, SPLIT>), dim3((unsigned)(segments * (1 + parts))), dim3(64 * kLinWaves), kLinearLds<D>, st, a, g,
                     (int)segments, parts);
  return check_launch("linear_attention_backward");
}
template <int D>
static int run_backward(LinearArgs a, LinearArgs g, int64_t pairs, int parts, float* workspace, hipStream_t st) {
  const int64_t segments = pairs * a.nseg;
  if (a.nseg > 1) {
    a.seg = workspace;
    g.seg = workspace + segments * D * D;
    if (int rc = run_states<D>(a, &g, pairs, st)) return rc;
    return launch_grad<D, 2>(a, g, segments, parts, st);
  }
  return launch_grad<D, 3>(a, g, segments, parts, st);
}

int launch_linear_attention_fwd(const LinearCall& c, const float* s_in, void* o, float* s_out, void* workspace, hipStream_t st) {
  const int64_t pairs = c.B * c.Hkv;
  const LinearPlan plan = linear_plan(false, pairs, c.S, c.Hq, c.Hkv, c.dh);
  LinearArgs a = linear_args(c, plan);
  a.o = (bf16_t*)o; a.s_in = s_in; a.s_out = s_out;
  const auto run = c.dh == 128 ? run_forward<128> : c.dh == 64 ? run_forward<64> : run_forward<32>;
  return run(a, pairs, plan.parts, (float*)workspace, st);
}

int launch_linear_attention_bwd(const LinearCall& c, const float* s_in, const void* d_o, const float* ds_out, void* dq, void* dk, void* dv,
                                float* ds_in, void* workspace, hipStream_t st) {
  // dq is the forward's o of (d_o, v, k) and the transposed state
  const int64_t pairs = c.B * c.Hkv;
  const LinearPlan plan = linear_plan(true, pairs, c.S, c.Hq, c.Hkv, c.dh);
  LinearArgs a = linear_args(c, plan), g = a;
  a.q = (const bf16_t*)d_o; a.k = (const bf16_t*)c.v; a.v = (const bf16_t*)c.k;
  a.o = (bf16_t*)dq; a.s_in = s_in; a.flip = 1;
  g.d_o = (const bf16_t*)d_o; g.dk = (bf16_t*)dk; g.dv = (bf16_t*)dv; g.s_in = ds_out; g.s_out = ds_in;
  const auto run = c.dh == 128 ? run_backward<128> : c.dh == 64 ? run_backward<64> : run_backward<32>;
  return run(a, g, pairs, plan.parts, (float*)workspace, st);
}

// ------------------------------------------------------------------------------------------
// One token for every batch row.  Bound by HBM: the state is read and written once, 8 bytes an element: 256 rows of 8 states of 128 x 128 in 60
// us (0.28 GB, 4.7 TB/s, a copy's rate; 46.5 us where the memory's side cache holds a part of them from call to call); of one row by what waits for each other, 3.9 us.  Workgroup: COLS columns of one state; a thread holds four columns of
// every RG-th row, so that the state stays in registers between its update and the products with the group's queries.  HEADS of these at once, read
// before the state is: one after the other a group of four takes 4.6 and, from that cache, 49 us; but four where there is one, 6.6 us for 4.6 (40 rows of 12
// heads of 64), and one of two 4.6 for 4.2.
// ------------------------------------------------------------------------------------------
template <int D, int COLS, int HEADS>
__global__ __launch_bounds__(256) void linear_step_kernel(const bf16_t* __restrict__ q, const bf16_t* __restrict__ k, const bf16_t* __restrict__ v,
                                                          const float* __restrict__ log_decay, const int64_t* __restrict__ lengths,
                                                          float* __restrict__ state, int Hq, int Hkv, float scale, bf16_t* __restrict__ o) {
  constexpr int CV = COLS / 4, RG = 256 / CV, R = D / RG;
  static_assert(D % RG == 0, "every thread holds R rows");
  __shared__ f32x4 red[4][HEADS][CV];
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
  float qv[HEADS][R];
  auto load_queries = [&](int h0) {
#pragma unroll
    for (int n = 0; n < HEADS; ++n)
#pragma unroll
      for (int i = 0; i < R; ++i) qv[n][i] = (float)qp[(int64_t)min(h0 + n, G - 1) * D + i * RG + rg];
  };
  load_queries(0);
  const Decay lam = decay_of(log_decay[j], 1);
  const bf16_t* kp = k + (int64_t)pair * D;
  const bf16x4 vv = *reinterpret_cast<const bf16x4*>(v + (int64_t)pair * D + c);
  float* sp = state + (int64_t)pair * D * D + c;
  f32x4 s[R];
#pragma unroll
  for (int i = 0; i < R; ++i) s[i] = *reinterpret_cast<const f32x4*>(sp + (i * RG + rg) * D);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const float kk = (float)kp[i * RG + rg];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[i][e] = decayed(lam, s[i][e], kk * (float)vv[e]);
    *reinterpret_cast<f32x4*>(sp + (i * RG + rg) * D) = s[i];
  }
  for (int h0 = 0; h0 < G; h0 += HEADS) {
    f32x4 acc[HEADS];
#pragma unroll
    for (int n = 0; n < HEADS; ++n) {
      acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < R; ++i) acc[n] += s[i] * qv[n][i];
    }
    if (h0 + HEADS < G) load_queries(h0 + HEADS);
#pragma unroll
    for (int off = CV; off < 64; off <<= 1)
#pragma unroll
      for (int n = 0; n < HEADS; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] += __shfl_xor(acc[n][e], off, 64);
    if (h0 > 0) __syncthreads();
    if ((threadIdx.x & 63) < CV)
#pragma unroll
      for (int n = 0; n < HEADS; ++n) red[wave][n][cv] = acc[n];
    __syncthreads();
    const int h = h0 + threadIdx.x / CV;
    if (threadIdx.x < HEADS * CV && h < G) {
      const int n = threadIdx.x / CV;
      const f32x4 t = ((red[0][n][cv] + red[1][n][cv]) + (red[2][n][cv] + red[3][n][cv])) * scale;
      bf16x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = (bf16_t)t[e];
      *reinterpret_cast<bf16x4*>(op + (int64_t)h * D + c) = w;
    }
  }
}

int launch_linear_attention_step(const LinearCall& c, float* state, void* o, hipStream_t st) {
  const int64_t pairs = c.B * c.Hkv;
  const int64_t G = c.Hq / c.Hkv;
#define STEP(D, HEADS)                                                                                                          \
  hipLaunchKernelGGL((linear_step_kernel<D, 32, HEADS>), dim3((unsigned)pairs, D / 32), dim3(256), 0, st, (const bf16_t*)c.q,   \
                     (const bf16_t*)c.k, (const bf16_t*)c.v, c.log_decay, c.lengths, state, (int)c.Hq, (int)c.Hkv, c.scale, (bf16_t*)o)
#define STEP_HEADS(D) if (G > 2) STEP(D, 4); else if (G == 2) STEP(D, 2); else STEP(D, 1)
  if (c.dh == 128) { STEP_HEADS(128); }
  else if (c.dh == 64) { STEP_HEADS(64); }
  else { STEP_HEADS(32); }
#undef STEP_HEADS
#undef STEP
  return check_launch("linear_attention_step");
}

}  // namespace dl
