// What the attention kernels share: [rows][head_dim] tiles in LDS with their swizzle and operand reads, score tiles in registers, and the order of
// workgroups.
//
// An MFMA sums over its 16 k-slots in any order, so the slot -> key assignment is chosen to match the accumulator layout of the score tile: for a
// 16-key step, slot (half = lane / 32, e = 0..7) holds key 8*(e/4) + 4*half + e%4.  The transposed loads of the other operand use the same map.
#pragma once
#include "common.h"

namespace dl {

constexpr float kLn2 = 0.6931471805599453f;

// v_exp_f32: 2^x without the denormal-range fix-up (results below 2^-126 flush to zero, which is
// what a softmax weight that small should be anyway).
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ __amdgpu_buffer_rsrc_t attn_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}

// [ROWS][DH] bf16 tile in LDS, DH*2 bytes per row, 16-byte chunk c of row r stored at chunk
// c ^ swz(r).  Loaded by NW waves with 1 KiB wave-wide async loads.  swz is chosen so that both
// access patterns are free of bank conflicts (the LDS serves 256 B of banks per clock):
//   row reads  (ds_read_b128, 16 lanes = 16 consecutive rows, one logical chunk), and
//   transposed reads (ds_read_b64_tr_b16, 32 lanes = 4 consecutive rows x 64 B).
template <int ROWS, int DH, int NW>
struct RowTile {
  static constexpr int ROW_B = DH * 2;
  static constexpr int LPR = DH / 8;          // lanes (16 B chunks) per row
  static constexpr int RPI = 1024 / ROW_B;    // rows per wave-wide load
  static constexpr int NINSTR = ROWS / RPI;
  static constexpr int PER_WAVE = NINSTR / NW;
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (LPR == 16) { const int i = row & 15; return ((i & 3) << 2) | (i >> 2); }
    else if constexpr (LPR == 8) { const int i = (row >> 1) & 7; return ((i & 1) << 2) | (i >> 1); }
    else { return (row >> 2) & 3; }
  }
  static_assert(NINSTR % NW == 0 && ((ROWS / NW) % 16) == 0, "tile split");
  static constexpr int BYTES = ROWS * ROW_B;

  // rs describes memory starting at the tile's first row; ld = row stride in elements.
  // AUX: cache-policy bits of the load (0 = default, 2 = non-temporal)
  template <int AUX = 0>
  static __device__ __forceinline__ void issue(__amdgpu_buffer_rsrc_t rs, char* lds_tile, int wave,
                                               int lane, int64_t ld) {
    const int r = lane / LPR, pc = lane % LPR;
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      const int j = wave * PER_WAVE + i;
      const int c = pc ^ swz(i * RPI + r);   // rows per wave are a multiple of 16
      const uint32_t vo = (uint32_t)(r * ld * 2 + (c << 4));
      const uint32_t so = (uint32_t)((int64_t)j * RPI * ld * 2);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LDS_PTR(void))(lds_tile + j * 1024), 16, vo, so, 0, AUX);
    }
  }
  // MFMA operand for rows row0 + lane%32, contraction over the DH index, step kk (16 of DH).
  static __device__ __forceinline__ bf16x8 frag_rows(const char* t, int row0, int kk, int lane) {
    const int row = row0 + (lane & 31);
    const int c = (kk * 2 + (lane >> 5)) ^ swz(row);
    return *reinterpret_cast<const bf16x8*>(t + row * ROW_B + (c << 4));
  }
  // MFMA operand for "rows" = 32 columns of the tile starting at col0 (the DH index), contraction
  // over 16 tile rows starting at krow0, with the slot -> row map described at the top of the file.
  static __device__ __forceinline__ bf16x8 frag_cols(const char* t, int col0, int krow0, int lane) {
    const int grp = lane >> 4, s = lane & 15, e = s >> 2, g = s & 3;
    const int col = col0 + ((grp & 1) << 4) + (g << 2);
    const int row = krow0 + ((grp >> 1) << 2) + e;
    const char* p0 = t + row * ROW_B + ((((col >> 3) ^ swz(row)) << 4) | ((col & 7) << 1));
    const int row2 = row + 8;
    const char* p1 = t + row2 * ROW_B + ((((col >> 3) ^ swz(row2)) << 4) | ((col & 7) << 1));
    bf16x8 v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(p0));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(p1));
    return v;
  }
};

__device__ __forceinline__ bf16x8 pack_slots(const f32x16& a, int first) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (bf16_t)a[first + e];
  return v;
}


// Value exchange between lane l and lane l ^ 32 without the LDS round trip of a bpermute: after the swap
// `a` holds the low half's values in both halves and `b` the high half's.
__device__ __forceinline__ float max_across_halves(float x) {
  float a = x, b = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  return __builtin_fmaxf(a, b);
}
__device__ __forceinline__ float sum_across_halves(float x) {
  float a = x, b = x;
  asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
  return a + b;
}
// max of three as one instruction, without the canonicalising self-maximum the compiler puts in front of
// fmaxf operands (scores are finite or -inf here, never NaN)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

// Causal mask for a score tile held in the "lane owns one query (or key) column" accumulator
// layout: register r of 32-row block i holds row i*32 + 8*(r/4) + 4*(lane/32) + r%4.  `lim` is the
// largest row offset this lane may keep (computed by the caller with the 4*(lane/32) folded in);
// rows above it get `fill`.  The empty volatile asm keeps the compiler from turning the caller's
// wave-uniform `if (diagonal tile)` into per-element selects executed on every tile.
template <int NBLK>
__device__ __forceinline__ void mask_rows_above(f32x16 (&s)[NBLK], int lim, float fill) {
  asm volatile("" ::: "memory");
#pragma unroll
  for (int i = 0; i < NBLK; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (i * 32 + ((r >> 2) << 3) + (r & 3) > lim) s[i][r] = fill;
}

// ------------------------------------------------------------------------------------------
// Workgroup -> work mapping shared by all kernels here.  Consecutive workgroup ids are dealt to the
// eight XCDs in turn and every XCD has an L2 of its own, so all work on one (batch, kv head) pair is
// given to ONE XCD (ids congruent mod 8) when the number of pairs is a multiple of 8: the K/V tiles
// (forward, dQ) or Q/dO tiles (dK, dV) of that pair are then fetched into one L2 only, and the
// workgroups that share them run side by side and walk them in the same order.  `j` counts the
// position in the pair's own queue (heaviest first is the caller's business).
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ void split_block_id(int id, int npairs, int& j, int& pair) {
  int per_xcd = npairs, xcd = 0, slot = id;
  if ((npairs & 7) == 0) { per_xcd = npairs >> 3; xcd = id & 7; slot = id >> 3; }
  j = slot / per_xcd;
  pair = xcd * per_xcd + slot % per_xcd;
}

}  // namespace dl
