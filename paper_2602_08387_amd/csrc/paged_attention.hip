// Softmax attention of new tokens over a paged cache of keys and values:
//
//   o = sum_s w_s v_s / sum_s w_s,  w_s = exp(scale q . k_s - m),  s = 0 .. the token's own position;   lse = m + log sum_s w_s
//
// One pass over the keys with the running maximum and sum.  The query heads of a KV head's group share its keys, so a matrix product's rows are (token,
// head of the group) pairs, row = token * group + head: the keys of a group are read once for all of them.
//
// tile_kernel: workgroup = 128 rows of one (batch row, KV head), four waves of 32; score tiles S^T[key][row] = K Q^T on v_mfma_f32_32x32x16_bf16, whose
// layout is that of the next product's operand, O^T[d][row] += V^T P^T.  Tiles of 64 keys stream to LDS, double buffered; a wave loads the 16 keys of
// its own part of the tile, which lie in one page (a page has 16 tokens or a multiple), so a tile needs one page number a wave.  bf16 pages go to LDS
// directly; e4m3 comes through registers, where it becomes the bf16 values that it stands for.  The keys can be split over workgroups, whose sums
// combine_kernel joins.
//
// Rows behind a tile's last key and pages that do not exist are behind the end of the buffer that a load is given, and read as zeros: what a page
// holds behind a row's last token is never read.
#include "attention_tile.h"
#include "common.h"
#include "kernels.h"
#include "paged_cache.h"

namespace dl {

constexpr float kNoKey = -1e30f;       // a maximum before the first key: finite, so that exp2(-inf - m) is 0 and not NaN
constexpr int kTileRows = 128, kTileKeys = 64;

struct AttendArgs {
  PagedCache cache;
  const bf16_t* q;                     // [batch][seq][Hq][DH]
  const int64_t *start, *lengths;
  bf16_t* o;
  float* lse;                          // [batch][Hq][seq] or null
  float *sums, *stats;                 // parts of a split: [pair][tile][split][rows][DH], and maximum and sum of a row [..][rows][2]
  int seq, Hq, group, tiles, splits;
  float scale_log2;
};

// Where a row's result goes: (token, query head) of row r of a pair's rows.
struct RowPlace { int t, h; };
__device__ __forceinline__ RowPlace row_place(const AttendArgs& a, int hk, int r) {
  const int t = r / a.group;
  return {t, hk * a.group + (r - t * a.group)};
}

// page_of for a position that is the wave's: a scalar load (the table is not written to while the kernel runs).
__device__ __forceinline__ int page_of_wave(const PagedCache& c, int b, int p) {
  if ((p >> c.shift) >= c.columns) return -1;
  const auto* table = (__attribute__((address_space(4))) const int32_t*)(uintptr_t)c.table;
  const int page = table[(int64_t)b * c.columns + (p >> c.shift)];
  return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}

// The keys of one wave's 16 rows of a tile: first vector in the cache, and how many of the 16 there are.
struct Keys16 { int64_t vec; int n; };
__device__ __forceinline__ Keys16 keys16(const PagedCache& c, int b, int hk, int p, int end) {
  const int page = p < end ? page_of_wave(c, b, p) : -1;
  if (page < 0) return {0, 0};
  const int n = end - p;
  return {vector_of(c, page, hk, p), n < 16 ? n : 16};
}

// Whether one of 8 bf16 is infinite or NaN; and: those out of v, with a 1 for each in count.
__device__ __forceinline__ bool any_not_finite(const bf16x8& v) {
  const u32x4 u = __builtin_bit_cast(u32x4, v);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= (u[i] & 0x7f80u) == 0x7f80u || (u[i] & 0x7f800000u) == 0x7f800000u;
  return odd;
}
__device__ __forceinline__ void split_not_finite(bf16x8& v, bf16x8& count) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool odd = !(fabsf((float)v[e]) < INFINITY);
    count[e] = (bf16_t)(odd ? 1.f : 0.f);
    if (odd) v[e] = (bf16_t)0.f;
  }
}

template <int DH, bool E4M3>
__global__ __launch_bounds__(256, 2) void tile_kernel(const AttendArgs a) {
  using Tile = RowTile<kTileKeys, DH, 4>;
  constexpr int STAGE = 2 * Tile::BYTES;
  // e4m3: a lane's part of a wave's 16 keys
  constexpr int PER_LANE = DH / 4, CHUNK = PER_LANE < 16 ? PER_LANE : 16, NLOAD = PER_LANE / CHUNK, LANES = DH / CHUNK, ROWS = 64 / LANES;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const PagedCache& c = a.cache;
  int j, pair;
  split_block_id((int)blockIdx.x, c.batch * c.heads, j, pair);
  const int b = pair / c.heads, hk = pair % c.heads;
  const int tile = a.tiles - 1 - j / a.splits, split = j % a.splits;     // long rows (late tokens) first
  const int lq = lane & 31, half = lane >> 5;
  const int n_rows = row_length(a.lengths, b, a.seq) * a.group, row0 = tile * kTileRows;
  const int r = row0 + wave * 32 + lq;

  // keys that the tile's last row sees, and this lane's row: positions 0 .. lim
  const int64_t start = row_start(a.start, b), cap = (int64_t)c.columns << c.shift;
  const auto last_key = [&](int row) { const int64_t p = start + row / a.group; return (int)(p < -1 ? -1 : p >= cap ? cap - 1 : p); };
  const int end = row0 < n_rows ? last_key(min(row0 + kTileRows, n_rows) - 1) + 1 : 0;
  const int lim = n_rows > 0 ? last_key(min(r, n_rows - 1)) : -1, lim0 = __builtin_amdgcn_readfirstlane(lim);
  // the last key that any of the wave's rows sees; none for a wave behind the last row
  const int lim1 = row0 + wave * 32 < n_rows ? __builtin_amdgcn_readlane(lim, 31) : -1;
  const int all = (end + kTileKeys - 1) / kTileKeys, per = (all + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = min(all, t0 + per);

  f32x16 oacc[DH / 32];
#pragma unroll
  for (int t = 0; t < DH / 32; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) oacc[t][e] = 0.f;
  float m = kNoKey, lsum = 0.f;        // m: reference exponent in scaled log2 units

  if (t0 < t1) {
    // pages that do not exist take their keys out of the sum: looked for once, so that no tile has to ask where all are there
    bool missing = false;
    for (int i = (t0 * kTileKeys >> c.shift) + threadIdx.x, n = (min(end, t1 * kTileKeys) - 1) >> c.shift; i <= n; i += 256)
      missing |= (uint32_t)c.table[(int64_t)b * c.columns + i] >= (uint32_t)c.n_pages;
    missing = __syncthreads_or(missing);

    bf16x8 qf[DH / 16];
    {
      const RowPlace at = row_place(a, hk, min(r, n_rows - 1));
      const bf16_t* qp = a.q + (((int64_t)b * a.seq + at.t) * a.Hq + at.h) * DH + half * 8;
#pragma unroll
      for (int kk = 0; kk < DH / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 16);
    }

    u32x4 raw[2][NLOAD];               // e4m3: the next tile's
    float scl[2][NLOAD];
    const auto load = [&](int t, int stage) {
      const Keys16 k16 = keys16(c, b, hk, t * kTileKeys + wave * 16, end);
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if constexpr (!E4M3) {
          const auto rs = attn_rsrc(c.x[w] + k16.vec * (DH * 2), (uint32_t)(k16.n * DH * 2));
          char* to = smem + stage * STAGE + w * Tile::BYTES + wave * (16 * DH * 2);
#pragma unroll
          for (int i = 0; i < Tile::PER_WAVE; ++i) {
            const int row = i * Tile::RPI + lane / Tile::LPR, ch = (lane % Tile::LPR) ^ Tile::swz(row);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (LDS_PTR(void))(to + i * 1024), 16, row * (DH * 2) + (ch << 4), 0, 0, 0);
          }
        } else {
          const auto rs = attn_rsrc(c.x[w] + k16.vec * DH, (uint32_t)(k16.n * DH));
          const auto ss = attn_rsrc(c.scale[w] + k16.vec, (uint32_t)k16.n);
#pragma unroll
          for (int i = 0; i < NLOAD; ++i) {
            const int row = i * ROWS + lane / LANES, at = row * DH + (lane % LANES) * CHUNK;
            if constexpr (CHUNK == 16) raw[w][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0));
            else { const u32x2 u = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, 0)); raw[w][i][0] = u[0]; raw[w][i][1] = u[1]; }
            scl[w][i] = __uint_as_float((uint32_t)__builtin_amdgcn_raw_buffer_load_b8(ss, row, 0, 0) << 23);
          }
        }
      }
    };
    const auto unpack = [&](int stage) {
      if constexpr (E4M3) {
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int i = 0; i < NLOAD; ++i) {
            const int row = wave * 16 + i * ROWS + lane / LANES, ch = (lane % LANES) * (CHUNK / 8);
            char* to = smem + stage * STAGE + w * Tile::BYTES + row * Tile::ROW_B;
#pragma unroll
            for (int h = 0; h < CHUNK / 8; ++h)
              *reinterpret_cast<bf16x8*>(to + (((ch + h) ^ Tile::swz(row)) << 4)) = unpack_e4m3(u32x2{raw[w][i][2 * h], raw[w][i][2 * h + 1]}, scl[w][i]);
          }
      }
    };

    load(t0, 0);
    unpack(0);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int stage = 0;
    for (int t = t0; t < t1; ++t) {
      if (t + 1 < t1) load(t + 1, stage ^ 1);
      const int kv0 = t * kTileKeys;
      const char* tk = smem + stage * STAGE;
      const char* tv = tk + Tile::BYTES;
      if (kv0 <= lim1) {
      f32x16 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
#pragma unroll
      for (int kk = 0; kk < DH / 16; ++kk)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::frag_rows(tk, i * 32, kk, lane), qf[kk], s[i], 0, 0, 0);
      // keys after the row's own position (only on tiles that reach past this wave's first row)
      const bool masked = kv0 + kTileKeys - 1 > lim0;
      if (masked) mask_rows_above<2>(s, lim - kv0 - (half << 2), -INFINITY);
      if (missing) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if (page_of_wave(c, b, kv0 + g * 16) < 0)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[g >> 1][(g & 1) * 8 + e] = -INFINITY;
      }
      float mx = s[0][0];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[i][e]);
      mx = max_across_halves(mx) * a.scale_log2;
      // raised only where some row's maximum grew by more than 2^8: weights stay below 256, and sum and result carry the same reference
      if (__builtin_amdgcn_ballot_w64(mx > m + 8.0f) != 0) {
        const float m_new = fmaxf(m, mx);
        const float alpha = fast_exp2(m - m_new);
        lsum *= alpha;
        m = m_new;
#pragma unroll
        for (int t2 = 0; t2 < DH / 32; ++t2)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[t2][e] *= alpha;
      }
      float psum = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float pv = fast_exp2(__builtin_fmaf(s[i][e], a.scale_log2, -m));
          s[i][e] = pv;
          psum += pv;
        }
      lsum += psum;
      // a weight of 0 times a value that is not finite is NaN: where a masked tile holds such values, they are counted apart, for the rows that see them
      bool odd = false;
      if (masked) {
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int t2 = 0; t2 < DH / 32; ++t2) odd |= any_not_finite(Tile::frag_cols(tv, t2 * 32, ks * 16, lane));
        odd = __builtin_amdgcn_ballot_w64(odd) != 0;
      }
      if (!odd) {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const bf16x8 pf = pack_slots(s[ks >> 1], (ks & 1) * 8);
#pragma unroll
          for (int t2 = 0; t2 < DH / 32; ++t2)
            oacc[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Tile::frag_cols(tv, t2 * 32, ks * 16, lane), pf, oacc[t2], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          const bf16x8 pf = pack_slots(s[ks >> 1], (ks & 1) * 8);
          bf16x8 seen;
#pragma unroll
          for (int e = 0; e < 8; ++e) seen[e] = (bf16_t)(kv0 + ks * 16 + ((e >> 2) << 3) + (half << 2) + (e & 3) <= lim ? 1.f : 0.f);
#pragma unroll
          for (int t2 = 0; t2 < DH / 32; ++t2) {
            bf16x8 v = Tile::frag_cols(tv, t2 * 32, ks * 16, lane), count;
            split_not_finite(v, count);
            f32x16 n;
#pragma unroll
            for (int e = 0; e < 16; ++e) n[e] = 0.f;
            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(count, seen, n, 0, 0, 0);
            oacc[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf, oacc[t2], 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 16; ++e) oacc[t2][e] = n[e] > 0.f ? NAN : oacc[t2][e];
          }
        }
      }
      }
      if (t + 1 < t1) unpack(stage ^ 1);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      stage ^= 1;
    }
    lsum = sum_across_halves(lsum);
  }

  if (a.splits > 1) {
    const int64_t at = ((((int64_t)pair * a.tiles + tile) * a.splits + split) * kTileRows) + wave * 32 + lq;
    if (half == 0) {
      a.stats[at * 2] = m;
      a.stats[at * 2 + 1] = lsum;
    }
    if (t0 >= t1) return;
    float* op = a.sums + at * DH + half * 4;
#pragma unroll
    for (int t2 = 0; t2 < DH / 32; ++t2)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 ov = {oacc[t2][g * 4], oacc[t2][g * 4 + 1], oacc[t2][g * 4 + 2], oacc[t2][g * 4 + 3]};
        *reinterpret_cast<f32x4*>(op + t2 * 32 + g * 8) = ov;
      }
    return;
  }
  if (r >= a.seq * a.group) return;
  const bool any = r < n_rows && lsum != 0.f;          // a sum that is NaN is one
  const float inv = any ? 1.0f / lsum : 0.f;
  const RowPlace at = row_place(a, hk, r);
  bf16_t* op = a.o + (((int64_t)b * a.seq + at.t) * a.Hq + at.h) * DH + half * 4;
#pragma unroll
  for (int t2 = 0; t2 < DH / 32; ++t2)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 ov;
#pragma unroll
      for (int e = 0; e < 4; ++e) ov[e] = (bf16_t)(any ? oacc[t2][g * 4 + e] * inv : 0.f);
      *reinterpret_cast<bf16x4*>(op + t2 * 32 + g * 8) = ov;
    }
  if (a.lse && half == 0) a.lse[((int64_t)b * a.Hq + at.h) * a.seq + at.t] = any ? (m + log2f(lsum)) * kLn2 : -INFINITY;
}

// Joins the parts of split rows: DH / 4 lanes a row.
template <int DH>
__global__ __launch_bounds__(256) void combine_kernel(const AttendArgs a, int64_t rows, int rows_per_tile) {
  constexpr int LPR = DH / 4;
  const PagedCache& c = a.cache;
  const int64_t i = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;      // (pair, row of the pair)
  if (i >= rows) return;
  const int per_pair = a.seq * a.group, d = (threadIdx.x % LPR) * 4;
  const int64_t pair = i / per_pair;
  const int r = (int)(i % per_pair), b = (int)(pair / c.heads), hk = (int)(pair % c.heads);
  const int64_t first = (pair * a.tiles + r / rows_per_tile) * a.splits;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = kNoKey, sum = 0.f;
  if (r < row_length(a.lengths, b, a.seq) * a.group) {
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.stats[((first + s) * rows_per_tile + r % rows_per_tile) * 2]);
    for (int s = 0; s < a.splits; ++s) {
      const int64_t at = (first + s) * rows_per_tile + r % rows_per_tile;
      const float l = a.stats[at * 2 + 1];
      if (l == 0.f) continue;
      const float w = fast_exp2(a.stats[at * 2] - m);
      sum += w * l;
      acc += w * *reinterpret_cast<const f32x4*>(a.sums + at * DH + d);
    }
  }
  const RowPlace at = row_place(a, hk, r);
  const float inv = sum != 0.f ? 1.0f / sum : 0.f;
  bf16x4 ov;
#pragma unroll
  for (int e = 0; e < 4; ++e) ov[e] = (bf16_t)(acc[e] * inv);
  *reinterpret_cast<bf16x4*>(a.o + (((int64_t)b * a.seq + at.t) * a.Hq + at.h) * DH + d) = ov;
  if (a.lse && d == 0) a.lse[((int64_t)b * a.Hq + at.h) * a.seq + at.t] = sum != 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
}

// Which way a call goes.  Rows of tile_kernel's workgroups, tiles of a pair, and parts of a tile's keys: as many as fill the chip twice over, of no
// fewer than 4 tiles of keys each.
struct AttendPlan { int rows, tiles, splits; int64_t pairs; };
constexpr int kWorkgroupsWanted = 512;
static AttendPlan attend_plan(int64_t batch, int64_t seq, int64_t Hkv, int64_t group, int64_t max_tokens) {
  AttendPlan p;
  p.rows = kTileRows;
  p.pairs = batch * Hkv;
  p.tiles = (int)((seq * group + p.rows - 1) / p.rows);
  const int64_t have = p.pairs * p.tiles, most = (max_tokens + 4 * kTileKeys - 1) / (4 * kTileKeys);
  int64_t splits = have >= kWorkgroupsWanted ? 1 : kWorkgroupsWanted / have;
  if (splits > most) splits = most;
  p.splits = (int)(splits < 1 ? 1 : splits);
  return p;
}

// Sums and statistics of the parts.  Rows of all workgroups of a split call, bounded so that the size does not fall as the call grows: pairs * tiles *
// splits stays within kWorkgroupsWanted wherever there is a split at all.
size_t paged_attention_workspace(int64_t batch, int64_t seq, int64_t Hq, int64_t Hkv, int64_t dh, int64_t max_tokens) {
  return (size_t)kWorkgroupsWanted * kTileRows * (dh + 2) * sizeof(float);
}

template <int DH, bool E4M3>
static int launch_attend(AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  constexpr int lds = 2 * 2 * kTileKeys * DH * 2;
  static std::atomic<unsigned long long> done{0};
  if (int rc = reserve_lds(tile_kernel<DH, E4M3>, lds, done, "paged_attention_forward")) return rc;
  hipLaunchKernelGGL((tile_kernel<DH, E4M3>), dim3((unsigned)(p.pairs * p.tiles * p.splits)), dim3(256), lds, st, a);
  if (int rc = check_launch("paged_attention_forward")) return rc;
  if (p.splits == 1) return 0;
  const int64_t rows = p.pairs * a.seq * a.group;
  constexpr int per = 256 / (DH / 4);
  hipLaunchKernelGGL((combine_kernel<DH>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, st, a, rows, p.rows);
  return check_launch("paged_attention_forward, joining parts");
}

int launch_paged_attention(const CacheCall& c, const void* q, int64_t seq, int64_t Hq, float scale, void* o, float* lse, void* workspace,
                           hipStream_t st) {
  const AttendPlan p = attend_plan(c.batch, seq, c.heads, Hq / c.heads, c.columns * c.page_size);
  AttendArgs a{};
  a.cache = paged_cache(c);
  a.q = (const bf16_t*)q;
  a.start = c.start; a.lengths = c.lengths;
  a.o = (bf16_t*)o;
  a.lse = lse;
  a.stats = (float*)workspace;
  a.sums = a.stats + (int64_t)kWorkgroupsWanted * kTileRows * 2;
  a.seq = (int)seq; a.Hq = (int)Hq; a.group = (int)(Hq / c.heads);
  a.tiles = p.tiles; a.splits = p.splits;
  a.scale_log2 = scale * kLog2e;
  if (c.e4m3) return c.dh == 128 ? launch_attend<128, true>(a, p, st) : c.dh == 64 ? launch_attend<64, true>(a, p, st) : launch_attend<32, true>(a, p, st);
  return c.dh == 128 ? launch_attend<128, false>(a, p, st) : c.dh == 64 ? launch_attend<64, false>(a, p, st) : launch_attend<32, false>(a, p, st);
}

}  // namespace dl
