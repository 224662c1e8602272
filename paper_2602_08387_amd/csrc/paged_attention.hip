// Softmax attention of new tokens over a paged cache of keys and values:
//
//   o = sum_s w_s v_s / sum_s w_s,  w_s = exp(scale q . k_s - m),  s = 0 .. the token's own position;   lse = m + log sum_s w_s
//
// One pass over the keys with the running maximum and sum.  The query heads of a KV head's group share its keys, so a matrix product's rows are (token, head
// of the group) pairs, row = token * group + head: the keys of a group are read once for all of them.
//
// tile_kernel: workgroup = 128 rows of one (batch row, KV head), four waves of 32 (or 256 rows, eight waves); score tiles S^T[key][row] = K Q^T on
// v_mfma_f32_32x32x16_bf16, whose layout is that of the next product's operand, O^T[d][row] += V^T P^T.  Tiles of 64 (128) keys stream to LDS, double
// buffered; a wave loads the 16 keys of its own part of the tile, which lie in one page (a page has 16 tokens or a multiple), so a tile needs one page number
// a wave.  Loads go to LDS directly; a wave then writes its 16 keys of e4m3, in their place, as the bf16 values that they stand for.  The keys can be split
// over workgroups, whose sums combine_kernel joins.
//
// Rows behind a tile's last key and pages that do not exist are behind the end of the buffer that a load is given, and read as zeros: what a page holds
// behind a row's last token is never read.
//
// What bounds them (32 query and 8 KV heads of 128).  rows_kernel: memory, 256 rows of up to 4096 bf16 tokens in 378 us (5.7 TB/s of keys and values), one
// row over 32768 e4m3 tokens in 20.0 (traced apart 16.2 us for the reading, 4.2 TB/s, and 4.5 for joining 64 parts).  tile_kernel: two prompts of 8192 tokens
// in 1.00 to 1.06 ms (1040 to 1100 TFLOP/s), the clock at 1.6 to 1.7 GHz by the card's power limit, the matrix units busy 58 % of the cycles (47 % with two
// workgroups a compute unit) and the vector units, exponentials above all, 53 %.  The next tile's scores beside this tile's exponentials within a wave: 6 %
// fewer cycles, at a lower clock, and no less time.
#include "attention_tile.h"
#include "common.h"
#include "kernels.h"
#include "paged_cache.h"

namespace dl {

constexpr float kNoKey = -1e30f;       // a maximum before the first key: finite, so that exp2(-inf - m) is 0 and not NaN
constexpr int kSubKeys = 64;             // keys whose scores a wave has at a time

struct AttendArgs {
  PagedCache cache;
  const bf16_t* q;                     // [batch][seq][Hq][DH]
  const int64_t *start, *lengths;
  bf16_t* o;
  float* lse;                          // [batch][Hq][seq] or null
  float *sums, *stats;                 // parts of a split: [pair][tile][split][rows][DH], and maximum and sum of a row [..][rows][2]
  int seq, Hq, group, tiles, splits, least;   // least: tiles of keys in a part
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

// Positions of a batch row that its new tokens see, all of them together: 0 .. result - 1.
__device__ __forceinline__ int row_keys(const AttendArgs& a, int b) {
  const int n = row_length(a.lengths, b, a.seq);
  const int64_t end = row_start(a.start, b) + n, cap = (int64_t)a.cache.columns << a.cache.shift;
  return n <= 0 || end <= 0 ? 0 : (int)(end < cap ? end : cap);
}

// Of up to 64 batch rows, which lie one a lane: the one with the rank-th most keys.
__device__ __forceinline__ int row_of_rank(const AttendArgs& a, int rank, int lane) {
  const int batch = a.cache.batch, n = lane < batch ? row_keys(a, lane) : -1;
  int above = 0;
  for (int j = 0; j < batch; ++j) {
    const int other = __builtin_amdgcn_readlane(n, j);
    above += other > n || (other == n && j < lane);
  }
  return __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < batch && above == rank));
}

// Workgroup -> (batch row, KV head, place in their queue of workgroups).  Ids go to the eight XCDs in turn, each with an L2 of its own: where the heads are a
// multiple of 8 a head's workgroups, which share its keys, stay on one XCD, and every XCD has as much of each batch row.  A queue's places are dealt to the
// heads in turn, long ones first.  SORTED: the rows with most keys come first, since the last workgroups to start should be short ones (5 rows of 0 to 1037
// tokens behind 1600 to 8000, 8 heads: 381 us, 472 in the order of the rows); worth its microsecond where workgroups are long and of different length.
struct Work { int b, hk, j; };
template <bool SORTED>
__device__ __forceinline__ Work work_of(const AttendArgs& a, int id, int queue, int lane) {
  const PagedCache& c = a.cache;
  const bool pinned = (c.heads & 7) == 0;
  const int heads = pinned ? c.heads >> 3 : c.heads, slot = pinned ? id >> 3 : id;       // heads that take turns
  const int rank = slot / (queue * heads), left = slot % (queue * heads);
  const int hk = pinned ? (left % heads) * 8 + (id & 7) : left % heads;
  return {SORTED && c.batch > 1 && c.batch <= 64 ? __builtin_amdgcn_readfirstlane(row_of_rank(a, rank, lane)) : rank, hk, left / heads};
}

// Memory to LDS without registers between, 16 bytes a lane: lane l's go to `to` + 16 l.  As assembly, which names no register as an output: behind the builtin the
// compiler waits for all such loads in front of every transposing read, of which it does not know that it stays clear of the stage being
// filled.  The kernels wait for them themselves (wait_loads), so nothing counts on the compiler here.  Nor does it count the distance that a buffer load keeps
// from a vector instruction that wrote its descriptor, as one does that brings a spilled scalar register back: five wait states, of which writing m0 is one.
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 descriptor(const void* p, uint32_t bytes) {
  const uint64_t at = (uint64_t)(uintptr_t)p;
  return i32x4{(int)(uint32_t)at, (int)((uint32_t)(at >> 32) & 0xffffu), (int)bytes, 0x00020000};
}
__device__ __forceinline__ void load_to_lds(const i32x4& from, uint32_t to, int offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(from)
               : "memory", "m0");
}
// Until LEFT of them are under way.  The builtin tells the compiler that its own loads are done too (it does not read assembly, and would wait for them, and so for
// the loads to LDS, at their next use).
template <int LEFT>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
  if constexpr (LEFT == 0) __builtin_amdgcn_s_waitcnt(0x0f70);
}
// Until no load and no read of LDS of this wave is: in front of loads to a place that the wave has read from, where no barrier lies between.  Its reads may have
// been issued without having been served (what uses them can be moved behind).
__device__ __forceinline__ void wait_loads_and_reads() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(LDS_PTR(const char))p; }

// Whether x holds for a thread of the workgroup; word: of LDS.
__device__ __forceinline__ bool any_of_workgroup(bool x, int* word) {
  if (threadIdx.x == 0) *word = 0;
  __syncthreads();
  if (x) *word = 1;
  __syncthreads();
  const bool any = *word != 0;
  __syncthreads();
  return any;
}

// The keys of one wave's 16 rows of a tile: first vector in the cache, and how many of the 16 there are.
struct Keys16 { int64_t vec; int n; };
__device__ __forceinline__ Keys16 keys16(const PagedCache& c, int b, int hk, int p, int end) {
  const int page = p < end ? page_of_wave(c, b, p) : -1;
  if (page < 0) return {0, 0};
  const int n = end - p;
  return {vector_of(c, page, hk, p), n < 16 ? n : 16};
}

// LDS addresses of a lane's operands in a tile of RowTile's layout.  Its swizzle is an XOR of chunk numbers, so that the steps along head_dim are XORs of one
// address and steps of 16 rows an offset: key(kk, i) of keys 32 i + lane % 32, step kk; value(t2, ks) of columns 32 t2 .., keys 16 ks .., as frag_cols.
template <int DH, int NW>
struct Operands {
  using Tile = RowTile<16 * NW, DH, NW>;
  uint32_t k, v;
  __device__ __forceinline__ Operands(uint32_t tiles, int lane) {
    const int row = lane & 31, grp = lane >> 4, s = lane & 15, vrow = ((grp >> 1) << 2) + (s >> 2), col = ((grp & 1) << 4) + ((s & 3) << 2);
    k = tiles + row * Tile::ROW_B + (((lane >> 5) ^ Tile::swz(row)) << 4);
    v = tiles + vrow * Tile::ROW_B + ((((col >> 3) ^ Tile::swz(vrow)) << 4) | ((col & 7) << 1));
  }
  __device__ __forceinline__ bf16x8 key(int kk, int i) const {
    return *(LDS_PTR(const bf16x8))(uintptr_t)((k ^ (kk << 5)) + i * (32 * Tile::ROW_B));
  }
  __device__ __forceinline__ bf16x8 value(int t2, int ks) const {
    const uint32_t lo = v ^ (t2 << 6), hi = v ^ (t2 << 6) ^ 32;       // swz(row + 8) = swz(row) ^ 2
    bf16x8 x;
    x.lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(lo + ks * 16 * Tile::ROW_B));
    x.hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(hi + (ks * 16 + 8) * Tile::ROW_B));
    return x;
  }
};

// Values that are not finite out of v, with a 1 for each in count.
__device__ __forceinline__ void split_not_finite(bf16x8& v, bf16x8& count) {
  u32x4 u = __builtin_bit_cast(u32x4, v), n;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t odd = ((u[i] & 0x7f80u) == 0x7f80u ? 0xffffu : 0) | ((u[i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0);
    n[i] = odd & 0x3f803f80u;          // 1.0
    u[i] &= ~odd;
  }
  v = __builtin_bit_cast(bf16x8, u);
  count = __builtin_bit_cast(bf16x8, n);
}

// Whether one of 8 bf16 is infinite or NaN.
__device__ __forceinline__ bool any_not_finite(const bf16x8& v) {
  const u32x4 u = __builtin_bit_cast(u32x4, v);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= (u[i] & 0x7f80u) == 0x7f80u || (u[i] & 0x7f800000u) == 0x7f800000u;
  return odd;
}

// Whether the tiles of values share one place in LDS, so that three workgroups fit a compute unit (48 KB each at heads of 128): of bf16 with four waves.
// Values are then asked for when the last tile's are done with, and waited for behind the exponentials (two prompts of 8192 tokens, 32 and 8 heads of 128, in
// one run: 1060 us with two workgroups, 993 with three: products of some beside exponentials of others is what counts).  Over e4m3 this takes 15 % longer than
// eight waves do: bf16 is made of e4m3 between scores and products then, and for half as many rows.
template <bool E4M3, int NW>
constexpr bool kThin = !E4M3 && NW == 4;
template <int DH, bool E4M3, int NW>
constexpr int tile_lds() { return (kThin<E4M3, NW> ? 3 : 4) * 16 * NW * DH * 2; }

template <int DH, bool E4M3, int NW>
__global__ __launch_bounds__(64 * NW, (kThin<E4M3, NW>) ? 3 : 2) void tile_kernel(const AttendArgs a) {
  constexpr int kTileRows = 32 * NW, kTileKeys = 16 * NW;
  using Tile = RowTile<kTileKeys, DH, NW>;
  constexpr bool THIN = kThin<E4M3, NW>;
  // where keys and values of a stage lie; THIN: one place for values
  constexpr int K_STAGE = THIN ? Tile::BYTES : 2 * Tile::BYTES, V_FIRST = THIN ? 2 * Tile::BYTES : Tile::BYTES, V_STAGE = THIN ? 0 : K_STAGE;
  constexpr int TILES = tile_lds<DH, E4M3, NW>();
  const auto place = [](int w, int stage) { return w ? V_FIRST + stage * V_STAGE : stage * K_STAGE; };
  // e4m3: a wave's 16 keys as they are held; CHUNK bytes a lane and load, LANES of them a key
  constexpr int HELD = 16 * DH, CHUNK = HELD < 1024 ? 8 : 16, NLOAD = HELD / (64 * CHUNK), LANES = DH / CHUNK, ROWS = 64 / LANES;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const PagedCache& c = a.cache;
  const Work work = work_of<true>(a, (int)blockIdx.x, a.tiles * a.splits, lane);
  const int b = work.b, hk = work.hk, pair = b * c.heads + hk;
  const int tile = a.tiles - 1 - work.j / a.splits, split = work.j % a.splits;     // late tokens first
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
  const int first_lim = n_rows > 0 ? __builtin_amdgcn_readfirstlane(last_key(min(row0, n_rows - 1))) : -1;     // the first row's
  int* first_odd = reinterpret_cast<int*>(smem + TILES);       // the first key with a value that is not finite, of each column; whether there is any
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
    for (int i = (t0 * kTileKeys >> c.shift) + threadIdx.x, n = (min(end, t1 * kTileKeys) - 1) >> c.shift; i <= n; i += 64 * NW)
      missing |= (uint32_t)c.table[(int64_t)b * c.columns + i] >= (uint32_t)c.n_pages;
    if (threadIdx.x <= DH) first_odd[threadIdx.x] = threadIdx.x < DH ? 0x7fffffff : 0;
    missing = any_of_workgroup(missing, reinterpret_cast<int*>(smem));

    bf16x8 qf[DH / 16];
    {
      const RowPlace at = row_place(a, hk, min(r, n_rows - 1));
      const bf16_t* qp = a.q + (((int64_t)b * a.seq + at.t) * a.Hq + at.h) * DH + half * 8;
#pragma unroll
      for (int kk = 0; kk < DH / 16; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qp + kk * 16);
    }

    // e4m3: of the wave's 16 keys of the next tile in lanes 0 .. 15, of its values in the next 16; and how many of the keys there are
    uint32_t scales = 0;
    int there = 0;
    const auto load = [&](int t, int stage, int first, int last) {             // keys (0), values (1), or both
      const Keys16 k16 = keys16(c, b, hk, t * kTileKeys + wave * 16, end);
#pragma unroll
      for (int w = first; w <= last; ++w) {
        const uint32_t to = lds_address(smem) + place(w, stage) + wave * (16 * Tile::ROW_B);
        if constexpr (!E4M3) {
          const i32x4 from = descriptor(c.x[w] + k16.vec * (DH * 2), (uint32_t)(k16.n * DH * 2));
#pragma unroll
          for (int i = 0; i < Tile::PER_WAVE; ++i) {
            const int row = i * Tile::RPI + lane / Tile::LPR, ch = (lane % Tile::LPR) ^ Tile::swz(row);
            load_to_lds(from, to + i * 1024, row * (DH * 2) + (ch << 4));
          }
        } else {
          const i32x4 from = descriptor(c.x[w] + k16.vec * DH, (uint32_t)(k16.n * DH));
#pragma unroll
          for (int i = 0; i < (HELD + 1023) / 1024; ++i)
            if (HELD >= 1024 || lane < HELD / 16) load_to_lds(from, to + i * 1024, i * 1024 + lane * 16);
        }
      }
      if constexpr (E4M3) {
        scales = ((lane & 16 ? c.scale[1] : c.scale[0]) + k16.vec)[lane & 15];
        there = k16.n;
      }
    };
    // what a wave has loaded, made ready for all: e4m3 in its place as bf16; and, of a tile that some row sees in part, values that are not finite taken
    // out, since a weight of 0 times one of them is NaN: the first key that has one in a column is remembered, and the rows that see it get NaN at the end
    const auto arrived = [&](int t, int stage) {
      if constexpr (E4M3) {
        scales = (lane & 15) < there ? scales << 23 : 0;        // keys that are not there are zeros times whatever was read
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          char* own = smem + place(w, stage) + wave * (16 * Tile::ROW_B);
          u32x2 raw[NLOAD][CHUNK / 8];
#pragma unroll
          for (int i = 0; i < NLOAD; ++i)
#pragma unroll
            for (int h = 0; h < CHUNK / 8; ++h) raw[i][h] = *reinterpret_cast<const u32x2*>(own + (i * 64 + lane) * CHUNK + h * 8);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // all of it is read before any of it is written over
#pragma unroll
          for (int i = 0; i < NLOAD; ++i) {
            const int key = i * ROWS + lane / LANES, ch = (lane % LANES) * (CHUNK / 8);
            const float scale = __uint_as_float((uint32_t)__shfl((int)scales, w * 16 + key, 64));
#pragma unroll
            for (int h = 0; h < CHUNK / 8; ++h)
              *reinterpret_cast<bf16x8*>(own + key * Tile::ROW_B + (((ch + h) ^ Tile::swz(key)) << 4)) = unpack_e4m3(raw[i][h], scale);
          }
        }
      }
      if (t * kTileKeys + kTileKeys - 1 > first_lim) {
        char* own = smem + place(1, stage) + wave * (16 * Tile::ROW_B);
#pragma unroll 1
        for (int i = 0; i < Tile::PER_WAVE; ++i) {
          bf16x8* at = reinterpret_cast<bf16x8*>(own + i * 1024 + lane * 16);
          bf16x8 v = *at;
          if (!any_not_finite(v)) continue;
          const int key = i * Tile::RPI + lane / Tile::LPR, ch = (lane % Tile::LPR) ^ Tile::swz(key);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!(fabsf((float)v[e]) < INFINITY)) {
              atomicMin(&first_odd[ch * 8 + e], t * kTileKeys + wave * 16 + key);
              v[e] = (bf16_t)0.f;
            }
          *at = v;
          first_odd[DH] = 1;
        }
      }
    };

    const Operands<DH, NW> operands(lds_address(smem), lane);
    load(t0, 0, 0, THIN ? 0 : 1);
    wait_loads<0>();
    if (!THIN) arrived(t0, 0);
    __syncthreads();
    int stage = 0;
    for (int t = t0; t < t1; ++t) {
      const bool more = t + 1 < t1;
      if (THIN) load(t, stage, 1, 1);
      if (more) load(t + 1, stage ^ 1, 0, THIN ? 0 : 1);
#pragma unroll
      for (int sub = 0; sub < kTileKeys / kSubKeys; ++sub) {
        const int kv0 = t * kTileKeys + sub * kSubKeys;
        f32x16 s[2];
        Operands<DH, NW> at = operands;
        at.k += place(0, stage) + sub * (kSubKeys * Tile::ROW_B);
        at.v += place(1, stage) + sub * (kSubKeys * Tile::ROW_B);
        asm volatile("" : "+v"(at.k), "+v"(at.v));                 // their XORs are formed here, and take no registers across the loop
        if (kv0 <= lim1) {
          // the wave that has products to issue goes first, so that the other ones' exponentials fall beside them and not beside their own products
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[i][e] = 0.f;
#pragma unroll
          for (int kk = 0; kk < DH / 16; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.key(kk, i), qf[kk], s[i], 0, 0, 0);
          __builtin_amdgcn_s_setprio(0);
          // keys after the row's own position (only on tiles that reach past this wave's first row)
          if (kv0 + kSubKeys - 1 > lim0) mask_rows_above<2>(s, lim - kv0 - (half << 2), -INFINITY);
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
        }
        if constexpr (THIN) {
          // the values, asked for before the next keys: all waves have theirs
          if (more) wait_loads<Tile::PER_WAVE>(); else wait_loads<0>();
          arrived(t, 0);
          __syncthreads();
        }
        if (kv0 <= lim1) {
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            // a weight is rounded to bf16, as in the layer's own attention: results are off by 2.1e-3 to 2.4e-3 of their norm where their own rounding
            // makes it 1.65e-3.  The sum of two bf16, which rows_kernel takes, brings that back and costs half of the matrix work again: two prompts of 8192 tokens
            // 1041 -> 1480 us (e4m3 1088 -> 1480), 512 behind 8000 87 -> 118
            const bf16x8 pf = pack_slots(s[ks >> 1], (ks & 1) * 8);
#pragma unroll
            for (int t2 = 0; t2 < DH / 32; ++t2) oacc[t2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.value(t2, ks), pf, oacc[t2], 0, 0, 0);
          }
          __builtin_amdgcn_s_setprio(0);
        }
      }
      wait_loads<0>();
      if (!THIN && more) arrived(t + 1, stage ^ 1);
      __syncthreads();
      stage ^= 1;
    }
    if (first_odd[DH]) {
#pragma unroll
      for (int t2 = 0; t2 < DH / 32; ++t2)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (first_odd[t2 * 32 + ((e >> 2) << 3) + (half << 2) + (e & 3)] <= lim) oacc[t2][e] = NAN;
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

// max (sum) over the four lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them
__device__ __forceinline__ float max_across_quarters(float x) {
  x = max_across_halves(x);
  return fmaxf(x, __shfl_xor(x, 16, 64));
}
__device__ __forceinline__ float sum_across_quarters(float x) {
  x = sum_across_halves(x);
  return x + __shfl_xor(x, 16, 64);
}

// A wave's tile of 32 keys, or values, in LDS as the cache holds it: rows of ROW_B bytes, 16-byte chunk c of row r at chunk c ^ swz(r).  Free of bank
// conflicts (the LDS serves 256 B of banks a clock) for both of its reads:
//   row reads: 16 lanes, 16 consecutive rows, one chunk;
//   transposing reads: 32 lanes, which take 32 B (bf16) of rows 0 .. 7 or 8 .. 15 of 16, or 16 B (e4m3) of rows 0 .. 7 and 16 .. 23, or 8 .. 15 and 24 .. 31.
template <int DH, bool E4M3>
struct HeldTile {
  static constexpr int ROW_B = DH * (E4M3 ? 1 : 2), CHUNKS = ROW_B / 16, BYTES = 32 * ROW_B;
  static constexpr int WIDTH = ROW_B == 32 ? 4 : 16;                 // bytes a lane loads: a load's rows lie in one group of 16
  static constexpr int RPI = 64 * WIDTH / ROW_B, LOADS = 32 / RPI;   // rows of a load, loads
  static __device__ __forceinline__ int swz(int r) {
    constexpr int SHARE = 16 / CHUNKS;                               // rows that 256 B hold
    const int j = (r / SHARE) & (CHUNKS - 1);
    if constexpr (E4M3) return j ^ (((r >> 4) & 1) * (CHUNKS / 2));
    else return ((j << 1) | (j >> (CHUNKS == 16 ? 3 : CHUNKS == 8 ? 2 : 1))) & (CHUNKS - 1);
  }
  // loads a group of 16 rows, of which the first vector starts at p and n are there (the others are zeros)
  static __device__ __forceinline__ void load(const char* p, int n, uint32_t to, int group, int lane) {
    const i32x4 from = descriptor(p, (uint32_t)(n * ROW_B));
#pragma unroll
    for (int i = 0; i < LOADS / 2; ++i) {
      const int at = lane * WIDTH, row = i * RPI + at / ROW_B, ch = (at % ROW_B) / 16 ^ swz(group * 16 + row);
      const int offset = row * ROW_B + ch * 16 + at % 16;
      const uint32_t dst = to + (group * (LOADS / 2) + i) * (64 * WIDTH);
      if constexpr (WIDTH == 16) load_to_lds(from, dst, offset);
      else asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(dst)), "v"(offset), "s"(from)
                        : "memory", "m0");
    }
  }
};

// Few rows (NR groups of 16), many keys: bound by the reading of the cache.  Each of the workgroup's four waves takes every fourth tile of 32 keys, which it
// loads to LDS for itself, a tile ahead, so that the waves wait for nothing but their own loads; the four results are joined in LDS at the end.
//   S[key][row] = K Q^T and O[d][row] += V^T P^T on v_mfma_f32_16x16x32_bf16: lane l has row l % 16 of its group, keys 4 (l / 16) .. + 3 of each
//   half of the tile, and those are the slots that it gives the second product, whose other operand (transposing reads) is taken in that order.
// e4m3 is read as it is held; scores and weights take the powers of two of their keys and values, exactly.
template <int DH, bool E4M3, int NR>
__global__ __launch_bounds__(256, NR == 1 ? 2 : 1) void rows_kernel(const AttendArgs a) {
  using Tile = HeldTile<DH, E4M3>;
  constexpr int STAGE = 2 * Tile::BYTES + (E4M3 ? 64 : 0), ROWS = 16 * NR;      // keys, values, and their 32 + 32 powers of two
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const PagedCache& c = a.cache;
  const Work work = work_of<false>(a, (int)blockIdx.x, a.tiles * a.splits, lane);
  const int b = work.b, hk = work.hk, pair = b * c.heads + hk, tile = a.tiles - 1 - work.j / a.splits, split = work.j % a.splits;
  const int lr = lane & 15, quarter = lane >> 4;
  const int n_rows = row_length(a.lengths, b, a.seq) * a.group, row0 = tile * ROWS;
  const int64_t start = row_start(a.start, b), cap = (int64_t)c.columns << c.shift;
  const auto last_key = [&](int row) { const int64_t p = start + row / a.group; return (int)(p < -1 ? -1 : p >= cap ? cap - 1 : p); };
  const int end = row0 < n_rows ? last_key(min(row0 + ROWS, n_rows) - 1) + 1 : 0;
  const int lim0 = n_rows > 0 ? __builtin_amdgcn_readfirstlane(last_key(min(row0, n_rows - 1))) : -1;
  const int all = (end + 31) / 32, per = max((all + a.splits - 1) / a.splits, a.least);
  const int u0 = split * per, u1 = min(all, u0 + per);

  f32x4 acc[NR][DH / 16];
  float m[NR], lsum[NR];
  int lim[NR];
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    m[n] = kNoKey;
    lsum[n] = 0.f;
    lim[n] = n_rows > 0 ? last_key(min(row0 + n * 16 + lr, n_rows - 1)) : -1;
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) acc[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (u0 < u1) {
    const uint32_t own = lds_address(smem) + wave * (2 * STAGE);
    const auto load = [&](int u, int stage) {
      const Keys16 k16[2] = {keys16(c, b, hk, u * 32, end), keys16(c, b, hk, u * 32 + 16, end)};
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int w = 0; w < 2; ++w) Tile::load(c.x[w] + k16[g].vec * Tile::ROW_B, k16[g].n, own + stage * STAGE + w * Tile::BYTES, g, lane);
      if constexpr (E4M3) {
        // four lanes for each of (keys, values) x (first 16, last 16), from addresses of their own; where there are no keys, of others that take no part
        const uint8_t* from = (lane & 8 ? c.scale[1] : c.scale[0]) + (lane & 4 ? k16[1].vec : k16[0].vec) + (lane & 3) * 4;
        const uint32_t to = __builtin_amdgcn_readfirstlane(own + stage * STAGE + 2 * Tile::BYTES);
        if (lane < 16)
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory", "m0");
      }
    };
    // the first tile is on its way before anything else is looked at
    int u = u0 + wave, stage = 0;
    if (u < u1) load(u, 0);

    bf16x8 qf[NR][DH / 32];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const RowPlace at = row_place(a, hk, min(row0 + n * 16 + lr, n_rows - 1));
      const bf16_t* qp = a.q + (((int64_t)b * a.seq + at.t) * a.Hq + at.h) * DH;
      // e4m3: a 16-byte read of a key holds the slots of two steps
#pragma unroll
      for (int kk = 0; kk < DH / 32; ++kk)
        qf[n][kk] = *reinterpret_cast<const bf16x8*>(qp + (E4M3 && DH >= 64 ? (kk >> 1) * 64 + quarter * 16 + (kk & 1) * 8 : kk * 32 + quarter * 8));
    }

    // pages that do not exist: every wave looks for itself, without waiting for others
    bool missing = false;
    for (int i = (u0 * 32 >> c.shift) + lane, n = (min(end, u1 * 32) - 1) >> c.shift; i <= n; i += 64)
      missing |= (uint32_t)c.table[(int64_t)b * c.columns + i] >= (uint32_t)c.n_pages;
    missing = __builtin_amdgcn_ballot_w64(missing) != 0;

    // a byte of 255 is no power of two, and may stand where there is no key: finite, so that a weight of 0 times it is 0
    const auto scale_of = [](uint32_t four, int e) { return __uint_as_float(min((four >> (8 * e)) & 0xffu, 254u) << 23); };

    for (; u < u1; u += 4) {
      wait_loads_and_reads();
      if (u + 4 < u1) load(u + 4, stage ^ 1);
      const uint32_t tk = own + stage * STAGE, tv = tk + Tile::BYTES;
      const int kv0 = u * 32;
      uint32_t ks[2] = {}, vs[2] = {};           // of four keys of each half
      if constexpr (E4M3)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          ks[g] = *(LDS_PTR(const uint32_t))(uintptr_t)(tv + Tile::BYTES + g * 16 + quarter * 4);
          vs[g] = *(LDS_PTR(const uint32_t))(uintptr_t)(tv + Tile::BYTES + 32 + g * 16 + quarter * 4);
        }
      f32x4 s[NR][2];
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int g = 0; g < 2; ++g) s[n][g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int row = g * 16 + lr;
        if constexpr (E4M3 && DH >= 64) {
#pragma unroll
          for (int k2 = 0; k2 < DH / 64; ++k2) {
            const u32x4 raw = *(LDS_PTR(const u32x4))(uintptr_t)(tk + row * Tile::ROW_B + (((k2 * 4 + quarter) ^ Tile::swz(row)) << 4));
            const bf16x8 k0 = unpack_e4m3(u32x2{raw[0], raw[1]}, 1.f), k1 = unpack_e4m3(u32x2{raw[2], raw[3]}, 1.f);
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              s[n][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[n][2 * k2], s[n][g], 0, 0, 0);
              s[n][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[n][2 * k2 + 1], s[n][g], 0, 0, 0);
            }
          }
        } else {
#pragma unroll
          for (int kk = 0; kk < DH / 32; ++kk) {
            bf16x8 kf;
            if constexpr (E4M3)
              kf = unpack_e4m3(*(LDS_PTR(const u32x2))(uintptr_t)(tk + row * Tile::ROW_B + (((quarter >> 1) ^ Tile::swz(row)) << 4) + (quarter & 1) * 8), 1.f);
            else kf = *(LDS_PTR(const bf16x8))(uintptr_t)(tk + row * Tile::ROW_B + (((kk * 4 + quarter) ^ Tile::swz(row)) << 4));
#pragma unroll
            for (int n = 0; n < NR; ++n) s[n][g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[n][kk], s[n][g], 0, 0, 0);
          }
        }
      }
      if constexpr (E4M3)
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float k = scale_of(ks[g], e);
#pragma unroll
            for (int n = 0; n < NR; ++n) s[n][g][e] *= k;
          }
      const bool masked = kv0 + 31 > lim0;
      if (masked) {
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][g][e] = kv0 + g * 16 + quarter * 4 + e > lim[n] ? -INFINITY : s[n][g][e];
      }
      if (missing) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
          if (page_of_wave(c, b, kv0 + g * 16) < 0)
#pragma unroll
            for (int n = 0; n < NR; ++n) s[n][g] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      }
      // a weight is the sum of two bf16: rounded to one it would add as much to the error as the rounding of the result does (2.3e-3 of a result, 1.7e-3 with
      // two), and the matrix unit has little to do here (one row over 32768 e4m3 tokens 20.3 us with one, 20.7 with two)
      bf16x8 pf[NR][2];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float mx = fmaxf(fmaxf(fmaxf(s[n][0][0], s[n][0][1]), fmaxf(s[n][0][2], s[n][0][3])),
                         fmaxf(fmaxf(s[n][1][0], s[n][1][1]), fmaxf(s[n][1][2], s[n][1][3]))) * a.scale_log2;
        // the reference is raised only where some row's maximum grew by more than 2^8; until then the lanes of a row need not know each other's
        if (__builtin_amdgcn_ballot_w64(mx > m[n] + 8.0f) != 0) {
          const float m_new = fmaxf(m[n], max_across_quarters(mx)), alpha = fast_exp2(m[n] - m_new);
          lsum[n] *= alpha;
          m[n] = m_new;
#pragma unroll
          for (int t = 0; t < DH / 16; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][t][e] *= alpha;
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = fast_exp2(__builtin_fmaf(s[n][g][e], a.scale_log2, -m[n]));
            lsum[n] += p;
            const float w = E4M3 ? p * scale_of(vs[g], e) : p;
            pf[n][0][g * 4 + e] = (bf16_t)w;
            pf[n][1][g * 4 + e] = (bf16_t)(w - (float)pf[n][0][g * 4 + e]);
          }
      }
      const auto value = [&](int t) {
        if constexpr (E4M3) {
          const int row = (lr >> 1) < 4 ? quarter * 4 + (lr >> 1) : 16 + quarter * 4 + (lr >> 1) - 4;
          const uintptr_t from = tv + row * Tile::ROW_B + ((t ^ Tile::swz(row)) << 4) + (lr & 1) * 8;
          return unpack_e4m3(__builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_PTR(i32x2))from)), 1.f);
        } else {
          const int row = quarter * 4 + (lr >> 2), ch = t * 2 + ((lr & 3) >> 1), in = (lr & 1) * 8;
          bf16x8 x;
          x.lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(tv + row * Tile::ROW_B + ((ch ^ Tile::swz(row)) << 4) + in));
          x.hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LDS_PTR(bf16x4))(uintptr_t)(tv + (row + 16) * Tile::ROW_B + ((ch ^ Tile::swz(row + 16)) << 4) + in));
          return x;
        }
      };
      if (!masked || a.seq == 1) {
#pragma unroll
        for (int t = 0; t < DH / 16; ++t) {
          const bf16x8 vf = value(t);
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n][i], acc[n][t], 0, 0, 0);
        }
      } else {
        // a weight of 0 times a value that is not finite is NaN: of a tile that some row does not see whole, such values are counted apart, for the rows that
        // see them
#pragma unroll
        for (int t = 0; t < DH / 16; ++t) {
          bf16x8 vf = value(t), count;
          const bool odd = __builtin_amdgcn_ballot_w64(any_not_finite(vf)) != 0;
          if (odd) split_not_finite(vf, count);
#pragma unroll
          for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n][i], acc[n][t], 0, 0, 0);
            if (odd) {
              bf16x8 seen;
#pragma unroll
              for (int e = 0; e < 8; ++e) seen[e] = (bf16_t)(kv0 + (e >> 2) * 16 + quarter * 4 + (e & 3) <= lim[n] ? 1.f : 0.f);
              const f32x4 k = __builtin_amdgcn_mfma_f32_16x16x32_bf16(count, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[n][t][e] = k[e] > 0.f ? NAN : acc[n][t][e];
            }
          }
        }
      }
      stage ^= 1;
    }
  }

  // the four waves' results: every wave's maximum and sum, and its rows relative to the largest maximum, added up by all threads
  float* stats = reinterpret_cast<float*>(smem);                       // [wave][ROWS][2]
  float* rows = stats + 4 * ROWS * 2;                                  // [wave][ROWS][DH + 4]
  __syncthreads();
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    lsum[n] = sum_across_quarters(lsum[n]);
    if (quarter == 0) {
      stats[(wave * ROWS + n * 16 + lr) * 2] = m[n];
      stats[(wave * ROWS + n * 16 + lr) * 2 + 1] = lsum[n];
    }
#pragma unroll
    for (int t = 0; t < DH / 16; ++t) *reinterpret_cast<f32x4*>(rows + (wave * ROWS + n * 16 + lr) * (DH + 4) + t * 16 + quarter * 4) = acc[n][t];
  }
  __syncthreads();
  constexpr int LPR = DH / 4;
  for (int i = threadIdx.x; i < ROWS * LPR; i += 256) {
    const int row = i / LPR, d = (i % LPR) * 4, r = row0 + row;
    if (r >= a.seq * a.group) continue;
    float top = stats[row * 2];
#pragma unroll
    for (int w = 1; w < 4; ++w) top = fmaxf(top, stats[(w * ROWS + row) * 2]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float l = stats[(w * ROWS + row) * 2 + 1], f = l == 0.f ? 0.f : fast_exp2(stats[(w * ROWS + row) * 2] - top);
      sum += f * l;
      const f32x4 x = *reinterpret_cast<const f32x4*>(rows + (w * ROWS + row) * (DH + 4) + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += f * x[e];
    }
    if (a.splits > 1) {
      const int64_t at = (((int64_t)pair * a.tiles + tile) * a.splits + split) * ROWS + row;
      if (d == 0) {
        a.stats[at * 2] = top;
        a.stats[at * 2 + 1] = sum;
      }
      if (u0 < u1) *reinterpret_cast<f32x4*>(a.sums + at * DH + d) = o;
      continue;
    }
    const bool any = r < n_rows && sum != 0.f;
    const float inv = any ? 1.0f / sum : 0.f;
    const RowPlace at = row_place(a, hk, r);
    bf16x4 ov;
#pragma unroll
    for (int e = 0; e < 4; ++e) ov[e] = (bf16_t)(any ? o[e] * inv : 0.f);
    *reinterpret_cast<bf16x4*>(a.o + (((int64_t)b * a.seq + at.t) * a.Hq + at.h) * DH + d) = ov;
    if (a.lse && d == 0) a.lse[((int64_t)b * a.Hq + at.h) * a.seq + at.t] = any ? (top + log2f(sum)) * kLn2 : -INFINITY;
  }
}

// Joins the parts of split rows.  DH / 4 lanes hold a row; `side` such groups of lanes share a row's parts, four of which they have under way at a time, and
// are joined in LDS.
template <int DH>
__global__ __launch_bounds__(1024) void combine_kernel(const AttendArgs a, int rows, int rows_per_tile, int side) {
  constexpr int LPR = DH / 4;
  __shared__ float stats[1024 / LPR][2], scaled[1024 / LPR];
  __shared__ f32x4 sums[1024];
  const PagedCache& c = a.cache;
  const int group = threadIdx.x / LPR, lane = threadIdx.x % LPR, here = blockDim.x / LPR;
  const int i = blockIdx.x * (here / side) + group / side, within = min(i, rows - 1);      // (pair, row of the pair)
  const int per_pair = a.seq * a.group, d = lane * 4;
  const int pair = within / per_pair, r = within - pair * per_pair, b = pair / c.heads, hk = pair - b * c.heads;
  const int at0 = (pair * a.tiles + r / rows_per_tile) * a.splits * rows_per_tile + r % rows_per_tile;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float m = kNoKey, sum = 0.f;
  for (int s0 = group % side; s0 < a.splits; s0 += 4 * side) {
    float ms[4], ls[4], top = m;
    f32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = at0 + min(s0 + k * side, a.splits - 1) * rows_per_tile;
      ms[k] = a.stats[at * 2];
      ls[k] = s0 + k * side < a.splits ? a.stats[at * 2 + 1] : 0.f;
      x[k] = *reinterpret_cast<const f32x4*>(a.sums + at * DH + d);        // of a part without keys: whatever is there, and not used
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) top = ls[k] == 0.f ? top : fmaxf(top, ms[k]);
    const float old = sum == 0.f ? 0.f : fast_exp2(m - top);
    sum *= old;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = old == 0.f ? 0.f : acc[e] * old;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (ls[k] == 0.f) continue;
      const float w = fast_exp2(ms[k] - top);
      sum += w * ls[k];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += w * x[k][e];
    }
    m = top;
  }
  // of padding, whose length is asked for beside the parts: nothing, whatever they hold
  if (r >= row_length(a.lengths, b, a.seq) * a.group) {
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (side > 1) {
    const int own = group - group % side;              // of the row's groups the first
    if (lane == 0) { stats[group][0] = m; stats[group][1] = sum; }
    __syncthreads();
    float top = kNoKey;
    for (int k = 0; k < side; ++k) top = stats[own + k][1] == 0.f ? top : fmaxf(top, stats[own + k][0]);
    const float w = sum == 0.f ? 0.f : fast_exp2(m - top);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = sum == 0.f ? 0.f : acc[e] * w;
    sums[threadIdx.x] = acc;
    if (lane == 0) scaled[group] = sum == 0.f ? 0.f : sum * w;
    __syncthreads();
    if (group != own) return;
    m = top;
    sum = scaled[own];
#pragma unroll 8
    for (int k = 1; k < side; ++k) {
      sum += scaled[own + k];
      const f32x4 x = sums[threadIdx.x + k * LPR];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += x[e];
    }
  }
  if (i >= rows) return;
  const RowPlace at = row_place(a, hk, r);
  const float inv = sum != 0.f ? 1.0f / sum : 0.f;
  bf16x4 ov;
#pragma unroll
  for (int e = 0; e < 4; ++e) ov[e] = (bf16_t)(acc[e] * inv);
  *reinterpret_cast<bf16x4*>(a.o + (((int64_t)b * a.seq + at.t) * a.Hq + at.h) * DH + d) = ov;
  if (a.lse && d == 0) a.lse[((int64_t)b * a.Hq + at.h) * a.seq + at.t] = sum != 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
}

// Which way a call goes: rows of a workgroup (16 or 32: rows_kernel; 128 or 256: tile_kernel), tiles of a pair's rows, and parts of a tile's keys.  Up to 32
// rows the cache's bytes are what counts and rows_kernel is as fast as they come; tile_kernel's matrix products of 32 rows a wave are for more.  Eight waves
// a workgroup make bf16 of e4m3 once for twice the rows (two prompts of 8192 tokens, heads of 128: 1088 us, 1211 with four waves; 5 rows of up to 1037 behind
// up to 8009 360 and 404; bf16 itself, whose four waves share the place of their values, 1053 and 1041), where that leaves every compute unit two workgroups to
// take.  As many parts as fill the chip once: of rows_kernel the workgroups whose tiles the LDS holds
// (more of them, shorter, take longer: 8 rows over 16000 bf16 tokens 139 us in 4096 workgroups, 99 in 512), of tile_kernel two a compute unit (three, which
// fit: 512 tokens behind 8000 85.6 -> 90.2 us, 8 rows of 128 behind up to 4000 77.0 -> 69.2), and no more than the table's tokens hold kKeysLeast; one only
// where they hold no more than two, which a second launch would cost more than it saves.  Of a row shorter than its table rows_kernel's parts are kKeysLeast long
// all the same, and the others have none; tile_kernel's are equal shares, however short: kKeysLeast for it too is slower (64 tokens behind 1000, a table of
// 131072: 22.9 -> 25.5 us, behind 40: 20.7 -> 22.2), since the longest part lasts longer and joining walks over all parts either way.
struct AttendPlan { int rows, tiles, splits, least; int64_t pairs; };
constexpr int64_t kUnits = 256, kKeysLeast = 256;
static int64_t most_splits(int64_t max_tokens) { return max_tokens <= 2 * kKeysLeast ? 1 : (max_tokens + kKeysLeast - 1) / kKeysLeast; }
static int rows_lds(int64_t dh, bool e4m3) { return 4 * 2 * (2 * 32 * (int)dh * (e4m3 ? 1 : 2) + (e4m3 ? 64 : 0)); }
static AttendPlan attend_plan(int64_t batch, int64_t seq, int64_t Hkv, int64_t group, int64_t dh, bool e4m3, int64_t max_tokens) {
  AttendPlan p;
  const int64_t rows = seq * group, fit = 160 * 1024 / rows_lds(dh, e4m3);
  p.pairs = batch * Hkv;
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : e4m3 && dh == 128 && p.pairs * ((rows + 255) / 256) >= 2 * kUnits ? 256 : 128;
  p.tiles = (int)((rows + p.rows - 1) / p.rows);
  const int64_t wanted = kUnits * (p.rows == 256 ? 1 : p.rows == 128 || fit > 2 ? 2 : fit) / (p.pairs * p.tiles), most = most_splits(max_tokens);
  p.splits = (int)(wanted < 1 ? 1 : wanted < most ? wanted : most);
  p.least = (int)(kKeysLeast / 32);
  return p;
}

// Sums and statistics of the parts, in rows: pairs * tiles * splits * rows of a workgroup is within two workgroups a compute unit wherever there is a split,
// and within pairs * (rows, filled up) * most_splits, neither of which falls as the call grows.
static int64_t rows_held(int64_t batch, int64_t seq, int64_t Hkv, int64_t group, int64_t dh, bool e4m3, int64_t max_tokens) {
  const AttendPlan p = attend_plan(batch, seq, Hkv, group, dh, e4m3, max_tokens);
  const int64_t rows = p.pairs * p.tiles, most = most_splits(max_tokens), bound = 2 * kUnits * p.rows;
  return rows < bound && rows * p.rows < bound && most < bound && rows * p.rows * most < bound ? rows * p.rows * most : bound;
}
size_t paged_attention_workspace(int64_t batch, int64_t seq, int64_t Hq, int64_t Hkv, int64_t dh, bool e4m3, int64_t max_tokens) {
  return (size_t)rows_held(batch, seq, Hkv, Hq / Hkv, dh, e4m3, max_tokens) * (dh + 2) * sizeof(float);
}

template <int DH, bool E4M3, int NR>
static int launch_rows(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  const int tiles = rows_lds(DH, E4M3), results = 4 * 16 * NR * (DH + 6) * (int)sizeof(float), lds = tiles > results ? tiles : results;
  static std::atomic<unsigned long long> done{0};
  if (int rc = reserve_lds(rows_kernel<DH, E4M3, NR>, lds, done, "paged_attention_forward")) return rc;
  hipLaunchKernelGGL((rows_kernel<DH, E4M3, NR>), dim3((unsigned)(p.pairs * p.tiles * p.splits)), dim3(256), lds, st, a);
  return check_launch("paged_attention_forward");
}
template <int DH, bool E4M3, int NW>
static int launch_tiles(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  constexpr int lds = tile_lds<DH, E4M3, NW>() + (DH + 4) * (int)sizeof(int);
  static std::atomic<unsigned long long> done{0};
  if (int rc = reserve_lds(tile_kernel<DH, E4M3, NW>, lds, done, "paged_attention_forward")) return rc;
  hipLaunchKernelGGL((tile_kernel<DH, E4M3, NW>), dim3((unsigned)(p.pairs * p.tiles * p.splits)), dim3(64 * NW), lds, st, a);
  return check_launch("paged_attention_forward");
}
template <int DH, bool E4M3>
static int launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  int rc;
  if (p.rows == 16) rc = launch_rows<DH, E4M3, 1>(a, p, st);
  else if (p.rows == 32) rc = launch_rows<DH, E4M3, 2>(a, p, st);
  else if (p.rows == 128) rc = launch_tiles<DH, E4M3, 4>(a, p, st);
  else if constexpr (DH == 128 && E4M3) rc = launch_tiles<DH, E4M3, 8>(a, p, st);
  else return fail(-1, "paged_attention_forward: no kernel for %d rows", p.rows);
  if (rc || p.splits == 1) return rc;
  // groups of lanes to a row: enough that each has no more than four parts, as far as a workgroup of 1024 threads goes
  constexpr int LPR = DH / 4;
  int side = 1;
  while (side < 1024 / LPR && side * 4 < p.splits) side *= 2;
  const int threads = side * LPR > 256 ? side * LPR : 256, per = threads / (side * LPR);
  const int64_t rows = p.pairs * a.seq * a.group;              // with parts, the sums of 512 workgroups of 128 rows at most: indices fit 32 bits
  hipLaunchKernelGGL((combine_kernel<DH>), dim3((unsigned)((rows + per - 1) / per)), dim3(threads), 0, st, a, (int)rows, p.rows, side);
  return check_launch("paged_attention_forward, joining parts");
}

int launch_paged_attention(const CacheCall& c, const void* q, int64_t seq, int64_t Hq, float scale, void* o, float* lse, void* workspace,
                           hipStream_t st) {
  const int64_t group = Hq / c.heads, max_tokens = c.columns * c.page_size;
  const AttendPlan p = attend_plan(c.batch, seq, c.heads, group, c.dh, c.e4m3, max_tokens);
  AttendArgs a{};
  a.cache = paged_cache(c);
  a.q = (const bf16_t*)q;
  a.start = c.start; a.lengths = c.lengths;
  a.o = (bf16_t*)o;
  a.lse = lse;
  a.sums = (float*)workspace;
  a.stats = a.sums + rows_held(c.batch, seq, c.heads, group, c.dh, c.e4m3, max_tokens) * c.dh;
  a.seq = (int)seq; a.Hq = (int)Hq; a.group = (int)group;
  a.tiles = p.tiles; a.splits = p.splits; a.least = p.least;
  a.scale_log2 = scale * kLog2e;
  if (c.e4m3) return c.dh == 128 ? launch_attend<128, true>(a, p, st) : c.dh == 64 ? launch_attend<64, true>(a, p, st) : launch_attend<32, true>(a, p, st);
  return c.dh == 128 ? launch_attend<128, false>(a, p, st) : c.dh == 64 ? launch_attend<64, false>(a, p, st) : launch_attend<32, false>(a, p, st);
}

}  // namespace dl
