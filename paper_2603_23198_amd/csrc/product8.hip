// Products of 8-bit codes with a power-of-two scale for each block of 128:
//   C[m][n] = sum_b 2^(sa[m][b] + sb[n][b]) sum_{k in block b} A[m][k] B[n][k]
// Rows of the result are the rows of an expert's run, or (the weights' gradients) the sum runs over the
// run's tokens. Codes become bf16 with their scale by one instruction for two of them, exactly for scales from
// 2^-117 on, and bf16 products are exact in the fp32 sums of the matrix cores. The 8-bit matrix instructions
// are not: they add the products of eight neighbouring k with 13 bits below the largest of them, by measurement
// (1.6e-5 of the result's magnitude for normal operands). They are up to 1.8 times as fast and serve bf16 results of
// many rows, and gradients, of a caller who asks for that (BF16_FAST).
#include "blocks8.h"
#include "direct.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

// Eight codes times 2^(byte - 127).
__device__ __forceinline__ bf16x8_t decode8(uint32_t lo, uint32_t hi, float by) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A buffer of so many bytes, of values that are the same in every lane.
__device__ __forceinline__ u32x4_t buffer_of(const void* base, int64_t bytes) {
  u32x4_t w = rsrc_words(base, bytes);
  w[2] = __builtin_amdgcn_readfirstlane(w[2]);
  return w;
}

typedef int i32x8_t __attribute__((ext_vector_type(8)));

// ---- tiles of 256 or 128 rows by 256 columns ---------------------------------------------
// Eight waves, 2 along the rows x 4 along the columns, 128 (64) x 64 results each. A step is one block of
// 128 k: both operands come straight from memory into LDS (one 128-byte line a row), into a ring of two
// stages (three where tiles are 128 rows high), the next ones in flight while one feeds the matrix cores.
// Chunk c (16 k) of row r lies at position c ^ swizzle(r), so that the 8 lanes of a fragment read's phase
// meet 8 different positions. Scales travel the same way, a word of four blocks per row.
// A workgroup stays on its CU and takes tile after tile; the next tile's first stage is on its way while
// the results of one are stored. 16384 x 4096 x 4096 over eight experts of uneven load, exact products: 491 us in bf16, 507
// in fp32 (1.11 PFLOP/s; a library product in bf16 of 8192^3 reaches 1.24 to 1.48), the gradients of their weights 464 and 495.
// On the 8-bit instruction 276 and 294 (1.99 PFLOP/s; the library's 2.66). Loads in whole tiles: 426 and 252.
constexpr int kTileN = 256, kTileThreads = 512, kTileWaves = 8, kStep = 128;
constexpr int kWordRing = 4;  // scale words: the one in use, and up to two ahead of it

template <int BMT> struct Geo {
  static constexpr int LA = BMT * kStep / 1024 / kTileWaves, LB = kTileN * kStep / 1024 / kTileWaves;
  static constexpr int A = BMT * kStep, STAGE = (BMT + kTileN) * kStep, NS = BMT == 256 ? 2 : 3;
  static constexpr int WORDS = (BMT + kTileN) * 4;           // bytes of a scale word of all rows
  static constexpr int TM = BMT / 2 / 16, TN = 4;            // 16 x 16 results of a wave
  static constexpr int SMEM = NS * STAGE + kWordRing * WORDS;
};

// Of the columns' rows (B) two neighbouring fragments hold eight neighbouring columns per lane in a bf16
// result (see column_of): their rows 0 .. 3 and 8 .. 11 are read together.
template <bool PAIRED> __device__ __forceinline__ int swizzle_b(int row) {
  return PAIRED ? (row & 3) | (row >> 1 & 4) : row & 7;
}
// Column, of a wave's 64, of row r of fragment j. The result has columns r = 4 g .. 4 g + 3 of a row in one
// lane, and stores 16 bytes: 4 fp32 or, of two fragments, 8 bf16, 64 bytes of a row by four lanes.
template <bool PAIRED> __device__ __forceinline__ int column_of(int j, int r) {
  return PAIRED ? (j >> 1) * 32 + (r >> 2) * 8 + (j & 1) * 4 + (r & 3) : j * 16 + r;
}

// What a workgroup needs of one tile.
struct Where {
  u32x4_t ra, rb, rs;          // buffers of the operands, and of this wave's scales
  uint32_t offs;               // of this lane's scale row
  int blocks, b0;              // steps, and the first block's place in its scale word
  int m, n;                    // rows and columns that are there
  char* C;
  int64_t ldc;
};

template <int BMT, bool PAIRED> struct Loader {
  typedef Geo<BMT> G;
  int lane, wave;
  uint32_t lds;
  uint32_t offa[G::LA], offb[G::LB];
  int stage_in = 0, word_in = 0;  // where the next stage and the next scale word go

  __device__ __forceinline__ explicit Loader(const uint8_t* smem) {
    lane = lane_id();
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lds = __builtin_amdgcn_readfirstlane(
        (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)smem);
  }
  // Load q of this wave fills rows (wave L + q) 8 .. + 7 of an operand's tile, a line of 128 bytes each.
  __device__ __forceinline__ void setup(const Where& w, uint32_t lda, uint32_t ldb) {
#pragma unroll
    for (int q = 0; q < G::LA; ++q) {
      const int row = (wave * G::LA + q) * 8 + (lane >> 3);
      offa[q] = row < w.m ? (uint32_t)row * lda + ((lane & 7) ^ (row & 7)) * 16 : kOOB;
    }
#pragma unroll
    for (int q = 0; q < G::LB; ++q) {
      const int row = (wave * G::LB + q) * 8 + (lane >> 3);
      offb[q] = row < w.n ? (uint32_t)row * ldb + ((lane & 7) ^ swizzle_b<PAIRED>(row)) * 16 : kOOB;
    }
  }
  __device__ __forceinline__ void issue(const Where& w, int kt) {
    const uint32_t at = lds + stage_in * G::STAGE, k = (uint32_t)kt * kStep;
#pragma unroll
    for (int q = 0; q < G::LA; ++q) load_lds16_settled(w.ra, at + (wave * G::LA + q) * 1024, offa[q], k);
#pragma unroll
    for (int q = 0; q < G::LB; ++q) load_lds16_settled(w.rb, at + G::A + (wave * G::LB + q) * 1024, offb[q], k);
    stage_in = stage_in == G::NS - 1 ? 0 : stage_in + 1;
    if (kt == 0 || ((w.b0 + kt) & 3) == 0) {
      // waves 0 .. BMT / 64 - 1 bring the rows' scales, waves 4 .. 7 the columns'
      const int first = wave < 4 ? wave * 64 : BMT + (wave - 4) * 64;
      if (wave >= 4 || wave * 64 < BMT)
        load_lds4_settled(w.rs, lds + G::NS * G::STAGE + word_in * G::WORDS + first * 4, w.offs, (uint32_t)((w.b0 + kt) >> 2) * 4);
      word_in = (word_in + 1) & (kWordRing - 1);
    }
  }
  __device__ __forceinline__ void prologue(const Where& w) {
#pragma unroll
    for (int i = 0; i < G::NS - 1; ++i)
      if (i < w.blocks) issue(w, i);
  }
};

// The tile's sums. EXACT: in bf16, with exact products; else on the 8-bit instruction (BF16_FAST).
template <int BMT, bool PAIRED, bool EXACT> struct Worker {
  typedef Geo<BMT> G;
  f32x4_t acc[G::TM][G::TN];
  int stage = 0, word = 0;
  uint32_t sa[G::TM], sb[G::TN];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < G::TM; ++i)
#pragma unroll
      for (int j = 0; j < G::TN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  // 16 bytes (16 k) of a row: chunk g for the step's first half of k, g + 4 for its second. (Which k
  // of a block a lane has does not matter as long as both operands agree.)
  static __device__ __forceinline__ u32x4_t chunk(const uint8_t* rows, int row, int swizzle, int c) {
    return *(const u32x4_t*)(rows + row * kStep + (c ^ swizzle) * 16);
  }
  static __device__ __forceinline__ i32x8_t joined(u32x4_t lo, u32x4_t hi) {
    return i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
  }
  // Fragments are read ahead of the products that take them, so that the matrix cores do not wait for
  // LDS; the scheduling barriers keep the reads where they are.
  __device__ __forceinline__ void step(const uint8_t* smem, int wm, int wn, int lane, int b, bool first) {
    const int x = lane & 15, g = lane >> 4;
    const uint8_t *As = smem + stage * G::STAGE, *Bs = As + G::A;
    if (first || (b & 3) == 0) {
      const uint32_t* w = (const uint32_t*)(smem + G::NS * G::STAGE + word * G::WORDS);
#pragma unroll
      for (int i = 0; i < G::TM; ++i) sa[i] = w[wm * (BMT / 2) + i * 16 + x] >> (b & 3) * 8;
#pragma unroll
      for (int j = 0; j < G::TN; ++j) sb[j] = w[BMT + wn * 64 + column_of<PAIRED>(j, x)] >> (b & 3) * 8;
      word = (word + 1) & (kWordRing - 1);
    } else {
#pragma unroll
      for (int i = 0; i < G::TM; ++i) sa[i] >>= 8;
#pragma unroll
      for (int j = 0; j < G::TN; ++j) sb[j] >>= 8;
    }
    const int arow = wm * (BMT / 2) + x, brow = wn * 64;
    auto read_a = [&](int i, int h) { return chunk(As, arow + i * 16, x & 7, g + 4 * h); };
    auto read_b = [&](int j, int h) {
      const int row = brow + column_of<PAIRED>(j, x);
      return chunk(Bs, row, swizzle_b<PAIRED>(row), g + 4 * h);
    };
    if constexpr (EXACT) {
      u32x4_t raw[G::TN], a = read_a(0, 0);
      bf16x8_t bw[G::TN][2];
#pragma unroll
      for (int j = 0; j < G::TN; ++j) raw[j] = read_b(j, 0);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int j = 0; j < G::TN; ++j) {
          const float by = scale8(sb[j] & 0xff);
          bw[j][0] = decode8(raw[j][0], raw[j][1], by);
          bw[j][1] = decode8(raw[j][2], raw[j][3], by);
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < G::TM; ++i) {
          const u32x4_t now = a;
          if (i + 1 < G::TM)
            a = read_a(i + 1, h);
          else if (h == 0)
            a = read_a(0, 1);
          if (h == 0 && i >= G::TM - 4) raw[i - (G::TM - 4)] = read_b(i - (G::TM - 4), 1);
          __builtin_amdgcn_sched_barrier(0);
          const float by = scale8(sa[i] & 0xff);
          const bf16x8_t a0 = decode8(now[0], now[1], by), a1 = decode8(now[2], now[3], by);
#pragma unroll
          for (int j = 0; j < G::TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[j][0], a0, acc[i][j], 0, 0, 0);
#pragma unroll
          for (int j = 0; j < G::TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[j][1], a1, acc[i][j], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
      }
    } else {
      i32x8_t bw[G::TN];
      u32x4_t a[2] = {read_a(0, 0), read_a(0, 1)};
#pragma unroll
      for (int j = 0; j < G::TN; ++j) bw[j] = joined(read_b(j, 0), read_b(j, 1));
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < G::TM; ++i) {
        const i32x8_t now = joined(a[0], a[1]);
        if (i + 1 < G::TM) {
          a[0] = read_a(i + 1, 0);
          a[1] = read_a(i + 1, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bw[j], now, acc[i][j], 0, 0, 0, (int)sb[j], 0,
                                                                       (int)sa[i]);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    stage = stage == G::NS - 1 ? 0 : stage + 1;
  }
  template <typename V> __device__ __forceinline__ void store(const Where& w, int wm, int wn, int lane) const {
    constexpr int each = 16 / sizeof(V);
    const int x = lane & 15, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < G::TM; ++i) {
      const int m = wm * (BMT / 2) + i * 16 + x;
      if (m >= w.m) continue;
      V* row = (V*)w.C + m * w.ldc;
#pragma unroll
      for (int j = 0; j < G::TN; j += PAIRED ? 2 : 1) {
        const int n = wn * 64 + column_of<PAIRED>(j, 4 * g);
        u32x4_t out;
        if constexpr (PAIRED) {
          const f32x4_t &a = acc[i][j], &c = acc[i][j + 1];
          out = u32x4_t{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(c[0], c[1]), pack_bf16(c[2], c[3])};
        } else {
          __builtin_memcpy(&out, &acc[i][j], 16);
        }
        if (n + each <= w.n) {
          __builtin_memcpy(row + n, &out, 16);
        } else {
          V v[each];
          __builtin_memcpy(v, &out, 16);
#pragma unroll
          for (int e = 0; e < each; ++e)
            if (n + e < w.n) row[n + e] = v[e];
        }
      }
    }
  }
};

// before[e]: units of `size` rows in the runs before run e, up to before[E]; by the first wave.
__device__ __forceinline__ void count_units(const int32_t* __restrict__ offsets, int E, int rows, int size, int* before) {
  if (threadIdx.x >= kWave) return;
  const int lane = lane_id(), per = (E + kWave - 1) / kWave, e0 = min(lane * per, E), e1 = min(e0 + per, E);
  int n = 0;
  for (int e = e0; e < e1; ++e) {
    const int len = offsets ? max(offset8(offsets, e + 1, rows) - offset8(offsets, e, rows), 0) : rows;
    before[e] = n;
    n += (len + size - 1) / size;
  }
  const int incl = wave_incl_scan(n);
  for (int e = e0; e < e1; ++e) before[e] += incl - n;
  if (lane == kWave - 1) before[E] = incl;
}

// Tile `id` of tiles_m x tiles_n: neighbouring workgroups are on different XCDs, so each XCD (id % 8) gets a
// run of tiles, walked in groups of 8 rows of tiles so that its L2 serves them. false: no such tile.
__device__ __forceinline__ bool tile_at(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
  const uint32_t total = tiles_m * tiles_n, run = (total + 7) / 8, at = id / 8, v = id % 8 * run + at;
  if (at >= run || v >= total) return false;
  const uint32_t first = v / (8 * tiles_n) * 8, high = min(tiles_m - first, 8u), in = v - first * tiles_n;
  tn = in / high;
  tm = first + in - tn * high;
  return true;
}

// WEIGHTS: results are the weights' gradients of expert after expert; else the rows of run after run.
template <int BMT, bool EXACT, bool WEIGHTS, typename V>
__global__ __launch_bounds__(kTileThreads) void k_product8_tiles(Product8 p) {
  constexpr bool PAIRED = sizeof(V) == 2;
  typedef Geo<BMT> G;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[G::SMEM];
  __shared__ int before[kMaxExperts8 + 1];
  const int rows = (int)p.rows;
  count_units(p.offsets, p.E, rows, WEIGHTS ? kBlock8 : BMT, before);
  __syncthreads();
  const uint32_t tiles_n = (uint32_t)cdiv(WEIGHTS ? p.K : p.N, kTileN), each = (uint32_t)cdiv(p.N, BMT);
  // the gradients go by one expert after the other, each dealt over all XCDs: their sums are as long as
  // the experts' runs
  const uint32_t tiles_m = __builtin_amdgcn_readfirstlane(WEIGHTS ? each : (uint32_t)before[p.E]);
  const uint32_t turn = (tiles_m * tiles_n + 7) / 8 * 8, limit = WEIGHTS ? p.E * turn : turn;
  const int64_t ld = WEIGHTS ? p.columns : p.K, ls = WEIGHTS ? p.columns / kBlock8 : scale_row8(p.K);
  Loader<BMT, PAIRED> load(smem);
  const int lane = load.lane, wave = load.wave, wm = wave & 1, wn = wave >> 1;

  auto find = [&](uint32_t id, Where& w) {  // the tile at id or later of this workgroup's
    uint32_t e = 0, tm, tn;
    for (; id < limit; id += gridDim.x) {
      if (WEIGHTS) e = id / turn;
      if (tile_at(id - e * turn, tiles_m, tiles_n, tm, tn)) break;
    }
    if (id >= limit) return id;
    const uint8_t *A, *As, *B, *Bs;
    int bshift = 0;
    if constexpr (WEIGHTS) {
      const int64_t m0 = (int64_t)tm * BMT, n0 = (int64_t)tn * kTileN;
      const int b = before[e];
      w.m = (int)min((int64_t)BMT, p.N - m0);
      w.n = (int)min((int64_t)kTileN, p.K - n0);
      w.blocks = max(min(before[e + 1] - b, (int)ls - b), 0);
      w.b0 = b & 3;
      A = p.A + m0 * ld + (int64_t)b * kBlock8;
      B = p.B + n0 * ld + (int64_t)b * kBlock8;
      As = p.As + m0 * ls + (b - w.b0);
      Bs = p.Bs + n0 * ls + (b - w.b0);
      w.C = (char*)p.C + (((int64_t)e * p.N + m0) * p.K + n0) * (int64_t)sizeof(V);
      w.ldc = p.K;
    } else {
      int lo = 0, hi = p.E - 1;  // the last run with before[e] <= tm; it has units
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (before[mid] <= (int)tm)
          lo = mid;
        else
          hi = mid - 1;
      }
      e = __builtin_amdgcn_readfirstlane(lo);
      const int run = p.offsets ? offset8(p.offsets, (int)e, rows) : 0;
      const int end = p.offsets ? offset8(p.offsets, (int)e + 1, rows) : rows;
      const int64_t m0 = run + (int64_t)((int)tm - before[e]) * BMT, n0 = (int64_t)tn * kTileN;
      w.m = (int)min((int64_t)BMT, end - m0);
      w.n = (int)min((int64_t)kTileN, p.N - n0);
      w.blocks = (int)(p.K / kBlock8);
      w.b0 = 0;
      A = p.A + m0 * ld;
      As = p.As + m0 * ls;
      B = p.B + ((int64_t)e * p.N + n0) * ld;
      Bs = p.Bs + ((int64_t)e * blocks8(p.N) + n0 / kBlock8) * ls;
      bshift = 7;
      w.C = (char*)p.C + (m0 * p.N + n0) * (int64_t)sizeof(V);
      w.ldc = p.N;
    }
    w.m = __builtin_amdgcn_readfirstlane(w.m);
    w.n = __builtin_amdgcn_readfirstlane(w.n);
    w.blocks = __builtin_amdgcn_readfirstlane(w.blocks);
    w.b0 = __builtin_amdgcn_readfirstlane(w.b0);
    w.ra = buffer_of(A, w.m * ld);
    w.rb = buffer_of(B, w.n * ld);
    const int row = (wave & 3) * 64 + lane;
    w.rs = wave < 4 ? buffer_of(As, w.m * ls) : buffer_of(Bs, (((w.n - 1) >> bshift) + 1) * ls);
    w.offs = row < (wave < 4 ? w.m : w.n) ? (uint32_t)(wave < 4 ? row : row >> bshift) * (uint32_t)ls : kOOB;
    return id;
  };

  Where w;
  uint32_t id = find(blockIdx.x, w);
  if (id >= limit) return;
  Worker<BMT, PAIRED, EXACT> work;
  load.setup(w, (uint32_t)ld, (uint32_t)ld);
  load.prologue(w);
  for (;;) {
    work.clear();
    for (int kt = 0; kt < w.blocks; ++kt) {
      // this stage has landed (of three, the next may still be on its way) and this wave's reads of the
      // last one are done; after the barrier that holds for all waves, and its place may be filled again
      static_assert(G::LA + G::LB < 16, "the wait's low bits");
      if (G::NS == 3 && kt + 1 < w.blocks)
        __builtin_amdgcn_s_waitcnt(0x0070 | (G::LA + G::LB));
      else
        __builtin_amdgcn_s_waitcnt(0x0070);
      __syncthreads();
      if (kt + G::NS - 1 < w.blocks) load.issue(w, kt + G::NS - 1);
      work.step(smem, wm, wn, lane, w.b0 + kt, kt == 0);
    }
    Where next;
    const uint32_t id2 = find(id + gridDim.x, next);
    if (id2 < limit) {
      load.setup(next, (uint32_t)ld, (uint32_t)ld);
      load.prologue(next);
    }
    work.template store<V>(w, wm, wn, lane);
    if (id2 >= limit) break;
    w = next;
    id = id2;
  }
}

// ---- few rows of an expert: its weights pass by once ---------------------------------------
// A wave has 16 columns and up to 16 MT rows. The weights come from memory into registers, the next ones
// on their way while some are used: bound by their bytes, so the products are the exact ones in bf16. The
// rows, which all waves of a workgroup need, lie in LDS in chunks of 1024 k (read by every wave from the L2,
// they and their scales took as long as the weights: 64 rows of eight experts, 4096 x 4096, 45 us, without
// them 27). The KS waves that share columns have a part of the blocks each and add their sums over LDS, in
// order; so few columns still fill the chip.
constexpr int kStreamThreads = 512, kStreamWaves = kStreamThreads / kWave;

template <int MT, int KS, typename V>
__global__ __launch_bounds__(kStreamThreads) void k_product8_stream(Product8 p, int64_t units) {
  constexpr int STRIPS = kStreamWaves / KS, UNROLL = 2;
  constexpr int CHUNK = 1024, BLOCKS = CHUNK / kBlock8, WORDS = BLOCKS / 4;  // of a row
  constexpr int CODES = 16 * MT * CHUNK, LOADS = CODES / 1024 / kStreamWaves;
  static_assert(BLOCKS % KS == 0 && 16 * MT * WORDS <= 2 * kWave && CODES >= kStreamWaves * MT * 1024, "");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[CODES + 512];
  const int lane = lane_id(), x = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), ks = wave % KS, strip = wave / KS;
  const int rows = (int)p.rows, blocks = (int)(p.K / kBlock8);
  const int64_t strips = cdiv(p.N, 16 * STRIPS), total = units * strips, sk = scale_row8(p.K);
  const uint32_t lds = __builtin_amdgcn_readfirstlane(
      (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)smem);
  for (int64_t id = blockIdx.x; id < total; id += gridDim.x) {
    const int64_t unit = id / strips, n0 = ((id - unit * strips) * STRIPS + strip) * 16;
    const Unit u = unit_of(p.offsets, p.E, rows, 16 * MT, (int)unit);
    if (u.expert < 0) return;
    const int count = __builtin_amdgcn_readfirstlane(u.count), expert = __builtin_amdgcn_readfirstlane(u.expert);
    const int64_t first = __builtin_amdgcn_readfirstlane(u.first), n = min(n0 + x, p.N - 1);
    const uint8_t* B = p.B + (expert * p.N + n) * p.K + g * 16;
    const uint32_t* Bs = (const uint32_t*)(p.Bs + (expert * blocks8(p.N) + min(n0, p.N - 1) / kBlock8) * sk);
    const u32x4_t ra = buffer_of(p.A + first * p.K, count * p.K), rs = buffer_of(p.As + first * sk, count * sk);
    f32x4_t acc[MT] = {};
    for (int c0 = 0; c0 < blocks; c0 += BLOCKS) {
      // a load fills 1 KB of one row, eight blocks; chunk c of a block lies at position c ^ (row & 7)
#pragma unroll
      for (int q = 0; q < LOADS; ++q) {
        const int at = (wave * LOADS + q) * 1024, row = at / CHUNK, b = c0 + at % CHUNK / kBlock8 + lane / 8;
        const bool there = row < count && b < blocks;
        load_lds16_settled(ra, lds + at, there ? (uint32_t)row * (uint32_t)p.K + b * kBlock8 + ((lane & 7) ^ (row & 7)) * 16 : kOOB, 0);
      }
      if (wave < 2) {
        const int word = wave * 64 + lane, row = word / WORDS, b = c0 + word % WORDS * 4;
        load_lds4_settled(rs, lds + CODES + wave * 256, row < count && b < blocks ? (uint32_t)row * (uint32_t)sk + b : kOOB, 0);
      }
      u32x4_t w[UNROLL][2], next[UNROLL][2];
      const int mine = (min(blocks - c0, BLOCKS) - ks + KS - 1) / KS;  // this wave's: c0 + ks, c0 + ks + KS, ...
      auto fetch = [&](int i0, u32x4_t(&to)[UNROLL][2]) {
#pragma unroll
        for (int q = 0; q < UNROLL; ++q) {
          const int b = min(c0 + ks + max(min(i0 + q, mine - 1), 0) * KS, blocks - 1);
          const uint8_t* at = B + (int64_t)b * kBlock8;
          to[q][0] = *(const u32x4_t*)at;
          to[q][1] = *(const u32x4_t*)(at + 64);
        }
      };
      fetch(0, w);
      __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wave's loads into LDS have landed
      __syncthreads();
      for (int i0 = 0; i0 < mine; i0 += UNROLL) {
        if (i0 + UNROLL < mine) fetch(i0 + UNROLL, next);
#pragma unroll
        for (int q = 0; q < UNROLL; ++q) {
          if (i0 + q >= mine) break;
          const int in = ks + (i0 + q) * KS, b = c0 + in;
          const float by = scale8(Bs[b >> 2] >> (b & 3) * 8 & 0xff);
          bf16x8_t bw[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) bw[h] = decode8(w[q][h / 2][h % 2 * 2], w[q][h / 2][h % 2 * 2 + 1], by);
#pragma unroll
          for (int i = 0; i < MT; ++i)
            if (i * 16 < count) {
              const uint8_t* row = smem + (i * 16 + x) * CHUNK + in * kBlock8;
              const u32x4_t a[2] = {*(const u32x4_t*)(row + (g ^ (x & 7)) * 16), *(const u32x4_t*)(row + ((g + 4) ^ (x & 7)) * 16)};
              const float bya = scale8(smem[CODES + (i * 16 + x) * BLOCKS + in]);
#pragma unroll
              for (int h = 0; h < 4; ++h)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    bw[h], decode8(a[h / 2][h % 2 * 2], a[h / 2][h % 2 * 2 + 1], bya), acc[i], 0, 0, 0);
            }
        }
#pragma unroll
        for (int q = 0; q < UNROLL; ++q) {
          w[q][0] = next[q][0];
          w[q][1] = next[q][1];
        }
      }
      __syncthreads();  // the chunk's place is free again
    }
    if (KS > 1) {
      f32x4_t* part = (f32x4_t*)smem;  // [wave][MT][lane]
#pragma unroll
      for (int i = 0; i < MT; ++i) part[(wave * MT + i) * kWave + lane] = acc[i];
      __syncthreads();
      if (ks == 0)
#pragma unroll
        for (int i = 0; i < MT; ++i)
          for (int q = 1; q < KS; ++q) acc[i] += part[((wave + q) * MT + i) * kWave + lane];
      __syncthreads();
    }
    if (ks == 0)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int m = i * 16 + x;
        const int64_t at = n0 + 4 * g;
        if (m >= count || at >= p.N) continue;
        V* to = (V*)p.C + (first + m) * p.N + at;
        V v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = VT<V>::cvt(acc[i][e]);
        if (at + 4 <= p.N) {
          __builtin_memcpy(to, v, sizeof(v));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at + e < p.N) to[e] = v[e];
        }
      }
  }
}

dim3 grid_of(int64_t tiles, int threads) { return dim3((unsigned)std::min<int64_t>(tiles, max_blocks(threads))); }

template <int BMT, bool EXACT, bool WEIGHTS, typename V> hipError_t tiles(const Product8& p, int64_t count, hipStream_t s) {
  if (count > INT32_MAX - 8 * p.E) return hipErrorInvalidValue;  // of 2^15 results or more each: beyond any memory
  const unsigned grid = (unsigned)std::min<int64_t>(up(count, 8), up(device_cus(), 8));  // 8: see tile_at
  hipLaunchKernelGGL((k_product8_tiles<BMT, EXACT, WEIGHTS, V>), dim3(grid), dim3(kTileThreads), 0, s, p);
  return hipGetLastError();
}

// The 8-bit instruction only where the caller asks for it: its sums drop what lies 13 bits below the largest of eight
// products, in bf16 results too (256 * 256 - 256 * 256 + 1 gives 0).
template <int BMT, bool WEIGHTS> hipError_t tiles_of(const Product8& p, int32_t dtype, int64_t count, hipStream_t s) {
  if (dtype == SFL_BF16_FAST) return tiles<BMT, false, WEIGHTS, bf16_t>(p, count, s);
  return dtype == SFL_BF16 ? tiles<BMT, true, WEIGHTS, bf16_t>(p, count, s) : tiles<BMT, true, WEIGHTS, float>(p, count, s);
}

template <int MT, int KS> hipError_t stream(const Product8& p, int bf16, int64_t units, hipStream_t s) {
  const dim3 grid = grid_of(units * cdiv(p.N, 16 * (kStreamWaves / KS)), kStreamThreads);
  if (bf16)
    hipLaunchKernelGGL((k_product8_stream<MT, KS, bf16_t>), grid, dim3(kStreamThreads), 0, s, p, units);
  else
    hipLaunchKernelGGL((k_product8_stream<MT, KS, float>), grid, dim3(kStreamThreads), 0, s, p, units);
  return hipGetLastError();
}

// Units that any runs of `rows` rows in all take: every run ends in one that may not be full.
int64_t most_units(const Product8& p, int64_t size) {
  return p.offsets ? std::min(p.rows, p.rows / size + p.E) : cdiv(p.rows, size);
}

}  // namespace

// Which kernel, at K = 4096 in bf16 (µs a call, captured, over several sets of buffers; K weighs on all alike):
//                                                      exact products        8-bit instruction
//   rows x columns, experts      few rows   tiles of 128        of 256         128       256
//   64 x 4096, 1                   15           54           89             29        44
//   256 x 4096, 1                  29           54           92             30        47
//   512 x 4096, 1                  39           56           92             30        47
//   256 x 8192, 2                  43           56           92             34        47
//   64 x 4096, 8                   34           55           91             37        50
//   512 x 4096, 8                  47           55           92             41        52
//   1024 x 4096, 8                 81           58           95             45        55
//   2048 x 4096, 8                              66          100             49        65
//   4096 x 4096, 8                             126          118             87        68
//   16384 x 4096, 8                            480          426            305       252
//   12288 x 64, 1                  35           55           93
// The kernel for few rows costs what it has of results, the tiles what one round of them does, twice as much with
// exact products; where runs are short it reads every weight once, which no tile does cheaper.
bool few_rows(const Product8& p, int32_t dtype, int64_t live) {
  return p.rows <= 16 * live || p.rows * p.N <= (dtype == SFL_BF16_FAST ? 3 << 18 : 1 << 21);
}
// Tiles of 256 rows read a third less, but a round of them (one a CU) takes as long as 1.6 rounds of 128. Runs end half
// a tile short on average.
bool high_tiles(const Product8& p, int64_t live) {
  auto rounds = [&](int64_t size) {
    const double units = p.offsets ? (double)p.rows / size + live / 2.0 : (double)cdiv(p.rows, size);
    return std::max(1.0, units * cdiv(p.N, kTileN) / device_cus());
  };
  return rounds(256) < 0.62 * rounds(128);
}

hipError_t launch_product8(const Product8& p, int32_t dtype, hipStream_t s) {
  const bool bf16 = dtype != SFL_F32;
  const int64_t live = std::min<int64_t>(p.E, p.rows);
  if (few_rows(p, dtype, live)) {
    // 16 rows a unit take fewer registers and less LDS; runs of more rows would read their weights once more
    // for every 16 (8 to 128 rows of eight experts: 35 us either way)
    const bool short_runs = p.rows <= 4 * live;
    // two workgroups a CU at least; parts of k beyond that only add sums (64 rows of eight experts: 37, 31 and 41 us
    // in one, two and four parts; 12288 rows of 64 columns: 39, 30, 34 and 47 in one to eight)
    const int64_t waves = std::max(live, cdiv(p.rows, short_runs ? 16 : 64)) * cdiv(p.N, 16), want = (int64_t)device_cus() * 16;
    const int ks = waves * 8 <= want ? 8 : waves * 4 <= want ? 4 : waves * 2 <= want ? 2 : 1;
    if (short_runs) {
      const int64_t units = most_units(p, 16);
      return ks == 8 ? stream<1, 8>(p, bf16, units, s) : ks == 4 ? stream<1, 4>(p, bf16, units, s)
           : ks == 2 ? stream<1, 2>(p, bf16, units, s) : stream<1, 1>(p, bf16, units, s);
    }
    const int64_t units = most_units(p, 64);
    return ks == 8 ? stream<4, 8>(p, bf16, units, s) : ks == 4 ? stream<4, 4>(p, bf16, units, s)
         : ks == 2 ? stream<4, 2>(p, bf16, units, s) : stream<4, 1>(p, bf16, units, s);
  }
  const bool high = high_tiles(p, live);
  const int64_t count = most_units(p, high ? 256 : 128) * cdiv(p.N, kTileN);
  return high ? tiles_of<256, false>(p, dtype, count, s) : tiles_of<128, false>(p, dtype, count, s);
}

// The higher tiles where they fill the CUs: they read a third less (4096 rows, 4096 x 4096, eight experts: 206 us in fp32 against
// 257; 2048 rows, 768 x 1024, where 96 of them leave most CUs idle: 32 against 14).
hipError_t launch_product8_weights(const Product8& p, int32_t dtype, hipStream_t s) {
  const int64_t high = p.E * cdiv(p.N, 256) * cdiv(p.K, kTileN), low = p.E * cdiv(p.N, 128) * cdiv(p.K, kTileN);
  return high >= device_cus() ? tiles_of<256, true>(p, dtype, high, s) : tiles_of<128, true>(p, dtype, low, s);
}

}  // namespace sfl
