// Tokens to their experts and back. Slot (t, j) is the j-th choice of token t; expert order is a
// stable counting sort of the slots by expert, so an expert's rows are in token order:
//   pos(s) = #{slots of lower experts} + #{earlier slots of the same expert}, -1 for a slot of
//   no expert; Xs[pos] = X[t]; Y[t] = sum_j w Ys[pos]; dYs[pos] = w dY[t]; dw = <dY[t], Ys[pos]>.
// The gradient of the way there, dX[t] = sum_j dXs[pos], is the way back with weights of one.
//
// The passes over the rows are bound by memory and walk the tokens, so a token's own row is read
// or written once however many experts it has; the expert side's rows (1 + k or 1 + 2 k rows of
// traffic per token in all) are whole contiguous rows wherever they lie. Sums run over j in order,
// in fp32, and no sum depends on another token; only whole-number counts are atomic. Measured at
// 16384 x 4096 bf16 to two of eight experts: dispatch 77 us (5.2 TB/s), combine 74 (5.4), its gradient
// 127 (5.3); a 1 GiB copy reaches 5.2.
#include "block.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;
constexpr int kOrderThreads = 1024;

// ------------------------------------------------------------------------- the order ----

__device__ __forceinline__ int valid_expert(int e, int E) { return e >= 0 && e < E ? e : -1; }

// Exclusive prefix sums of total[E] in place by the first wave's lanes (a run of E / 64 each);
// returns the sum of all to every lane of that wave.
__device__ __forceinline__ int scan_experts(int* total, int E) {
  const int lane = lane_id(), run = (E + kWave - 1) / kWave, e0 = min(lane * run, E), e1 = min(e0 + run, E);
  int s = 0;
  for (int e = e0; e < e1; ++e) s += total[e];
  const int incl = wave_incl_scan(s);
  s = incl - s;
  for (int e = e0; e < e1; ++e) {
    const int c = total[e];
    total[e] = s;
    s += c;
  }
  return readlane_i(incl, kWave - 1);
}

// Lanes of the wave that have this lane's expert; none for a lane without one.
__device__ __forceinline__ uint64_t same_expert(int e, int E) {
  uint64_t same = ballot(e >= 0);
  for (int b = 0; (1 << b) < E; ++b) {
    const uint64_t m = ballot((e >> b) & 1);
    same &= ((e >> b) & 1) ? m : ~m;
  }
  return e >= 0 ? same : 0;
}

// Adds the slots first + thread, ... below last to cnt; one LDS atomic per wave and expert, so a
// batch whose slots all have one expert costs no more.
__device__ __forceinline__ void count_experts(const int32_t* __restrict__ expert, int64_t first, int64_t last, int E,
                                              int* cnt, int threads) {
  for (int64_t i0 = first; i0 < last; i0 += threads) {
    const int64_t i = i0 + threadIdx.x;
    const int e = i < last ? valid_expert(expert[i], E) : -1;
    const uint64_t same = same_expert(e, E);
    if (same && mbcnt(same) == 0) atomicAdd(&cnt[e], __popcll(same));
  }
}

// Few slots: workgroup 1 + t finds the rows of token t's slots by counting over all slots, and
// copies the token's row to them; workgroup 0 writes the offsets. Every thread holds up to
// kSmallPer slots; a wave's count is a ballot per 64 slots.
// Every workgroup reads all slots, so above 2048 of them the three launches below are faster
// (4096 slots, 4096 x 2 bf16: 20.3 us this way, 16.6 that way; 2048: 9.9 and 13).
constexpr int kSmallPer = 8, kSmallSlots = kSmallPer * kThreads;

template <typename V>
__global__ __launch_bounds__(kThreads) void k_expert_small(const int32_t* __restrict__ expert, int n, int k, int E,
                                                           int32_t* __restrict__ pos, int32_t* __restrict__ offsets,
                                                           const V* __restrict__ X, int64_t d, int64_t rows,
                                                           V* __restrict__ Xs) {
  __shared__ int cnt[kRouteMaxExperts];  // the offsets' workgroup; [k][4] partial counts in the others
  const int64_t t = (int64_t)blockIdx.x - 1;
  if (t < 0) {
    for (int e = threadIdx.x; e < E; e += kThreads) cnt[e] = 0;
    __syncthreads();
    count_experts(expert, 0, n, E, cnt, kThreads);
    __syncthreads();
    if (threadIdx.x < kWave) {
      const int sum = scan_experts(cnt, E);
      if (threadIdx.x == 0) offsets[E] = sum;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kThreads) offsets[e] = cnt[e];
    return;
  }
  constexpr int W = kThreads / kWave;
  const int wave = threadIdx.x / kWave;
  // the row's first chunks come in while the slots are counted
  const V* from = X + t * d;
  Vec8<V> v[2];
  if (X)
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = load_raw(from, cols<V>(i, threadIdx.x, kThreads), (int)d);
  int mine[kSmallPer];
#pragma unroll
  for (int i = 0; i < kSmallPer; ++i) {
    const int s = i * kThreads + threadIdx.x;
    mine[i] = s < n ? valid_expert(expert[s], E) : -1;
  }
  for (int j = 0; j < k; ++j) {
    const int s = (int)t * k + j, e = valid_expert(expert[s], E);
    int before = 0;
#pragma unroll
    for (int i = 0; i < kSmallPer; ++i)
      if (i * kThreads < n)
        before += __popcll(ballot(mine[i] >= 0 && (mine[i] < e || (mine[i] == e && i * kThreads + (int)threadIdx.x < s))));
    if (lane_id() == 0) cnt[j * W + wave] = before;
  }
  __syncthreads();
  if ((int)threadIdx.x < k) {
    const int s = (int)t * k + threadIdx.x, e = valid_expert(expert[s], E);
    int p = -1;
    if (e >= 0) {
      p = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) p += cnt[threadIdx.x * W + w];
    }
    pos[s] = p;
    cnt[kRouteMaxK * W + threadIdx.x] = p;
  }
  if (!X) return;
  __syncthreads();
  for (int i0 = 0; cols<V>(i0, threadIdx.x, kThreads).c0 < d; i0 += 2) {
    if (i0)
#pragma unroll
      for (int i = 0; i < 2; ++i) v[i] = load_raw(from, cols<V>(i0 + i, threadIdx.x, kThreads), (int)d);
    for (int j = 0; j < k; ++j) {
      const int p = cnt[kRouteMaxK * W + j];
      if (p >= 0 && p < rows)
#pragma unroll
        for (int i = 0; i < 2; ++i) store_raw(Xs + p * d, cols<V>(i0 + i, threadIdx.x, kThreads), (int)d, v[i]);
    }
  }
}

// More slots: each workgroup takes a run of slots, a multiple of 1024, counts its experts, and in a
// second launch adds up the counts before it and places its slots. (One launch in which every
// workgroup counts all slots itself: 1.4 us less at 2050 slots, none at 4096, 6 more at 16384.)
__global__ __launch_bounds__(kOrderThreads) void k_expert_count(const int32_t* __restrict__ expert, int64_t n,
                                                                int64_t run, int E, int32_t* __restrict__ count) {
  extern __shared__ int lds[];
  const int64_t first = blockIdx.x * run;
  for (int e = threadIdx.x; e < E; e += kOrderThreads) lds[e] = 0;
  __syncthreads();
  count_experts(expert, first, min(first + run, n), E, lds, kOrderThreads);
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kOrderThreads) count[(int64_t)blockIdx.x * E + e] = lds[e];
}

// LDS: total[E], next[E] (the next free row of each expert) and tile[waves][E] (the current 1024
// slots of each wave and expert).
__global__ __launch_bounds__(kOrderThreads) void k_expert_place(const int32_t* __restrict__ expert, int64_t n,
                                                                int64_t run, int E, const int32_t* __restrict__ count,
                                                                int32_t* __restrict__ pos,
                                                                int32_t* __restrict__ offsets) {
  extern __shared__ int lds[];
  constexpr int W = kOrderThreads / kWave;
  int* total = lds;
  int* next = lds + E;
  int* tile = lds + 2 * E;
  const int wave = threadIdx.x / kWave;
  for (int e = threadIdx.x; e < E; e += kOrderThreads) total[e] = next[e] = 0;
  __syncthreads();
  // sums over the runs before this one and over all, 1024 / E' parts of them at a time
  int width = 1;
  while (width < E) width *= 2;
  const int parts = kOrderThreads / width, part = threadIdx.x / width, e0 = threadIdx.x % width;
  if (e0 < E) {
    int all = 0, before = 0;
    for (int b = part; b < (int)gridDim.x; b += parts) {
      const int c = count[(int64_t)b * E + e0];
      all += c;
      before += b < (int)blockIdx.x ? c : 0;
    }
    atomicAdd(&total[e0], all);  // whole numbers: their order does not matter
    atomicAdd(&next[e0], before);
  }
  __syncthreads();
  if (wave == 0) {
    const int sum = scan_experts(total, E);
    if (blockIdx.x == 0 && threadIdx.x == 0) offsets[E] = sum;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kOrderThreads) {
    if (blockIdx.x == 0) offsets[e] = total[e];
    next[e] += total[e];
  }
  const int64_t first = blockIdx.x * run, last = min(first + run, n);
  for (int64_t i0 = first; i0 < last; i0 += kOrderThreads) {
    for (int e = threadIdx.x; e < W * E; e += kOrderThreads) tile[e] = 0;
    __syncthreads();
    const int64_t i = i0 + threadIdx.x;
    const int e = i < last ? valid_expert(expert[i], E) : -1;
    const uint64_t same = same_expert(e, E);
    const int before = mbcnt(same);
    if (e >= 0 && before == 0) tile[wave * E + e] = __popcll(same);
    __syncthreads();
    if (e >= 0) {
      int row = next[e] + before;
      for (int w = 0; w < wave; ++w) row += tile[w * E + e];
      pos[i] = row;
    } else if (i < last) {
      pos[i] = -1;
    }
    if (i0 + kOrderThreads >= last) break;
    __syncthreads();
    for (int x = threadIdx.x; x < E; x += kOrderThreads) {
      int c = 0;
      for (int w = 0; w < W; ++w) c += tile[w * E + x];
      next[x] += c;
    }
    __syncthreads();
  }
}

// Slots of a workgroup: a tile of 1024, more where that would take over 256 workgroups (each adds
// up the others' counts).
constexpr int kOrderBlocks = 256;
int64_t order_run(int64_t n) { return cdiv(cdiv(n, kOrderBlocks), kOrderThreads) * kOrderThreads; }

// -------------------------------------------------------------------------- the rows ----
// NT threads per token, chunks of 8 columns each: as many threads as there are chunks, up to a
// workgroup of 256 (16384 x 4096 bf16 to two of eight experts: dispatch 97 us with a wave per token,
// 78 with 256 threads; combine 94 and 79, its gradient 167 and 141).

constexpr int kRowChunks = 2;  // of a token's row, on their way together (84 -> 78 us)

template <typename V, int NT>
__global__ __launch_bounds__(kThreads) void k_expert_rows(const V* __restrict__ X, int64_t T, int64_t d64, int k,
                                                          const int32_t* __restrict__ pos, int64_t rows,
                                                          V* __restrict__ Xs) {
  const int64_t t = (int64_t)blockIdx.x * (kThreads / NT) + threadIdx.x / NT;
  if (t >= T) return;
  const int d = (int)d64;
  const V* from = X + t * d64;
  const int x = threadIdx.x % NT;
  for (int i0 = 0; cols<V>(i0, x, NT).c0 < d; i0 += kRowChunks) {
    Vec8<V> v[kRowChunks];
#pragma unroll
    for (int i = 0; i < kRowChunks; ++i) v[i] = load_raw(from, cols<V>(i0 + i, x, NT), d);
    for (int j = 0; j < k; ++j) {
      const int p = pos[t * k + j];
      if (p >= 0 && p < rows)
#pragma unroll
        for (int i = 0; i < kRowChunks; ++i) store_raw(Xs + p * d64, cols<V>(i0 + i, x, NT), d, v[i]);
    }
  }
}

// KS: slots whose rows are in flight together. Two for tokens of one or two slots (combine 79 -> 74
// us, gradient 135 -> 127 against four), four for more (16384 x 1024 to eight of 64: 59 -> 57 and
// 129 -> 119 us against two; eight are slower everywhere).
template <typename V, int NT, int KS>
__global__ __launch_bounds__(kThreads) void k_expert_combine(const V* __restrict__ Ys, int64_t T, int64_t d64, int k,
                                                             const int32_t* __restrict__ pos, int64_t rows,
                                                             const float* __restrict__ weight, V* __restrict__ Y) {
  const int64_t t = (int64_t)blockIdx.x * (kThreads / NT) + threadIdx.x / NT;
  if (t >= T) return;
  const int d = (int)d64;
  for (int i = 0;; ++i) {
    const Cols c = cols<V>(i, threadIdx.x % NT, NT);
    if (c.c0 >= d) break;
    float s[kVec] = {};
    for (int j0 = 0; j0 < k; j0 += KS) {
      Vec8<V> v[KS];
      float w[KS];
      bool in[KS];
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        const int64_t slot = t * k + min(j0 + j, k - 1);
        const int p = pos[slot];
        in[j] = j0 + j < k && p >= 0 && p < rows;
        w[j] = weight ? weight[slot] : 1.f;
        if (in[j]) v[j] = load_raw(Ys + p * d64, c, d);
      }
#pragma unroll
      for (int j = 0; j < KS; ++j)
        if (in[j])
#pragma unroll
          for (int e = 0; e < kVec; ++e) s[e] = fmaf(w[j], v[j].get(e), s[e]);
    }
    store_raw(Y + t * d64, c, d, rounded<V>(s));
  }
}

template <typename V, int NT, int KS>
__global__ __launch_bounds__(kThreads) void k_expert_combine_bwd(const V* __restrict__ dY, const V* __restrict__ Ys,
                                                                 int64_t T, int64_t d64, int k,
                                                                 const int32_t* __restrict__ pos, int64_t rows,
                                                                 const float* __restrict__ weight, V* __restrict__ dYs,
                                                                 float* __restrict__ dweight) {
  constexpr int W = NT > kWave ? NT / kWave : 1;
  __shared__ float red[2][kThreads / NT][W][KS];
  const int group = threadIdx.x / NT;
  const int64_t mine = (int64_t)blockIdx.x * (kThreads / NT) + group;
  const bool in = mine < T;  // a token past the end goes along (barriers) without slots
  const int64_t t = in ? mine : T - 1;
  const int d = (int)d64;
  int turn = 0;
  for (int j0 = 0; j0 < k; j0 += KS, turn ^= 1) {
    int p[KS];
    float w[KS], dot[KS];
#pragma unroll
    for (int j = 0; j < KS; ++j) {
      const int64_t slot = t * k + min(j0 + j, k - 1);
      p[j] = in && j0 + j < k ? pos[slot] : -1;
      if (p[j] >= rows) p[j] = -1;
      w[j] = weight ? weight[slot] : 1.f;
      dot[j] = 0.f;
    }
    for (int i = 0;; ++i) {
      const Cols c = cols<V>(i, threadIdx.x % NT, NT);
      if (c.c0 >= d) break;
      const Vec8<V> g = load_raw(dY + t * d64, c, d);
      const bool whole = raw_whole<V>(c, d);  // else some elements count in the neighbour's dot product
      Vec8<V> v[KS];
      if (dweight)
#pragma unroll
        for (int j = 0; j < KS; ++j)
          if (p[j] >= 0) v[j] = load_raw(Ys + p[j] * d64, c, d);
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        if (p[j] < 0) continue;
        if (dweight) {
          if (whole) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) dot[j] = fmaf(g.get(e), v[j].get(e), dot[j]);
          } else {
#pragma unroll
            for (int e = 0; e < kVec; ++e) dot[j] = raw_own<V>(e, c, d) ? fmaf(g.get(e), v[j].get(e), dot[j]) : dot[j];
          }
        }
        if (dYs) {
          float o[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) o[e] = w[j] * g.get(e);
          store_raw(dYs + p[j] * d64, c, d, rounded<V>(o));
        }
      }
    }
    if (!dweight) continue;
#pragma unroll
    for (int j = 0; j < KS; ++j) dot[j] = group_sum<(NT < kWave ? NT : kWave)>(dot[j]);
    if (NT > kWave) {
      if (lane_id() == 0)
#pragma unroll
        for (int j = 0; j < KS; ++j) red[turn][group][threadIdx.x % NT / kWave][j] = dot[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < KS; ++j) {
        dot[j] = 0.f;
#pragma unroll
        for (int x = 0; x < W; ++x) dot[j] += red[turn][group][x][j];
      }
    }
    if (in && threadIdx.x % NT == 0)
#pragma unroll
      for (int j = 0; j < KS; ++j)
        if (j0 + j < k) dweight[t * k + j0 + j] = dot[j];
  }
}

// Calls f with the threads per token and the slots in flight.
template <typename F> hipError_t with_threads(int64_t d, int k, F f) {
  using std::integral_constant;
  const int64_t n = cdiv(d, kVec);
#define SFL_NT(nt)                                                                       \
  if (n <= nt || nt == kThreads)                                                         \
    return k <= 2 ? f(integral_constant<int, nt>{}, integral_constant<int, 2>{})         \
                  : f(integral_constant<int, nt>{}, integral_constant<int, 4>{});
  SFL_NT(8) SFL_NT(16) SFL_NT(32) SFL_NT(64) SFL_NT(128) SFL_NT(256)
#undef SFL_NT
  return hipErrorInvalidValue;
}

}  // namespace

// The counts of as many workgroups as n slots can take, not of those that they do take (with runs of
// 2048 slots half as many as with 1024): a batch needs no more than a larger one.
size_t expert_workspace_bytes(int64_t T, int k, int E) {
  const int64_t n = T * k;
  return n <= kSmallSlots ? 0 : (size_t)std::min<int64_t>(cdiv(n, kOrderThreads), kOrderBlocks) * E * sizeof(int32_t);
}

hipError_t launch_expert_dispatch(const int32_t* expert, int64_t T, int k, int E, int32_t* pos, int32_t* offsets,
                                  const void* X, int bf16, int64_t d, int64_t rows, void* Xs, void* workspace,
                                  hipStream_t s) {
  const int64_t n = T * k;
  if (n <= kSmallSlots) {
    const dim3 grid((unsigned)T + 1);
    if (bf16)
      hipLaunchKernelGGL(k_expert_small<bf16_t>, grid, dim3(kThreads), 0, s, expert, (int)n, k, E, pos, offsets,
                         (const bf16_t*)X, d, rows, (bf16_t*)Xs);
    else
      hipLaunchKernelGGL(k_expert_small<float>, grid, dim3(kThreads), 0, s, expert, (int)n, k, E, pos, offsets,
                         (const float*)X, d, rows, (float*)Xs);
    return hipGetLastError();
  }
  const int64_t run = order_run(n);
  const unsigned blocks = (unsigned)cdiv(n, run);
  const size_t lds = (size_t)E * (2 + kOrderThreads / kWave) * sizeof(int32_t);
  if (lds > (64 << 10)) {
    const hipError_t e = hipFuncSetAttribute((const void*)k_expert_place, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_expert_count, dim3(blocks), dim3(kOrderThreads), E * sizeof(int32_t), s, expert, n, run, E,
                     (int32_t*)workspace);
  hipLaunchKernelGGL(k_expert_place, dim3(blocks), dim3(kOrderThreads), lds, s, expert, n, run, E,
                     (const int32_t*)workspace, pos, offsets);
  if (!X || rows == 0) return hipGetLastError();
  return with_threads(d, k, [&](auto nt, auto) {
    constexpr int NT = decltype(nt)::value;
    return over_tokens<kThreads, kThreads / NT>(T, [&](int64_t t0, int64_t n, dim3 grid) {
      if (bf16)
        hipLaunchKernelGGL((k_expert_rows<bf16_t, NT>), grid, dim3(kThreads), 0, s, (const bf16_t*)X + t0 * d, n, d, k,
                           pos + t0 * k, rows, (bf16_t*)Xs);
      else
        hipLaunchKernelGGL((k_expert_rows<float, NT>), grid, dim3(kThreads), 0, s, (const float*)X + t0 * d, n, d, k,
                           pos + t0 * k, rows, (float*)Xs);
    });
  });
}

hipError_t launch_expert_combine(const void* Ys, int bf16, int64_t T, int64_t d, int k, const int32_t* pos,
                                 int64_t rows, const float* weight, void* Y, hipStream_t s) {
  return with_threads(d, k, [&](auto nt, auto ks) {
    constexpr int NT = decltype(nt)::value, KS = decltype(ks)::value;
    return over_tokens<kThreads, kThreads / NT>(T, [&](int64_t t0, int64_t n, dim3 grid) {
      const float* w = weight ? weight + t0 * k : nullptr;
      if (bf16)
        hipLaunchKernelGGL((k_expert_combine<bf16_t, NT, KS>), grid, dim3(kThreads), 0, s, (const bf16_t*)Ys, n, d, k,
                           pos + t0 * k, rows, w, (bf16_t*)Y + t0 * d);
      else
        hipLaunchKernelGGL((k_expert_combine<float, NT, KS>), grid, dim3(kThreads), 0, s, (const float*)Ys, n, d, k,
                           pos + t0 * k, rows, w, (float*)Y + t0 * d);
    });
  });
}

hipError_t launch_expert_combine_bwd(const void* dY, const void* Ys, int bf16, int64_t T, int64_t d, int k,
                                     const int32_t* pos, int64_t rows, const float* weight, void* dYs, float* dweight,
                                     hipStream_t s) {
  return with_threads(d, k, [&](auto nt, auto ks) {
    constexpr int NT = decltype(nt)::value, KS = decltype(ks)::value;
    return over_tokens<kThreads, kThreads / NT>(T, [&](int64_t t0, int64_t n, dim3 grid) {
      const float* w = weight ? weight + t0 * k : nullptr;
      float* dw = dweight ? dweight + t0 * k : nullptr;
      if (bf16)
        hipLaunchKernelGGL((k_expert_combine_bwd<bf16_t, NT, KS>), grid, dim3(kThreads), 0, s,
                           (const bf16_t*)dY + t0 * d, (const bf16_t*)Ys, n, d, k, pos + t0 * k, rows, w, (bf16_t*)dYs, dw);
      else
        hipLaunchKernelGGL((k_expert_combine_bwd<float, NT, KS>), grid, dim3(kThreads), 0, s,
                           (const float*)dY + t0 * d, (const float*)Ys, n, d, k, pos + t0 * k, rows, w, (float*)dYs, dw);
    });
  });
}

}  // namespace sfl
