// Log probabilities of given tokens, entropy and the largest alternatives of every row of logits (paper appendix A.1, eq. 4: the
// logits of a step), and the gradient of the first two.  With x = z / T:
//
//   lse = log sum_v e^x_v     logprob = x_t - lse     H = lse - sum_v p_v x_v     p_v = e^(x_v - lse)
//   dz_v = [ g_l (delta_vt - p_v) - g_H p_v (log p_v + H) ] / T
//
// Forward: bound by the one read of the logits.  A thread keeps the largest logit m so far, the reference r of it, s = sum e^(x - r) and
// t = sum (x - r) e^(x - r), in units of log 2, so that H = log s - t / s takes no second pass; moving the reference by d turns (s, t)
// into (s, t + d s) 2^d.  Sixteen or 32 elements are summed in 32 bits at a time, their sums in 64: a row may have a million
// entries.  r is the value that was really subtracted, rounded as it is, and the outputs are formed from it, so that its rounding
// cancels.  Logits so large that x leaves fp32's range (a mask of the type's lowest value, and nothing else left) are subtracted first.
// A row goes to one workgroup where there are many; few rows are split, and a second launch joins the parts.
//
// Alternatives ride in the same pass at three lane exchanges and one LDS write per 128 (16-bit: 256) elements: the maximum of every such
// block of the row.  The n-th largest block maximum is a lower bound on the n-th largest element, and only blocks that
// reach it are read again - n of a thousand, most often.  What they hold at or above the bound is a short list, ranked by counting.
// A row where it is not short (long runs of equal values, a mask that leaves less than n, values that rise along the row) takes
// bounded steps more: the exact n-th largest of the blocks above the bound, and equal values in the order of their ids.
#include "launch.hpp"

#include <algorithm>
#include <type_traits>

namespace aurora {

constexpr int kLpThreads = 256;
constexpr int kLpWaves = kLpThreads / kWave;
constexpr int kLpVecs = 4;                              // 16-byte vectors of a thread in one step
constexpr int kLpStep = kLpThreads * kLpVecs;           // vectors of a step
constexpr int kLpMaxSteps = 64;                         // steps of a workgroup: bounds the block maxima in LDS
constexpr int kLpLanes = 8;                             // lanes that share a block: 128 bytes a load
constexpr int kLpGroups = kLpThreads / kLpLanes;        // columns of blocks: at least kLpMaxTop of them
constexpr int kLpBlocks = kLpMaxSteps * kLpGroups;      // and one for the elements outside whole vectors
constexpr int kLpList = 512;
constexpr int kLpMaxTop = 32;
constexpr int kLpMaxSplits = 64;
constexpr float kLpLog2e = 1.4426950408889634f;
constexpr double kLpLn2 = 0.69314718055994530942;
constexpr float kLpFloor = -1e4f;  // stands in for -inf times zero: 2^-10000 is zero as well
constexpr int kLpGridRows = 1 << 22;

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

template <typename T> struct LpType { static constexpr int kV = 16 / (int)sizeof(T); };

template <typename T>
__device__ __forceinline__ void lp_widen(const u32x4_t raw, float (&x)[LpType<T>::kV]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (sizeof(T) == 4) {
      x[w] = __uint_as_float(raw[w]);
    } else {
      x[2 * w] = __uint_as_float(raw[w] << 16);
      x[2 * w + 1] = __uint_as_float(raw[w] & 0xffff0000u);
    }
  }
}

// order of floats as unsigned numbers (-0 and +0 equal); a larger key is a larger value, or the same value at a lower id
__device__ __forceinline__ unsigned lp_order(float z) {
  const unsigned u = __float_as_uint(z + 0.f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float lp_value(unsigned o) { return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ unsigned long long lp_key(float z, int id) {
  return (unsigned long long)lp_order(z) << 32 | (0xffffffffu - (unsigned)id);
}

// The part [lo, hi) of a row that a workgroup takes: `vecs` whole vectors from element `first` on, up to kV - 1 elements before them and
// as many after.
struct LpPart { int lo, first, vecs, tail, hi, steps; };
template <typename T>
__device__ __forceinline__ LpPart lp_part(const T* row, int V, int split, int splits) {
  constexpr int kV = LpType<T>::kV;
  const int h = min((int)(((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T)), V);
  const int all = (V - h) / kV, per = (all + splits - 1) / splits;
  LpPart p;
  const int from = min(split * per, all), to = min(from + per, all);
  p.first = h + from * kV;
  p.vecs = to - from;
  p.tail = p.first + p.vecs * kV;
  p.lo = split == 0 ? 0 : p.first;
  p.hi = split == splits - 1 ? V : p.tail;
  p.steps = (p.vecs + kLpStep - 1) / kLpStep;
  return p;
}

// what is subtracted for the reference m: its rounded multiple, or, past kLpFar / c, m itself before the product
constexpr float kLpFar = 8.5e37f;
__device__ __forceinline__ bool lp_far(float m, float c) { return fabsf(m) * c > kLpFar; }
__device__ __forceinline__ double lp_ref(float m, float c) { return lp_far(m, c) ? (double)m * (double)c : (double)(m * c); }

struct LpSums { float m; double s, t; };
// the sums with reference `to` (the largest of several, c as above); nothing so far counts for nothing
__device__ __forceinline__ LpSums lp_moved(const LpSums& a, float to, float c) {
  if (a.m == to) return a;
  if (a.m == -INFINITY) return {to, a.s, a.t};  // (zeros, or NaN)
  const float d = (float)(lp_ref(a.m, c) - lp_ref(to, c));
  const double f = (double)__builtin_amdgcn_exp2f(d);
  // (far below: its distance must not turn 0 into NaN)
  return {to, f * a.s, f > 0 ? f * (a.t + (double)d * a.s) : 0.0 * a.s};
}

// the row's numbers from its sums (a row without anything finite has lse -inf and entropy 0); returns the logsumexp in units of log 2
__device__ __forceinline__ double lp_finish(const LogprobLaunch& P, size_t row, const LpSums& x, float c, float z_t, bool known) {
  const bool none = x.s == 0.0 && x.m == -INFINITY;
  const double l2 = none ? 0.0 : log2(x.s), r = lp_ref(x.m, c);
  if (P.lse) P.lse[row] = none ? -INFINITY : (float)(kLpLn2 * (r + l2));
  if (P.entropy) P.entropy[row] = none ? 0.f : (float)(kLpLn2 * (l2 - x.t / x.s));
  if (P.logprob) {
    float lp = 0.f;
    if (known) lp = none || z_t == -INFINITY ? -INFINITY : (float)(kLpLn2 * ((double)z_t * (double)c - r - l2));
    P.logprob[row] = lp;
  }
  return r + l2;
}

__device__ __forceinline__ float lp_temperature(const LogprobLaunch& P, size_t row) {
  const float T = P.temperatures ? P.temperatures[row] : P.temperature;
  return T > 0.f ? T : 1.f;
}
__device__ __forceinline__ float lp_scale(const LogprobLaunch& P, size_t row) { return kLpLog2e / lp_temperature(P, row); }

// ---- selection of the n largest of a workgroup's part -------------------------------------------------------------------
struct LpLds {
  float bm[kLpBlocks + 1];            // block maxima; the last one is of the elements outside whole vectors
  float col[kLpGroups];               // and the maxima of their columns
  unsigned short blocks[kLpBlocks + 1];
  unsigned long long list[kLpList];
  int cnt[16][4];
  int n_blocks, n_list;
  int best[kLpWaves];
};

// The largest bound that at least n of the workgroup's values reach (thread t holds kPer of them, as lp_order keys; 0: no value):
// two bits at a time from the top.  0 if there are fewer than n.
template <int kPer>
__device__ __forceinline__ unsigned lp_nth(const unsigned (&v)[kPer], int n, LpLds& L) {
  const int tid = threadIdx.x, lane = tid & 63;
  __syncthreads();
  if (tid < 64) L.cnt[tid >> 2][tid & 3] = 0;
  __syncthreads();
  unsigned p = 0;
#pragma unroll 1
  for (int step = 0; step < 16; ++step) {
    const int sh = 30 - 2 * step;
    int c[3] = {0, 0, 0};
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      const unsigned bound = p | (unsigned)(q + 1) << sh;
#pragma unroll
      for (int i = 0; i < kPer; ++i) c[q] += __popcll(__ballot(v[i] >= bound));
    }
    if (lane < 3) {
      const int mine = lane == 0 ? c[0] : lane == 1 ? c[1] : c[2];
      if (mine) atomicAdd(&L.cnt[step][lane], mine);
    }
    __syncthreads();
    const int q = L.cnt[step][2] >= n ? 3 : L.cnt[step][1] >= n ? 2 : L.cnt[step][0] >= n ? 1 : 0;
    p |= (unsigned)q << sh;
  }
  return p;
}

// element `i` of block `blk` in the order lane, vector, element - and whether there is one
template <typename T>
__device__ __forceinline__ bool lp_element(const T* row, const LpPart& w, int blk, int i, int& id, float& z) {
  constexpr int kV = LpType<T>::kV;
  if (blk == kLpBlocks) {  // outside whole vectors
    const int before = w.first - w.lo;
    id = i < before ? w.lo + i : w.tail + i - before;
    if (i >= before + w.hi - w.tail) return false;
  } else {
    const int step = blk / kLpGroups, lane = (blk % kLpGroups) * kLpLanes + (i / kV) % kLpLanes;
    const int vec = step * kLpStep + i / (kV * kLpLanes) * kLpThreads + lane;
    if (vec >= w.vecs) return false;
    id = w.first + vec * kV + i % kV;
  }
  z = to_f32<T>(row[id]);
  return true;
}

// Lists what the blocks in L.blocks hold above the bound (or at it, with_ties), a vector a thread at a time; stops once the list is past
// its size.  Returns how many there are, kLpList + 1 if too many.
template <typename T>
__device__ __forceinline__ int lp_gather(const T* row, const LpPart& w, unsigned bound, bool with_ties, LpLds& L) {
  constexpr int kV = LpType<T>::kV, kPer = kLpLanes * kLpVecs;
  __syncthreads();
  if (threadIdx.x == 0) L.n_list = 0;
  __syncthreads();
  auto offer = [&](float z, int id) {
    const unsigned o = lp_order(z);
    if (o > bound || (with_ties && o == bound)) {
      const int at = atomicAdd(&L.n_list, 1);
      if (at < kLpList) L.list[at] = lp_key(z, id);
    }
  };
  const int all = L.n_blocks * kPer;
  for (int i = threadIdx.x; i < all; i += kLpThreads) {
    if (*(volatile int*)&L.n_list > kLpList) break;
    const int blk = L.blocks[i / kPer], u = i % kPer;
    if (blk == kLpBlocks) {  // outside whole vectors: less than a vector's elements before, and after them
      int id;
      float z;
      if (u < 2 * kV && lp_element(row, w, blk, u, id, z)) offer(z, id);
      continue;
    }
    const int vec = blk / kLpGroups * kLpStep + u / kLpLanes * kLpThreads + blk % kLpGroups * kLpLanes + u % kLpLanes;
    if (vec >= w.vecs) continue;
    const int id = w.first + vec * kV;
    float x[kV];
    lp_widen<T>(*(const u32x4_t*)(row + id), x);
#pragma unroll
    for (int e = 0; e < kV; ++e) offer(x[e], id + e);
  }
  __syncthreads();
  return min(L.n_list, kLpList + 1);
}

// lists the blocks whose maximum reaches the bound (above: is above it)
__device__ __forceinline__ void lp_blocks(int steps, unsigned bound, bool above, LpLds& L) {
  __syncthreads();
  if (threadIdx.x == 0) L.n_blocks = 0;
  __syncthreads();
  for (int i = threadIdx.x; i <= steps * kLpGroups; i += kLpThreads) {
    const int blk = i < steps * kLpGroups ? i : kLpBlocks;
    const unsigned o = lp_order(L.bm[blk]);
    if (above ? o > bound : o >= bound) L.blocks[atomicAdd(&L.n_blocks, 1)] = (unsigned short)blk;
  }
  __syncthreads();
}

// The n largest of the part, by value and then by id, to out(rank, key): every rank below n is given, key 0 where there is none.
template <typename T, typename Out>
__device__ __forceinline__ void lp_select(const T* row, const LpPart& w, int n, LpLds& L, Out out) {
  constexpr int kV = LpType<T>::kV, kBlock = kV * kLpLanes * kLpVecs;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // The n-th largest column maximum: as good a bound for most rows, and one wavefront finds it by counting, without a barrier.
  unsigned bound;
  {
    static_assert(kLpGroups <= kWave && kLpGroups >= kLpMaxTop, "a column a lane");
    const unsigned mine = lane < kLpGroups ? lp_order(L.col[lane]) : 0u;
    int above = 0;
#pragma unroll
    for (int i = 0; i < kLpGroups; ++i) {
      const unsigned other = __builtin_amdgcn_readlane(mine, i);
      above += other > mine || (other == mine && i < lane);
    }
    bound = __builtin_amdgcn_readlane(mine, __ffsll((unsigned long long)__ballot(above == n - 1)) - 1);
  }
  lp_blocks(w.steps, bound, false, L);
  int count = lp_gather(row, w, bound, true, L);
  bool ties = false;  // the equal ones are still to be found
  if (count > kLpList) {
    // The n-th largest block maximum is closer, and less than n blocks are above it.
    const int used = w.steps * kLpGroups;
    {
      constexpr int kPer = (kLpBlocks + kLpThreads - 1) / kLpThreads;
      unsigned v[kPer + 1];
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = tid + i * kLpThreads < used ? lp_order(L.bm[tid + i * kLpThreads]) : 0u;
      v[kPer] = tid == 0 ? lp_order(L.bm[kLpBlocks]) : 0u;
      bound = lp_nth(v, n, L);
    }
    lp_blocks(w.steps, bound, true, L);
    count = lp_gather(row, w, bound, false, L);
    ties = true;
    if (count > kLpList) {
      // They hold more than the list: the n-th largest element is among theirs.
      constexpr int kPer = (kLpMaxTop * kBlock + kLpThreads - 1) / kLpThreads;
      unsigned v[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = tid + i * kLpThreads;
        int id;
        float z;
        v[i] = e < L.n_blocks * kBlock && lp_element(row, w, L.blocks[e / kBlock], e % kBlock, id, z) ? lp_order(z) : 0u;
      }
      bound = lp_nth(v, n, L);
      count = lp_gather(row, w, bound, true, L);
      ties = count > kLpList;
      if (ties) count = lp_gather(row, w, bound, false, L);
    }
  }
  // rank by counting
  for (int i = tid; i < count; i += kLpThreads) {
    const unsigned long long k = L.list[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += L.list[j] > k;
    if (rank < n) out(rank, k);
  }
  int have = min(count, n);
  if (ties && have < n) {
    // Equal values in the order of their ids: the row's pieces in order, in each the lowest id not yet taken.
    const float at = lp_value(bound);
    for (int piece = -1; piece <= w.steps && have < n; ++piece) {
      int ids[kLpVecs * kV];
      int m = 0;
      if (piece < 0 || piece == w.steps) {  // the elements before, and after, the vectors
        const int id = (piece < 0 ? w.lo : w.tail) + tid;
        ids[0] = id < (piece < 0 ? w.first : w.hi) && to_f32<T>(row[id]) == at ? id : INT32_MAX;
        m = 1;
      } else {
#pragma unroll
        for (int u = 0; u < kLpVecs; ++u) {
          const int vec = piece * kLpStep + u * kLpThreads + tid;
#pragma unroll
          for (int e = 0; e < kV; ++e) {
            const int id = w.first + vec * kV + e;
            ids[u * kV + e] = vec < w.vecs && to_f32<T>(row[id]) == at ? id : INT32_MAX;
          }
        }
        m = kLpVecs * kV;
      }
      int last = -1;
      while (have < n) {
        int low = INT32_MAX;
#pragma unroll
        for (int i = 0; i < kLpVecs * kV; ++i)
          if (i < m && ids[i] > last) low = min(low, ids[i]);
        low = wave_min(low);
        __syncthreads();
        if (lane == 0) L.best[wave] = low;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kLpWaves; ++i) low = min(low, L.best[i]);
        if (low == INT32_MAX) break;
        if (tid == 0) out(have, lp_key(at, low));
        ++have;
        last = low;
      }
    }
  }
  for (int i = have + tid; i < n; i += kLpThreads) out(i, 0ull);
}

// ---- forward --------------------------------------------------------------------------------------------------------------
template <typename T, bool kTop>
__global__ __launch_bounds__(kLpThreads) void logprob_rows_kernel(LogprobLaunch P) {
  constexpr int kV = LpType<T>::kV;
  __shared__ LpSums s_part[kLpWaves];
  __shared__ float s_m[kLpWaves];
  __shared__ double s_lse2;
  __shared__ typename std::conditional<kTop, LpLds, int>::type s_lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long task = (long long)blockIdx.y * kLpGridRows + blockIdx.x;
  if (task >= (long long)P.rows * P.splits) return;  // the whole workgroup
  const size_t row = (size_t)(task / P.splits);
  const int split = (int)(task - (long long)row * P.splits);
  const T* z = (const T*)P.logits + row * (size_t)P.row_stride;
  const LpPart w = lp_part(z, P.V, split, P.splits);
  const u32x4_t* vp = (const u32x4_t*)(z + w.first);

  u32x4_t cur[kLpVecs];
  auto load = [&](int step, u32x4_t (&v)[kLpVecs]) {
#pragma unroll
    for (int u = 0; u < kLpVecs; ++u) v[u] = __builtin_nontemporal_load(vp + min(step * kLpStep + u * kLpThreads + tid, w.vecs - 1));
  };
  if (w.steps > 0) load(0, cur);
  const float c = lp_scale(P, row);
  const int token = P.tokens ? P.tokens[row] : -1;
  const bool known = token >= 0 && token < P.V;
  const float z_t = known ? to_f32<T>(z[token]) : 0.f;

  LpSums mine = {-INFINITY, 0.0, 0.0};
  float col = -INFINITY;
  float neg = 0.f;  // minus the reference
  bool far = false;
  // takes elements into the running sums (top: their maximum)
  auto add = [&](auto& x, float top) {
    constexpr int n = (int)(sizeof(x) / sizeof(float));
    if (top > mine.m) {
      mine = lp_moved(mine, top, c);
      neg = -(mine.m * c);
      far = lp_far(mine.m, c);
    }
    if (far) {
#pragma unroll
      for (int i = 0; i < n; ++i) x[i] -= mine.m;
      neg = 0.f;
    }
    float s[4] = {0.f, 0.f, 0.f, 0.f}, t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float d = fmaf(x[i], c, neg);
      const float e = __builtin_amdgcn_exp2f(d);
      s[i & 3] += e;
      t[i & 3] = fmaf(e, fmaxf(d, kLpFloor), t[i & 3]);
    }
    mine.s += (double)((s[0] + s[1]) + (s[2] + s[3]));
    mine.t += (double)((t[0] + t[1]) + (t[2] + t[3]));
  };

  // one step's elements, the next step's already on their way; kWhole: no vector of the step lies past the part
  auto take = [&](int step, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    float x[kLpVecs * kV];
#pragma unroll
    for (int u = 0; u < kLpVecs; ++u) {
      float y[kV];
      lp_widen<T>(cur[u], y);
      const bool in = kWhole || step * kLpStep + u * kLpThreads + tid < w.vecs;
#pragma unroll
      for (int e = 0; e < kV; ++e) x[u * kV + e] = in ? y[e] : -INFINITY;
    }
    if (step + 1 < w.steps) load(step + 1, cur);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kLpVecs * kV; i += 2) top = fmaxf(fmaxf(x[i], x[i + 1]), top);
    add(x, top);
    if constexpr (kTop) {
      // over the block's eight lanes: neighbours, pairs, then the other four
      top = fmaxf(top, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(top), 0xB1, 0xf, 0xf, true)));
      top = fmaxf(top, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(top), 0x4E, 0xf, 0xf, true)));
      top = fmaxf(top, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(top), 0x141, 0xf, 0xf, true)));
      if (tid % kLpLanes == 0) s_lds.bm[step * kLpGroups + tid / kLpLanes] = top;
      col = fmaxf(col, top);
    }
  };
  for (int step = 0; step < w.steps; ++step) {
    if ((step + 1) * kLpStep <= w.vecs) take(step, std::true_type{});
    else take(step, std::false_type{});
  }
  {  // the elements outside whole vectors: one each for the first threads
    const int before = w.first - w.lo, edges = before + w.hi - w.tail;
    float x[1] = {-INFINITY};
    float top = -INFINITY;
    if (tid < edges) {
      x[0] = to_f32<T>(z[tid < before ? w.lo + tid : w.tail + tid - before]);
      top = fmaxf(x[0], -INFINITY);  // (not a NaN)
      add(x, top);
    }
    if constexpr (kTop) {
      if (wave == 0) {
        top = wave_max(top);
        if (lane == 0) s_lds.bm[kLpBlocks] = top;
      }
      if (tid % kLpLanes == 0) s_lds.col[tid / kLpLanes] = col;
    }
  }

  // ---- the workgroup's sums ------------------------------------------------------------------------------------
  {
    float m = wave_max(mine.m);
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLpWaves; ++i) m = fmaxf(m, s_m[i]);
    mine = lp_moved(mine, m, c);
    const double s = wave_sum(mine.s), t = wave_sum(mine.t);
    if (lane == 0) s_part[wave] = {m, s, t};
  }
  __syncthreads();
  if (tid == 0) {
    LpSums all = s_part[0];
#pragma unroll
    for (int i = 1; i < kLpWaves; ++i) {
      all.s += s_part[i].s;
      all.t += s_part[i].t;
    }
    if (P.splits == 1) s_lse2 = lp_finish(P, row, all, c, z_t, known);
    else P.parts[task] = LogprobPart{all.s, all.t, all.m, 0.f};
  }
  if constexpr (kTop) {
    if (P.splits > 1) {
      unsigned long long* keys = P.keys + (size_t)task * P.n_top;
      lp_select(z, w, P.n_top, s_lds, [&](int rank, unsigned long long k) { keys[rank] = k; });
    } else {
      lp_select(z, w, P.n_top, s_lds, [&](int rank, unsigned long long k) {
        const double base = s_lse2;  // (the selection has barriers of its own)
        const float v = lp_value((unsigned)(k >> 32));
        const size_t at = row * P.n_top + rank;
        P.top_ids[at] = k ? (int32_t)(0xffffffffu - (unsigned)k) : -1;
        P.top_logprobs[at] = k && v > -INFINITY ? (float)(kLpLn2 * ((double)v * (double)c - base)) : -INFINITY;
      });
    }
  }
}

// Joins the parts of a row, one workgroup each.  The parts' lists are sorted, so with more parts than alternatives the n-th largest
// of their heads is a bound again, and few of their keys reach it.
constexpr int kLpMergeThreads = 256;
template <typename T>
__global__ __launch_bounds__(kLpMergeThreads) void logprob_merge_kernel(LogprobLaunch P) {
  __shared__ unsigned long long s_key[kLpMaxSplits * kLpMaxTop];
  __shared__ double s_lse2;
  __shared__ int s_n;
  __shared__ unsigned long long s_bound;
  const int tid = threadIdx.x;
  const long long at = (long long)blockIdx.y * kLpGridRows + blockIdx.x;
  if (at >= P.rows) return;
  const size_t row = (size_t)at;
  const float c = lp_scale(P, row);
  const int n = P.n_top, parts = P.splits;
  if (tid < kWave) {
    LpSums x = {-INFINITY, 0.0, 0.0};
    if (tid < parts) {
      const LogprobPart p = P.parts[row * parts + tid];
      x = {p.m, p.s, p.t};
    }
    const float m = wave_max(x.m);
    x = lp_moved(x, m, c);
    const double s = wave_sum(x.s), t = wave_sum(x.t);
    if (n > 0) {
      const unsigned long long head = tid < parts ? P.keys[(row * parts + tid) * n] : 0ull;
      int above = 0;
      for (int i = 0; i < parts; ++i) {
        const unsigned long long other = (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(head >> 32), i) << 32 |
                                         (unsigned)__builtin_amdgcn_readlane((int)head, i);
        above += other > head;
      }
      if (tid == 0) { s_n = 0; s_bound = 0; }
      if (above == n - 1 && head) s_bound = head;  // (keys are distinct)
    }
    if (tid == 0) {
      const int token = P.tokens ? P.tokens[row] : -1;
      const bool known = token >= 0 && token < P.V;
      const float z_t = known ? to_f32<T>(((const T*)P.logits)[row * (size_t)P.row_stride + token]) : 0.f;
      s_lse2 = lp_finish(P, row, {m, s, t}, c, z_t, known);
    }
  }
  if (n == 0) return;
  __syncthreads();
  for (int i = tid; i < parts * n; i += kLpMergeThreads) {
    const unsigned long long k = P.keys[row * parts * n + i];
    if (k && k >= s_bound) s_key[atomicAdd(&s_n, 1)] = k;
  }
  __syncthreads();
  const int count = s_n;
  const double base = s_lse2;
  for (int i = tid; i < count; i += kLpMergeThreads) {
    const unsigned long long k = s_key[i];
    int rank = 0;
    for (int j = 0; j < count; ++j) rank += s_key[j] > k;
    if (rank < n) {
      const float v = lp_value((unsigned)(k >> 32));
      P.top_ids[row * n + rank] = (int32_t)(0xffffffffu - (unsigned)k);
      P.top_logprobs[row * n + rank] = v > -INFINITY ? (float)(kLpLn2 * ((double)v * (double)c - base)) : -INFINITY;
    }
  }
  for (int i = count + tid; i < n; i += kLpMergeThreads) {
    P.top_ids[row * n + i] = -1;
    P.top_logprobs[row * n + i] = -INFINITY;
  }
}

// ---- backward: elementwise, one read and one write ----------------------------------------------------------------------
constexpr int kLpBackThreads = 256;
constexpr int kLpBackVecs = 4;
template <typename T>
__global__ __launch_bounds__(kLpBackThreads) void logprob_backward_kernel(LogprobLaunch P) {
  constexpr int kV = LpType<T>::kV;
  const int tid = threadIdx.x;
  const long long task = (long long)blockIdx.y * kLpGridRows + blockIdx.x;
  if (task >= (long long)P.rows * P.splits) return;
  const size_t row = (size_t)(task / P.splits);
  const int split = (int)(task - (long long)row * P.splits);
  const T* z = (const T*)P.logits + row * (size_t)P.row_stride;
  T* g = (T*)P.grad + row * (size_t)P.row_stride;
  const LpPart w = lp_part(z, P.V, split, P.splits);
  const u32x4_t* vp = (const u32x4_t*)(z + w.first);

  const float inv_t = 1.f / lp_temperature(P, row);
  const float lse = P.lse[row];
  const bool any = !(lse == -INFINITY);
  const int token = P.tokens ? P.tokens[row] : -1;
  const float gl = any && P.dlogprob && token >= 0 && token < P.V ? P.dlogprob[row] * inv_t : 0.f;
  const float gh = any && P.dentropy ? P.dentropy[row] * inv_t : 0.f;
  // dz = p (a - g_H log p) + [v = t] g_l, log p held between the floor and 0 (a row's NaN is in a)
  const float a = lse != lse ? lse : -fmaf(gh, P.dentropy ? P.entropy[row] : 0.f, gl);
  const float neg = any ? -lse : 0.f;
  auto one = [&](float x) {
    const float l = __builtin_amdgcn_fmed3f(fmaf(x, inv_t, neg), kLpFloor, 0.f);
    return __builtin_amdgcn_exp2f(l * kLpLog2e) * fmaf(-gh, l, a);
  };

  for (int v0 = 0; v0 < w.vecs; v0 += kLpBackThreads * kLpBackVecs) {
    u32x4_t raw[kLpBackVecs];
#pragma unroll
    for (int u = 0; u < kLpBackVecs; ++u) raw[u] = __builtin_nontemporal_load(vp + min(v0 + u * kLpBackThreads + tid, w.vecs - 1));
#pragma unroll
    for (int u = 0; u < kLpBackVecs; ++u) {
      const int vec = v0 + u * kLpBackThreads + tid;
      if (vec >= w.vecs) break;
      float x[kV];
      lp_widen<T>(raw[u], x);
      const int id = w.first + vec * kV;
#pragma unroll
      for (int e = 0; e < kV; ++e) x[e] = one(x[e]);
      if ((unsigned)(token - id) < (unsigned)kV) {  // one vector of the row (g_l is 0 where there is no token)
#pragma unroll
        for (int e = 0; e < kV; ++e) x[e] += id + e == token ? gl : 0.f;
      }
      u32x4_t o;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) o[i] = __float_as_uint(x[i]);
        else o[i] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2_t{x[2 * i], x[2 * i + 1]}), bf16x2_t));
      }
      if (P.wide) {
        __builtin_nontemporal_store(o, (u32x4_t*)(g + id));
      } else {  // the gradient's rows start elsewhere within 16 bytes than the logits'
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (sizeof(T) == 4) {
            ((uint32_t*)g)[id + i] = o[i];
          } else {
            ((uint16_t*)g)[id + 2 * i] = (uint16_t)o[i];
            ((uint16_t*)g)[id + 2 * i + 1] = (uint16_t)(o[i] >> 16);
          }
        }
      }
    }
  }
  const int before = w.first - w.lo, edges = before + w.hi - w.tail;
  if (tid < edges) {
    const int id = tid < before ? w.lo + tid : w.tail + tid - before;
    g[id] = from_f32<T>(one(to_f32<T>(z[id])) + (id == token ? gl : 0.f));
  }
}

// ---- launches -----------------------------------------------------------------------------------------------------------
// Workgroups per row: one where the rows fill the chip (256 compute units, several workgroups each), else as many as do, of no less than
// two steps; and never more than a workgroup's block maxima allow.
int logprob_splits(int64_t rows, int V, bool bf16) {
  const int per_vec = bf16 ? 8 : 4;
  const int64_t vecs = V / per_vec;
  const int64_t least = (vecs + (int64_t)kLpStep * kLpMaxSteps - 1) / ((int64_t)kLpStep * kLpMaxSteps);
  int64_t want = rows >= 1024 ? 1 : (1279 + rows) / std::max<int64_t>(rows, 1);
  want = std::min<int64_t>(want, vecs / (2 * kLpStep));
  want = std::min<int64_t>(want, kLpMaxSplits);
  return (int)std::max<int64_t>(std::max<int64_t>(want, least), 1);
}
int logprob_max_top() { return kLpMaxTop; }
int logprob_max_vocab() { return kLpMaxSplits * kLpMaxSteps * kLpStep * 4; }

template <typename T>
static hipError_t launch_logprob_t(const LogprobLaunch& P, hipStream_t st) {
  const int64_t tasks = (int64_t)P.rows * P.splits;
  auto grid = [](int64_t n) { return dim3((unsigned)std::min<int64_t>(n, kLpGridRows), (unsigned)((n + kLpGridRows - 1) / kLpGridRows)); };
  if (P.n_top > 0) hipLaunchKernelGGL((logprob_rows_kernel<T, true>), grid(tasks), dim3(kLpThreads), 0, st, P);
  else hipLaunchKernelGGL((logprob_rows_kernel<T, false>), grid(tasks), dim3(kLpThreads), 0, st, P);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || P.splits == 1) return e;
  hipLaunchKernelGGL(logprob_merge_kernel<T>, grid(P.rows), dim3(kLpMergeThreads), 0, st, P);
  return hipGetLastError();
}
hipError_t launch_logprob(const LogprobLaunch& P, hipStream_t st) {
  return P.bf16 ? launch_logprob_t<bf16_t>(P, st) : launch_logprob_t<float>(P, st);
}

hipError_t launch_logprob_backward(const LogprobLaunch& P0, hipStream_t st) {
  LogprobLaunch P = P0;
  const int64_t vecs = P.V / (P.bf16 ? 8 : 4);
  // a workgroup takes about four rounds of its loads
  P.wide = (((uintptr_t)P.grad ^ (uintptr_t)P.logits) & 15) == 0;
  P.splits = (int)std::max<int64_t>(1, std::min<int64_t>((vecs + 4095) / 4096, 4096));
  const int64_t tasks = (int64_t)P.rows * P.splits;
  const dim3 grid((unsigned)std::min<int64_t>(tasks, kLpGridRows), (unsigned)((tasks + kLpGridRows - 1) / kLpGridRows));
  if (P.bf16) hipLaunchKernelGGL(logprob_backward_kernel<bf16_t>, grid, dim3(kLpBackThreads), 0, st, P);
  else hipLaunchKernelGGL(logprob_backward_kernel<float>, grid, dim3(kLpBackThreads), 0, st, P);
  return hipGetLastError();
}

}  // namespace aurora
