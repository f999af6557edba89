// Log probabilities of given tokens, entropy and the largest alternatives of every row of logits (paper appendix A.1, eq. 4: the
// logits of a step), and the gradient of the first two.  With x = z / T:
//
//   lse = log sum_v e^x_v     logprob = x_t - lse     H = lse - sum_v p_v x_v     p_v = e^(x_v - lse)
//   dz_v = [ g_l (delta_vt - p_v) - g_H p_v (log p_v + H) ] / T
//
// Forward: bound by the one read of the logits.  A thread keeps a logit m near the largest so far, the reference r of it, s = sum e^(x - r) and
// t = sum (x - r) e^(x - r), in units of log 2, so that H = log s - t / s takes no second pass; moving the reference by d turns (s, t)
// into (s, t + d s) 2^d.  Sixteen or 32 elements are summed in 32 bits at a time, their sums in 64: a row may have a million
// entries.  r is the value that was really subtracted, rounded as it is, and the outputs are formed from it, so that its rounding
// cancels.  Logits so large that its rounding would not be small (a mask's value, and nothing else left) are subtracted first.
// A row goes to one workgroup where there are many; few rows are split, and a second launch joins the parts.
//
// Alternatives ride in the same pass at two lane exchanges and one LDS write per 64 (16-bit: 128) elements: the maximum of every such
// block of the row, and of 64 columns of blocks.  The n-th largest column maximum is a lower bound on the n-th largest element, and
// only blocks that reach it are read again - little more than n of a thousand, most often.  What they hold at or above the bound is a
// short list, ranked by counting.  A row where it is not short (long runs of equal values, a mask that leaves less than n, values that
// rise along the row) takes bounded steps more: the n-th largest block maximum, the exact n-th largest of the blocks above it, and equal
// values in the order of their ids.
//
// The logits are read with loads that do not stay in the caches, unless a gradient is likely to follow (kLpKeepBytes): 4096 x 32000 fp32
// 126 -> 80 us = 6.5 TB/s, what a read of memory gives; 1280 x 200064 bf16 with eight alternatives 87 us = 5.9.  The gradient: 4096 x 32000
// fp32 201 us (171 after a forward that left logits in the caches), 1024 x 128256 bf16 100 = 5.2 TB/s, as a device copy.
//
// Rows cut into parts with alternatives are further from it: 160 x 128256 fp32 with twenty 21 us and 4 for the merge, where the read takes
// 12.4; 160 x 151936 bf16 26 in all, where it takes 7.4.  A part is loaded whole, then summed, then searched: 20 vector instructions an
// element, to the streaming kernel's 10 (fp32, without alternatives) or 8 (bf16, with), and after the read rather than under it.  Nor do all
// parts start together: 113 registers hold 1024 workgroups of the first call's 1280, 138 hold 768 of the second's 800.  Short rows are a chain each -
// load, two 64-bit sums, a logarithm - in a wavefront that has nothing of its next row on the way (60000 x 777 fp32 49 us, the read 28); with
// alternatives the blocks that hold one are read from memory again, and listed in LDS (96).
#include "launch.hpp"

#include <float.h>

#include <algorithm>
#include <type_traits>

namespace aurora {

constexpr int kLpVecs = 4;  // 16-byte vectors of a thread in one step
// What a workgroup of kT threads takes: a step is kT * kLpVecs vectors of the row; a block is the kLanes lanes' vectors of one step, and
// the same lanes' blocks of all steps are one of 64 columns.
template <int kT>
struct LpShape {
  static constexpr int kThreads = kT, kWaves = kT / kWave;
  static constexpr int kStep = kT * kLpVecs;
  static constexpr int kColumns = kWave, kLanes = kT / kColumns;
  static constexpr int kMaxSteps = kT == 256 ? 64 : 16;  // bounds the block maxima in LDS
  static constexpr int kBlocks = kMaxSteps * kColumns;   // and one for the elements outside whole vectors
  static constexpr int kList = kT == 256 ? 512 : 256;    // elements, and blocks, that are ranked by counting
};
typedef LpShape<256> LpWide;    // long rows
typedef LpShape<64> LpNarrow;   // short rows: a wavefront each
constexpr int kLpMaxTop = 32;
constexpr int kLpMaxSplits = 64;
constexpr float kLpLog2e = 1.4426950408889634f;
constexpr double kLpLn2 = 0.69314718055994530942;
constexpr float kLpFloor = -256.f;  // stands in for -inf times zero: 2^-256 is zero as well (and 256 times a gradient no infinity)
// The reference only moves when a logit is so many bits above it: exponentials stay below 2^8, as exact as below 1, and the move - 60
// instructions, of which some lane of a wavefront has need in nearly every step if every new maximum counts - becomes rare.
constexpr float kLpLazyBits = 8.f;
constexpr int kLpGridRows = 1 << 22;

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// the largest, and the smallest, of three as they were loaded (fmaxf would first make quiet numbers of them, an instruction each)
__device__ __forceinline__ float lp_max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

__device__ __forceinline__ float lp_min3(float a, float b, float c) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// 16 bytes that are needed once (past the caches), or soon again
template <bool kKeep>
__device__ __forceinline__ u32x4_t lp_load(const u32x4_t* p) {
  if constexpr (kKeep) return *p;
  else return __builtin_nontemporal_load(p);
}

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
struct LpPart { int lo, first, vecs, tail, hi; };
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
  return p;
}

// What is subtracted for the reference m: its rounded multiple, or, past kLpFar / c, m itself before the product - there the rounding
// alone would be a sixteenth and more (at 10^10 it is 512, and every exponential zero, or infinite).  Past kLpLimit a product may overflow.
constexpr float kLpFar = 0x1p20f, kLpLimit = 8.5e37f;
__device__ __forceinline__ bool lp_far(float m, float c) { return fabsf(m) * c > kLpFar; }
__device__ __forceinline__ double lp_ref(float m, float c) { return lp_far(m, c) ? (double)m * (double)c : (double)(m * c); }

// reductions over a wavefront by data-parallel moves: within rows of sixteen, then across; every lane gets the result
template <int kCtl, int kRows>
__device__ __forceinline__ float lp_max_step(float v) {
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp((int)0xff800000u, __float_as_int(v), kCtl, kRows, 0xf, false)));
}
__device__ __forceinline__ float lp_wave_max(float v) {
  v = lp_max_step<0x111, 0xf>(v);
  v = lp_max_step<0x112, 0xf>(v);
  v = lp_max_step<0x114, 0xf>(v);
  v = lp_max_step<0x118, 0xf>(v);
  v = lp_max_step<0x142, 0xa>(v);
  v = lp_max_step<0x143, 0xc>(v);
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
template <int kCtl, int kRows>
__device__ __forceinline__ double lp_sum_step(double v) {
  const long long b = __double_as_longlong(v);
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)b, kCtl, kRows, 0xf, false);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), kCtl, kRows, 0xf, false);
  return v + __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double lp_wave_sum(double v) {
  v = lp_sum_step<0x111, 0xf>(v);
  v = lp_sum_step<0x112, 0xf>(v);
  v = lp_sum_step<0x114, 0xf>(v);
  v = lp_sum_step<0x118, 0xf>(v);
  v = lp_sum_step<0x142, 0xa>(v);
  v = lp_sum_step<0x143, 0xc>(v);
  const long long b = __double_as_longlong(v);
  return __longlong_as_double((long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(b >> 32), 63) << 32 |
                                          (unsigned)__builtin_amdgcn_readlane((int)b, 63)));
}

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
    if (known) lp = none ? -INFINITY : (float)(kLpLn2 * ((double)z_t * (double)c - r - l2));  // (a masked token's -inf, or the row's NaN)
    P.logprob[row] = lp;
  }
  return r + l2;
}

__device__ __forceinline__ float lp_temperature(const LogprobLaunch& P, size_t row) {
  const float T = P.temperatures ? P.temperatures[(unsigned)row / (unsigned)P.temperature_rows] : P.temperature;
  return T > 0.f ? fminf(fmaxf(T, FLT_MIN), FLT_MAX) : 1.f;  // (its reciprocal is finite, and not zero)
}
__device__ __forceinline__ float lp_scale(const LogprobLaunch& P, size_t row) { return kLpLog2e / lp_temperature(P, row); }

// how many of the list are larger, eight reads at a time (one at a time each waits for the last: 256 keys 12 us)
constexpr int kLpRankStep = 8;
__device__ __forceinline__ int lp_rank(const unsigned long long* list, int count, unsigned long long k) {
  int rank = 0;
  for (int j = 0; j < count; j += kLpRankStep) {
    unsigned long long other[kLpRankStep];
#pragma unroll
    for (int e = 0; e < kLpRankStep; ++e) other[e] = list[j + e];
#pragma unroll
    for (int e = 0; e < kLpRankStep; ++e) rank += other[e] > k;
  }
  return rank;
}

// ---- selection of the n largest of a workgroup's part -------------------------------------------------------------------
template <typename S>
struct LpLds {
  float bm[S::kBlocks + 1];           // block maxima; the last one is of the elements outside whole vectors
  float col[S::kColumns];             // and the maxima of their columns
  unsigned short blocks[S::kList];
  unsigned long long list[S::kList + kLpRankStep];  // (zeros behind the last)
  int cnt[16][4];
  int n_blocks, n_list;
  int best[S::kWaves];
};

// The largest bound that at least n of `count` values reach (value(i): an lp_order key, or 0 for none): two bits at a time from the top.
// 0 if there are fewer than n.
template <typename S, typename Value>
__device__ __forceinline__ unsigned lp_nth(int count, int n, LpLds<S>& L, Value value) {
  const int tid = threadIdx.x, lane = tid & 63;
  __syncthreads();
  if (tid < 64) L.cnt[tid >> 2][tid & 3] = 0;
  __syncthreads();
  unsigned p = 0;
#pragma unroll 1
  for (int step = 0; step < 16; ++step) {
    const int sh = 30 - 2 * step;
    int c[3] = {0, 0, 0};
#pragma unroll 1
    for (int i = tid; i - tid < count; i += S::kThreads) {
      const unsigned v = i < count ? value(i) : 0u;
#pragma unroll
      for (int q = 0; q < 3; ++q) c[q] += __popcll(__ballot(v >= (p | (unsigned)(q + 1) << sh)));
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
template <typename S, typename T>
__device__ __forceinline__ bool lp_element(const T* row, const LpPart& w, int blk, int i, int& id, float& z) {
  constexpr int kV = LpType<T>::kV;
  if (blk == S::kBlocks) {  // outside whole vectors
    const int before = w.first - w.lo;
    id = i < before ? w.lo + i : w.tail + i - before;
    if (i >= before + w.hi - w.tail) return false;
  } else {
    const int step = blk / S::kColumns, lane = (blk % S::kColumns) * S::kLanes + (i / kV) % S::kLanes;
    const int vec = step * S::kStep + i / (kV * S::kLanes) * S::kThreads + lane;
    if (vec >= w.vecs) return false;
    id = w.first + vec * kV + i % kV;
  }
  z = to_f32<T>(row[id]);
  return true;
}

// Lists what the blocks in L.blocks hold above the bound (or at it, with_ties), a vector a thread at a time; stops once the list is past
// its size.  Returns how many there are, S::kList + 1 if too many.
template <typename S, typename T>
__device__ __forceinline__ int lp_gather(const T* row, const LpPart& w, unsigned bound, bool with_ties, LpLds<S>& L) {
  constexpr int kV = LpType<T>::kV, kPer = S::kLanes * kLpVecs;
  __syncthreads();
  if (threadIdx.x == 0) L.n_list = 0;
  __syncthreads();
  auto offer = [&](float z, int id) {
    const unsigned o = lp_order(z);
    if (o > bound || (with_ties && o == bound)) {
      const int at = atomicAdd(&L.n_list, 1);
      if (at < S::kList) L.list[at] = lp_key(z, id);
    }
  };
  if (L.n_blocks > S::kList) return S::kList + 1;
  const int all = L.n_blocks * kPer;
  constexpr int kBatch = 4;  // loads of a thread on their way together
  for (int i0 = threadIdx.x; i0 < all; i0 += kBatch * S::kThreads) {
    if (*(volatile int*)&L.n_list > S::kList) break;
    u32x4_t raw[kBatch];
    int ids[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = i0 + k * S::kThreads;
      ids[k] = -1;
      if (i >= all) continue;
      const int blk = L.blocks[i / kPer], u = i % kPer;
      if (blk == S::kBlocks) {  // outside whole vectors: less than a vector's elements before, and after them
        for (int e = u; e < 2 * kV; e += kPer) {
          int id;
          float z;
          if (lp_element<S>(row, w, blk, e, id, z)) offer(z, id);
        }
        continue;
      }
      const int vec = blk / S::kColumns * S::kStep + u / S::kLanes * S::kThreads + blk % S::kColumns * S::kLanes + u % S::kLanes;
      if (vec >= w.vecs) continue;
      ids[k] = w.first + vec * kV;
      raw[k] = *(const u32x4_t*)(row + ids[k]);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (ids[k] < 0) continue;
      float x[kV];
      lp_widen<T>(raw[k], x);
#pragma unroll
      for (int e = 0; e < kV; ++e) offer(x[e], ids[k] + e);
    }
  }
  __syncthreads();
  return min(L.n_list, S::kList + 1);
}

// lists the blocks whose maximum reaches the bound (above: is above it)
template <typename S>
__device__ __forceinline__ void lp_blocks(int steps, unsigned bound, bool above, LpLds<S>& L) {
  __syncthreads();
  if (threadIdx.x == 0) L.n_blocks = 0;
  __syncthreads();
  for (int i = threadIdx.x; i <= steps * S::kColumns; i += S::kThreads) {
    const int blk = i < steps * S::kColumns ? i : S::kBlocks;
    const unsigned o = lp_order(L.bm[blk]);
    if (above ? o > bound : o >= bound) {
      const int at = atomicAdd(&L.n_blocks, 1);
      if (at < S::kList) L.blocks[at] = (unsigned short)blk;
    }
  }
  __syncthreads();
}

// The n-th largest column maximum, or a little less: as good a bound for most rows, and a wavefront finds it by counting, without a barrier.
template <typename S>
__device__ __forceinline__ unsigned lp_column_bound(int n, const LpLds<S>& L) {
  static_assert(S::kColumns == kWave && S::kColumns >= kLpMaxTop, "a column a lane");
  const int lane = threadIdx.x & 63;
  const unsigned mine = (lp_order(L.col[lane]) & ~63u) | lane;  // (distinct)
  int above = 0;
#pragma unroll
  for (int i = 0; i < S::kColumns; ++i) above += (unsigned)__builtin_amdgcn_readlane(mine, i) > mine;
  return __builtin_amdgcn_readlane(mine, __ffsll((unsigned long long)__ballot(above == n - 1)) - 1) & ~63u;
}

// The n largest of the part, by value and then by id, to out(rank, key): every rank below n is given, key 0 where there is none.  The list
// holds the `count` elements that reach the bound (past its size: more than it takes).
template <typename S, typename T, typename Out>
__device__ __forceinline__ void lp_select(const T* row, const LpPart& w, int steps, int n, unsigned bound, int count, LpLds<S>& L, Out out) {
  constexpr int kV = LpType<T>::kV, kBlock = kV * S::kLanes * kLpVecs;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  bool ties = false;  // the equal ones are still to be found
  if (count > S::kList) {
    // The n-th largest block maximum is closer, and less than n blocks are above it.
    const int used = steps * S::kColumns;
    bound = lp_nth<S>(used + 1, n, L, [&](int i) { return lp_order(L.bm[i < used ? i : S::kBlocks]); });
    lp_blocks<S>(steps, bound, true, L);
    count = lp_gather<S>(row, w, bound, false, L);
    ties = true;
    if (count > S::kList) {
      // They hold more than the list: the n-th largest element is among theirs.
      bound = lp_nth<S>(L.n_blocks * kBlock, n, L, [&](int i) {
        int id;
        float z;
        return lp_element<S>(row, w, L.blocks[i / kBlock], i % kBlock, id, z) ? lp_order(z) : 0u;
      });
      count = lp_gather<S>(row, w, bound, true, L);
      ties = count > S::kList;
      if (ties) count = lp_gather<S>(row, w, bound, false, L);
    }
  }
  if (tid < kLpRankStep) L.list[count + tid] = 0;
  __syncthreads();
  for (int i = tid; i < count; i += S::kThreads) {
    const unsigned long long k = L.list[i];
    const int rank = lp_rank(L.list, count, k);
    if (rank < n) out(rank, k);
  }
  int have = min(count, n);
  if (ties && have < n) {
    // Equal values in the order of their ids: the row's pieces in order, in each the lowest id not yet taken.  A thread's equal elements of
    // a piece are bits, in the order of their ids.
    static_assert(kLpVecs * kV <= 32, "a bit an element");
    const float at = lp_value(bound);
    for (int piece = -1; piece <= steps && have < n; ++piece) {
      const bool outside = piece < 0 || piece == steps;  // the elements before, and after, the vectors
      const int first = outside ? (piece < 0 ? w.lo : w.tail) + tid : w.first + (piece * S::kStep + tid) * kV;
      unsigned equal = 0;
      if (outside) {
        equal = first < (piece < 0 ? w.first : w.hi) && to_f32<T>(row[first]) == at ? 1u : 0u;
      } else {
#pragma unroll
        for (int u = 0; u < kLpVecs; ++u) {
          if (piece * S::kStep + u * S::kThreads + tid >= w.vecs) break;
          float x[kV];
          lp_widen<T>(*(const u32x4_t*)(row + first + u * S::kThreads * kV), x);
#pragma unroll
          for (int e = 0; e < kV; ++e) equal |= x[e] == at ? 1u << (u * kV + e) : 0u;
        }
      }
      while (have < n) {
        const int bit = __ffs(equal) - 1, mine = equal ? first + bit / kV * S::kThreads * kV + bit % kV : INT32_MAX;
        int low = wave_min(mine);
        __syncthreads();
        if (lane == 0) L.best[wave] = low;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < S::kWaves; ++i) low = min(low, L.best[i]);
        if (low == INT32_MAX) break;
        if (mine == low) {
          out(have, lp_key(at, low));
          equal &= equal - 1;
        }
        ++have;
      }
    }
  }
  for (int i = have + tid; i < n; i += S::kThreads) out(i, 0ull);
}

// ---- forward --------------------------------------------------------------------------------------------------------------
// kHeld: the part is at most so many steps long (P.splits sees to that): all of it is on its way at once and stays in registers, so
// that a selection reads nothing again.  0: a step at a time, the next one on its way.
template <typename T, typename S, bool kTop, int kHeld, bool kKeep>
__global__ __launch_bounds__(S::kThreads) void logprob_rows_kernel(LogprobLaunch P) {
  constexpr int kV = LpType<T>::kV;
  __shared__ LpSums s_part[S::kWaves];
  __shared__ float s_m[S::kWaves];
  __shared__ double s_lse2;
  __shared__ typename std::conditional<kTop, LpLds<S>, int>::type s_lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const unsigned task = blockIdx.y * (unsigned)kLpGridRows + blockIdx.x;
  if (task >= (unsigned)P.rows * (unsigned)P.splits) return;  // the whole workgroup
  const size_t row = task / (unsigned)P.splits;
  const int split = task % (unsigned)P.splits;
  const T* z = (const T*)P.logits + row * (size_t)P.row_stride;
  const LpPart w = lp_part(z, P.V, split, P.splits);
  const int steps = (w.vecs + S::kStep - 1) / S::kStep;
  const u32x4_t* vp = (const u32x4_t*)(z + w.first);

  // Two elements a word are twice the instructions a byte: 16-bit rows are near the vector units' limit (1280 x 200064: 97 % busy with
  // 10.7 instructions an element, 81 % now with 8.4), so that two buffers that need no moves, and one test a step in place of one
  // an element, pay.  fp32 rows are slower for both (4096 x 32000 83 -> 87 us: 144 registers), and so are short rows, a wavefront each,
  // which wait more than they work: the more of them at a time, the better (60000 x 777 bf16 50 us, 69 with 105 registers for 79).
  constexpr bool kTight = sizeof(T) == 2 && S::kThreads > kWave;
  u32x4_t cur[kHeld > 0 ? kHeld : kTight ? 2 : 1][kLpVecs];
  auto load = [&](int step, u32x4_t (&v)[kLpVecs]) {
#pragma unroll
    for (int u = 0; u < kLpVecs; ++u) v[u] = lp_load<kKeep>(vp + min(step * S::kStep + u * S::kThreads + tid, w.vecs - 1));
  };
  if constexpr (kHeld > 0) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (i < steps) load(i, cur[i]);
  } else {
    if (steps > 0) load(0, cur[0]);
  }
  const float c = lp_scale(P, row);
  const int token = P.tokens ? P.tokens[row] : -1;
  const bool known = token >= 0 && token < P.V;
  const float z_t = known ? to_f32<T>(z[token]) : 0.f;

  LpSums mine = {-INFINITY, 0.0, 0.0};
  float col = -INFINITY;
  float neg = 0.f;  // minus the reference
  const float lazy = fminf(kLpLazyBits / c, FLT_MAX), lowest = -kLpLimit / c;  // (at most -inf, which `low` may be too)
  bool far = false;
  // takes elements into the running sums (top, low: the largest and the smallest).  0 times -inf must not get into t: where there is
  // one, or a value whose x would be, distances stop at the floor.
  auto sums = [&](const auto& x, auto floor) {
    constexpr int n = (int)(sizeof(x) / sizeof(float));
    float s[4] = {0.f, 0.f, 0.f, 0.f}, t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float d = fmaf(x[i], c, neg);
      const float e = __builtin_amdgcn_exp2f(d);
      s[i & 3] += e;
      t[i & 3] = fmaf(e, decltype(floor)::value ? fmaxf(d, kLpFloor) : d, t[i & 3]);
    }
    mine.s += (double)((s[0] + s[1]) + (s[2] + s[3]));
    mine.t += (double)((t[0] + t[1]) + (t[2] + t[3]));
  };
  auto add = [&](auto& x, float top, float low) {
    constexpr int n = (int)(sizeof(x) / sizeof(float));
    if (top > mine.m + lazy) {
      asm volatile("");  // (what follows is rare: not to be worked out ahead of the test)
      mine = lp_moved(mine, top, c);
      neg = -(mine.m * c);
      far = lp_far(mine.m, c);
    }
    if (far) {
      asm volatile("");
#pragma unroll
      for (int i = 0; i < n; ++i) x[i] -= mine.m;
      neg = 0.f;
    }
    if (!kTight || far || low <= lowest) sums(x, std::true_type{});
    else sums(x, std::false_type{});
  };

  // one step's elements, the next step's already on their way; kWhole: no vector of the step lies past the part
  float tops[kHeld > 0 ? kHeld : 1];  // a held step's maximum
  auto take = [&](int step, u32x4_t (&v)[kLpVecs], u32x4_t (&next)[kLpVecs], float& held_top, auto whole, auto vecs) {
    constexpr bool kWhole = decltype(whole)::value;
    constexpr int kVecs = decltype(vecs)::value;  // that the step has at most
    float x[kVecs * kV];
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      float y[kV];
      lp_widen<T>(v[u], y);
      const bool in = kWhole || step * S::kStep + u * S::kThreads + tid < w.vecs;
#pragma unroll
      for (int e = 0; e < kV; ++e) x[u * kV + e] = in ? y[e] : -INFINITY;
    }
    if (kHeld == 0 && step + 1 < steps) load(step + 1, next);
    float top = -INFINITY, low = INFINITY;
#pragma unroll
    for (int i = 0; i < kVecs * kV; i += 2) {
      top = lp_max3(x[i], x[i + 1], top);
      if (kTight) low = lp_min3(x[i], x[i + 1], low);
    }
    held_top = top;
    add(x, top, low);
    if constexpr (kTop) {
      if constexpr (S::kLanes > 1) {  // over the block's four lanes: neighbours, then pairs
        static_assert(S::kLanes == 4 || S::kLanes == 1, "");
        top = fmaxf(top, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(top), 0xB1, 0xf, 0xf, true)));
        top = fmaxf(top, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(top), 0x4E, 0xf, 0xf, true)));
      }
      if (tid % S::kLanes == 0) s_lds.bm[step * S::kColumns + tid / S::kLanes] = top;
      col = fmaxf(col, top);
    }
  };
  constexpr std::integral_constant<int, kLpVecs> all;
  if constexpr (kHeld > 0) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      tops[i] = -INFINITY;
      if (i >= steps) continue;
      if ((i + 1) * S::kStep <= w.vecs) take(i, cur[i], cur[i], tops[i], std::true_type{}, all);
      else take(i, cur[i], cur[i], tops[i], std::false_type{}, all);
    }
  } else {
    const int whole = w.vecs / S::kStep;
    int step = 0;
    constexpr int kOther = kTight ? 1 : 0;
    // A short row's last step, which may be all of it, is worked out no further than it goes (60000 x 300 fp32 42 -> 37 us).
    auto last = [&](u32x4_t (&v)[kLpVecs]) {
      const int rest = w.vecs - whole * S::kStep;
      if (S::kThreads == kWave && rest <= S::kThreads) take(whole, v, v, tops[0], std::false_type{}, std::integral_constant<int, 1>{});
      else if (S::kThreads == kWave && rest <= 2 * S::kThreads) take(whole, v, v, tops[0], std::false_type{}, std::integral_constant<int, 2>{});
      else take(whole, v, v, tops[0], std::false_type{}, all);
    };
    if (!kTight)
      for (; step < whole; ++step) take(step, cur[0], cur[0], tops[0], std::true_type{}, all);
    for (; kTight && step + 1 < whole; step += 2) {
      take(step, cur[0], cur[kOther], tops[0], std::true_type{}, all);
      take(step + 1, cur[kOther], cur[0], tops[0], std::true_type{}, all);
    }
    if (kTight && step < whole) {
      take(step, cur[0], cur[kOther], tops[0], std::true_type{}, all);
      if (whole < steps) last(cur[kOther]);
    } else if (whole < steps) {
      last(cur[0]);
    }
  }
  int edge;
  float edge_z = 0.f;
  {  // the elements outside whole vectors: one each for the first threads
    const int before = w.first - w.lo, edges = before + w.hi - w.tail;
    float x[1] = {-INFINITY};
    float top = -INFINITY;
    edge = tid < edges ? (tid < before ? w.lo + tid : w.tail + tid - before) : -1;
    if (edge >= 0) {
      x[0] = edge_z = to_f32<T>(z[edge]);
      top = fmaxf(x[0], -INFINITY);  // (not a NaN)
      add(x, top, x[0]);
    }
    if constexpr (kTop) {
      if (wave == 0) {
        top = lp_wave_max(top);
        if (lane == 0) s_lds.bm[S::kBlocks] = top;
      }
      if (tid % S::kLanes == 0) s_lds.col[tid / S::kLanes] = col;
      if (tid == 0) s_lds.n_list = 0;
    }
  }

  // ---- the workgroup's sums ------------------------------------------------------------------------------------
  {
    float m = lp_wave_max(mine.m);
    if (lane == 0) s_m[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::kWaves; ++i) m = fmaxf(m, s_m[i]);
    mine = lp_moved(mine, m, c);
    const double s = lp_wave_sum(mine.s), t = lp_wave_sum(mine.t);
    if (lane == 0) s_part[wave] = {m, s, t};
  }
  __syncthreads();
  if (tid == S::kThreads - 1) {  // (a lane of the last wavefront: the first has the elements outside vectors)
    LpSums all = s_part[0];
#pragma unroll
    for (int i = 1; i < S::kWaves; ++i) {
      all.s += s_part[i].s;
      all.t += s_part[i].t;
    }
    if (P.splits == 1) s_lse2 = lp_finish(P, row, all, c, z_t, known);
    else P.parts[(size_t)task] = LogprobPart{all.s, all.t, all.m, z_t};
  }
  if constexpr (kTop) {
    LpLds<S>& L = s_lds;
    const int n = P.n_top;
    const unsigned bound = lp_column_bound(n, L);
    int count;
    if constexpr (kHeld > 0) {
      const float at_least = fmaxf(lp_value(bound), -INFINITY);  // (below the key of -inf come NaNs)
      auto offer = [&](float v, int id) {
        if (v >= at_least) {
          const int at = atomicAdd(&L.n_list, 1);
          if (at < S::kList) L.list[at] = lp_key(v, id);
        }
      };
      if (edge >= 0) offer(edge_z, edge);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        if (i >= steps || !(tops[i] >= at_least)) continue;
#pragma unroll
        for (int u = 0; u < kLpVecs; ++u) {
          const int vec = i * S::kStep + u * S::kThreads + tid;
          float y[kV], top = -INFINITY;
          lp_widen<T>(cur[i][u], y);
#pragma unroll
          for (int e = 0; e < kV; e += 2) top = lp_max3(y[e], y[e + 1], top);
          if (vec < w.vecs && top >= at_least) {
#pragma unroll
            for (int e = 0; e < kV; ++e) offer(y[e], w.first + vec * kV + e);
          }
        }
      }
      __syncthreads();
      count = min(L.n_list, S::kList + 1);
    } else {
      lp_blocks<S>(steps, bound, false, L);
      count = lp_gather<S>(z, w, bound, true, L);
    }
    if (P.splits > 1) {
      unsigned long long* keys = P.keys + (size_t)task * n;
      lp_select<S>(z, w, steps, n, bound, count, L, [&](int rank, unsigned long long k) { keys[rank] = k; });
    } else {
      lp_select<S>(z, w, steps, n, bound, count, L, [&](int rank, unsigned long long k) {
        const double base = s_lse2;  // (there are barriers in between)
        const float v = lp_value((unsigned)(k >> 32));
        const size_t at = row * n + rank;
        P.top_ids[at] = k ? (int32_t)(0xffffffffu - (unsigned)k) : -1;
        P.top_logprobs[at] = k && v > -INFINITY ? (float)(kLpLn2 * ((double)v * (double)c - base)) : -INFINITY;
      });
    }
  }
}

// Joins the parts of a row, one workgroup each.  The parts' lists are sorted, so with more parts than alternatives the n-th largest
// of their heads is a bound again, and few of their keys reach it.  Bound by latency: everything is loaded at once, and one wavefront
// joins the sums while another looks for the bound.  (A launch of its own: were the last workgroup of a row to do it, what the others hand
// over would have to pass between the dies' caches - 160 rows x 128256 with twenty 24 us so, 37 in one launch.)
constexpr int kLpMergeThreads = 256;
template <typename T>
__global__ __launch_bounds__(kLpMergeThreads) void logprob_merge_kernel(LogprobLaunch P) {
  constexpr int kHeld = 2;  // keys of a thread that are loaded ahead
  __shared__ unsigned long long s_key[kLpMaxSplits * kLpMaxTop + kLpRankStep];
  __shared__ double s_lse2;
  __shared__ int s_n;
  __shared__ unsigned long long s_bound;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long at = (long long)blockIdx.y * kLpGridRows + blockIdx.x;
  if (at >= P.rows) return;
  const size_t row = (size_t)at;
  const int n = P.n_top, parts = P.splits, all = parts * n;
  const unsigned long long* keys = P.keys + row * all;
  unsigned long long held[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = tid + i * kLpMergeThreads < all ? keys[tid + i * kLpMergeThreads] : 0ull;
  const float c = lp_scale(P, row);
  if (wave == 0) {
    LpSums x = {-INFINITY, 0.0, 0.0};
    const int token = P.tokens ? P.tokens[row] : -1;
    const LogprobPart p = P.parts[row * parts + min(lane, parts - 1)];
    if (lane < parts) x = {p.m, p.s, p.t};
    const float m = lp_wave_max(x.m);
    x = lp_moved(x, m, c);
    const double s = lp_wave_sum(x.s), t = lp_wave_sum(x.t);
    if (lane == 0) s_lse2 = lp_finish(P, row, {m, s, t}, c, p.z_t, token >= 0 && token < P.V);
  } else if (wave == 1 && n > 0) {
    // A bound that n keys reach: the n-th largest head of as many parts, or the smallest of all parts' q-th keys, n of them together.
    const int q = (n + parts - 1) / parts;
    const unsigned long long mine = lane < parts ? keys[lane * n + (q - 1)] : ~0ull;
    unsigned long long bound = 0;
    if (q > 1) {
      bound = mine;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor(bound, o, kWave);
        bound = other < bound ? other : bound;
      }
    } else {
      const unsigned long long head = lane < parts ? mine : 0ull;
      int above = 0;
      for (int i = 0; i < parts; ++i) {
        const unsigned long long other = (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(head >> 32), i) << 32 |
                                         (unsigned)__builtin_amdgcn_readlane((int)head, i);
        above += other > head;
      }
      const unsigned long long nth = __ballot(above == n - 1 && head != 0);  // (keys are distinct)
      if (nth) bound = __shfl(head, __ffsll(nth) - 1, kWave);
    }
    if (lane == 0) { s_n = 0; s_bound = bound; }
  }
  if (n == 0) return;
  __syncthreads();
  const unsigned long long bound = s_bound;
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (held[i] && held[i] >= bound) s_key[atomicAdd(&s_n, 1)] = held[i];
  for (int i = tid + kHeld * kLpMergeThreads; i < all; i += kLpMergeThreads) {
    const unsigned long long k = keys[i];
    if (k && k >= bound) s_key[atomicAdd(&s_n, 1)] = k;
  }
  __syncthreads();
  const int count = s_n;
  const double base = s_lse2;
  if (tid < kLpRankStep) s_key[count + tid] = 0;
  __syncthreads();
  for (int i = tid; i < count; i += kLpMergeThreads) {
    const unsigned long long k = s_key[i];
    const int rank = lp_rank(s_key, count, k);
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
template <typename T, bool kKeep>
__global__ __launch_bounds__(kLpBackThreads) void logprob_backward_kernel(LogprobLaunch P) {
  constexpr int kV = LpType<T>::kV;
  const int tid = threadIdx.x;
  const unsigned task = blockIdx.y * (unsigned)kLpGridRows + blockIdx.x;
  if (task >= (unsigned)P.rows * (unsigned)P.splits) return;
  const size_t row = task / (unsigned)P.splits;
  const int split = task % (unsigned)P.splits;
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
    for (int u = 0; u < kLpBackVecs; ++u) raw[u] = lp_load<kKeep>(vp + min(v0 + u * kLpBackThreads + tid, w.vecs - 1));
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
// Workgroups per row: one where the rows fill the chip, and never more than a workgroup's block maxima allow; few rows are cut into parts
// that a workgroup holds in registers.  The merge's launch is the price, the more rows the longer, the gain a row's length: us whole
// and cut, five alternatives, 128256 fp32 (eight parts) 26.3 and 19.5 at 128 rows, 34.6 and 34.0 at 320, 46.5 and 48.2 at 512; 151936 bf16
// (five) 23.8 and 19.5 at 128, 24.5 and 26.4 at 256; 45000 fp32 (three) 12.2 and 11.3 at 80, 13.0 and 13.6 at 144; 32000 fp32 (two)
// 8.3 and 8.7 at one row, 11.2 and 13.3 at 176.  Up to 64 rows leave compute units idle even so: they are cut further, down to one step
// a part, into up to 512 parts in all, where that makes at least eight of a row (five alternatives, parts of four steps and these: 5 x
// 128256 fp32 9.9 and 8.5, 12 x 151936 bf16 12.4 and 9.7, 64 x 64000 fp32 11.8 and 11.1, 5 x 32000 fp32 uncut 9.1, so 8.0, where it makes
// four of a row 5 x 32000 bf16 8.3 and 9.2; in 256 or 1024 parts 64 x 64000 11.7 and 11.6, 64 x 151936 bf16 14.4, 15.8 and 16.8).
constexpr int kLpHeld = 4, kLpHeldRows = 640, kLpCutParts = 3, kLpRowsPerPart = 40;
constexpr int kLpIdleRows = 64, kLpIdleParts = 8;
static int64_t logprob_parts(int V, bool bf16) {
  constexpr int64_t held = (int64_t)LpWide::kStep * kLpHeld;
  const int64_t parts = (V / (bf16 ? 8 : 4) + held - 1) / held;
  return parts >= kLpCutParts && parts <= kLpMaxSplits ? parts : 1;
}
int logprob_few_rows(int V, bool bf16) { return std::min((int)logprob_parts(V, bf16) * kLpRowsPerPart, kLpHeldRows); }
int logprob_splits(int64_t rows, int V, bool bf16) {
  constexpr int64_t most = (int64_t)LpWide::kStep * LpWide::kMaxSteps;
  const int64_t least = (V / (bf16 ? 8 : 4) + most - 1) / most;
  const int64_t steps = std::min<int64_t>((V / (bf16 ? 8 : 4) + LpWide::kStep - 1) / LpWide::kStep, kLpMaxSplits);
  const int64_t cut = rows <= logprob_few_rows(V, bf16) ? logprob_parts(V, bf16) : 1;
  const int64_t most_of_row = kLpIdleRows * kLpIdleParts / std::max<int64_t>(rows, 1);  // (eight or more up to 64 rows)
  return (int)std::max<int64_t>({rows <= kLpIdleRows && steps >= kLpIdleParts ? std::min(steps, most_of_row) : 1, cut, least, 1});
}
int logprob_idle_rows() { return kLpIdleRows; }
int logprob_max_top() { return kLpMaxTop; }
int logprob_max_vocab() { return kLpMaxSplits * LpWide::kMaxSteps * LpWide::kStep * 4; }

// Rows of so few vectors go to a wavefront each where there are many: what a row costs besides its bytes is barriers, the more of them with
// a selection.  us with 256 threads a row and with 64: 60000 rows x 777 fp32 135 and 47, with one alternative 270 and 98; 20000 x 2048 50
// and 29, with five 96 and 43; 10000 x 16001 bf16 with five 96 and 76; 10000 x 8192 fp32 without 53 and 53.
constexpr int kLpNarrowVecs = 1024, kLpNarrowVecsTop = 4096, kLpNarrowRows = 1024;
static_assert(kLpNarrowVecsTop <= LpNarrow::kStep * LpNarrow::kMaxSteps, "a row's block maxima");

// Up to so many bytes of logits are read so that they stay in the caches where a gradient is likely to follow: its logsumexp is wanted,
// and no alternatives.  us, past the caches and so, forward alone and with the gradient: 134 x 32000 fp32 8.2 and 7.0, 20.8 and 18.4;
// 1000 x 32000 22.7 and 25.6, 74.9 and 65.5; 4096 x 32000 80 and 91, 281 and 266; 1024 x 128256 bf16 49 and 54, 146 and 133; from 1 GB on
// nothing is left of the gain (8192 x 32000 fp32 156 and 177, 554 and 553).  The gradient itself reads up to kLpKeepBackBytes so (after
// such a forward, 134 x 32000 18.4 and 16.4, 1000 x 32000 bf16 36.1 and 36.7, fp32 65.5 and 67).
constexpr int64_t kLpKeepBytes = (int64_t)768 << 20, kLpKeepBackBytes = (int64_t)48 << 20;

static dim3 logprob_grid(int64_t n) {
  return dim3((unsigned)std::min<int64_t>(n, kLpGridRows), (unsigned)((n + kLpGridRows - 1) / kLpGridRows));
}
template <typename T>
static hipError_t launch_logprob_t(const LogprobLaunch& P, hipStream_t st) {
  const dim3 grid = logprob_grid((int64_t)P.rows * P.splits);
#define AURORA_LOGPROB(S, HELD)                                                                                        \
  do {                                                                                                                \
    if (P.n_top > 0) hipLaunchKernelGGL((logprob_rows_kernel<T, S, true, HELD, false>), grid, dim3(S::kThreads), 0, st, P);  \
    else if (keep) hipLaunchKernelGGL((logprob_rows_kernel<T, S, false, HELD, true>), grid, dim3(S::kThreads), 0, st, P);    \
    else hipLaunchKernelGGL((logprob_rows_kernel<T, S, false, HELD, false>), grid, dim3(S::kThreads), 0, st, P);             \
  } while (0)
  const int64_t vecs = P.V / LpType<T>::kV;
  const bool keep = P.lse && (int64_t)P.rows * P.V * (int64_t)sizeof(T) <= kLpKeepBytes;
  if ((vecs + P.splits - 1) / P.splits <= kLpHeld * LpWide::kStep && P.rows <= kLpHeldRows) AURORA_LOGPROB(LpWide, kLpHeld);
  else if (P.splits == 1 && P.rows >= kLpNarrowRows && vecs <= (P.n_top > 0 ? kLpNarrowVecsTop : kLpNarrowVecs)) AURORA_LOGPROB(LpNarrow, 0);
  else AURORA_LOGPROB(LpWide, 0);
#undef AURORA_LOGPROB
  if (hipError_t e = hipGetLastError(); e != hipSuccess || P.splits == 1) return e;
  hipLaunchKernelGGL(logprob_merge_kernel<T>, logprob_grid(P.rows), dim3(kLpMergeThreads), 0, st, P);
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
  const dim3 grid = logprob_grid((int64_t)P.rows * P.splits);
  const bool keep = (int64_t)P.rows * P.V * (P.bf16 ? 2 : 4) <= kLpKeepBackBytes;
  if (P.bf16 && keep) hipLaunchKernelGGL((logprob_backward_kernel<bf16_t, true>), grid, dim3(kLpBackThreads), 0, st, P);
  else if (P.bf16) hipLaunchKernelGGL((logprob_backward_kernel<bf16_t, false>), grid, dim3(kLpBackThreads), 0, st, P);
  else if (keep) hipLaunchKernelGGL((logprob_backward_kernel<float, true>), grid, dim3(kLpBackThreads), 0, st, P);
  else hipLaunchKernelGGL((logprob_backward_kernel<float, false>), grid, dim3(kLpBackThreads), 0, st, P);
  return hipGetLastError();
}

}  // namespace aurora
