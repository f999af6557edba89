// Rotary positions on the way into the paged KV cache, and back.  The attention of the verification step (paper section 3.1) reads
// rotated keys out of the cache; this turns a layer's fresh queries and keys by their positions and stores keys and values at their
// slots.
//
//   pair i of a head at position t:   (x, y) -> (x c - y s, y c + x s),   c = m cos(t f_i),  s = m sin(t f_i)
//
// The pairs are (i, i + R/2) or (2i, 2i + 1) of the first R elements; the others pass through.  The transpose of the same turn - the
// angle negated - takes a gradient back.
//
// Bound by the bytes of q, k and v in and out: one pass, nothing is read twice.  A unit is two vectors of one head that are turned
// together (or passed through, or a value's); a thread keeps one unit of a row and walks down the rows of its block, so where it
// reads and writes is worked out once.  The angles of a block's rows are formed once and shared through LDS while the first rows are on
// their way: t f in 64 bits, its whole turns dropped there - at position 10^6 float32 holds an angle to a sixteenth of a radian only - and the
// sine and cosine of what is left in 32.
//
// 16384 rows of 32 + 8 + 8 heads of 128, bf16: 77 us = 5.2 TB/s, what a device copy of as many bytes takes; the gradients of 8192 57 us
// = 5.3; 8192 rows of 48 + 8 + 8 into an 8-bit cache, half of each head turned, 52 us = 4.8; 160 rows 3.8 us; 8192 rows in fp32 80 us =
// 5.0, their gradients 79.  Where 16-byte vectors do not fit, an element an access: 8192 rows of 32 + 8 + 8 an element further apart 101 us
// for 42, their gradients 97 for 56; of 9 + 3 + 3 heads of 80 with 40 turned 25 us, with all 80 12, their gradients 23.5 and 13.4.
#include "launch.hpp"

#include <algorithm>
#include <type_traits>

namespace aurora {

// The units of a row are cut into workgroups of so many, and each forms its rows' angles again.  Between small ones that do so more often
// and large ones that wait for each other longer: 192, 128 and 256 threads take 77, 78 and 82 us for the first of these (384 units a
// row), 57, 56 and 57 for the gradients, 52, 59 and 54 for the third (512).
constexpr int kRopeThreads = 192;
constexpr int kRopeAhead = 2;  // rows on their way, and of a block where there are many

typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4_t;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2_t;

// N elements at p as fp32, by 16-byte loads (N > 1)
template <int N, typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = to_f32<T>(*p);
  } else {
    constexpr int kPer = 16 / (int)sizeof(T);
#pragma unroll
    for (int o = 0; o < N; o += kPer) {
      const u32x4_t raw = *(const u32x4_t*)(p + o);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if constexpr (sizeof(T) == 4) {
          x[o + w] = __uint_as_float(raw[w]);
        } else {
          x[o + 2 * w] = __uint_as_float(raw[w] << 16);
          x[o + 2 * w + 1] = __uint_as_float(raw[w] & 0xffff0000u);
        }
      }
    }
  }
}

typedef __attribute__((ext_vector_type(2))) float f32x2_t;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

// E4M3 codes of four values, to nearest with ties to even; beyond the largest finite one (448) they become that, NaN stays NaN
__device__ __forceinline__ float e4m3_range(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }
__device__ __forceinline__ unsigned e4m3_pack4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(a), e4m3_range(b), 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(c), e4m3_range(d), w, true);
}

// The one rounding of a result: to the type it is kept in.  kPast: past the caches, for rows, not for the pools, nor beside an 8-bit cache
// (32768 rows of 48 + 8 + 8 heads 182 us, 186 past them): 4096 rows of 32 + 8 + 8 23.4 -> 19.7, their gradients 31.6 -> 28.3, 16384 rows
// 78.4 -> 77.2.  The attention, which reads the turned queries next, does not lose by it: the two calls in turn, past the caches and not, 160
// rows 26.5 and 26.8 us (contexts of 512), 55.5 and 55.7 (2048), 1280 rows 215.6 and 215.9, 4096 277.5 and 277.6.  (Loads past them:
// gradients of 8192 57 -> 66.)
template <int N, bool kPast = false, typename T>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[N]) {
  auto put = [](auto w, auto* at) {
    if constexpr (kPast) __builtin_nontemporal_store(w, at);
    else *at = w;
  };
  if constexpr (sizeof(T) == 1) {
    if constexpr (N == 1) {
      ((uint8_t*)p)[0] = (uint8_t)(e4m3_pack4(x[0], 0.f, 0.f, 0.f) & 0xffu);
    } else if constexpr (N == 4) {
      *(unsigned*)p = e4m3_pack4(x[0], x[1], x[2], x[3]);
    } else {
      *(u32x2_t*)p = u32x2_t{e4m3_pack4(x[0], x[1], x[2], x[3]), e4m3_pack4(x[4], x[5], x[6], x[7])};
    }
  } else if constexpr (N == 1) {
    *p = from_f32<T>(x[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int o = 0; o < N; o += 4) put(f32x4_t{x[o], x[o + 1], x[o + 2], x[o + 3]}, (f32x4_t*)(p + o));
  } else {
    u32x4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2_t{x[2 * i], x[2 * i + 1]}), bf16x2_t));
    put(w, (u32x4_t*)p);
  }
}

// T: type of the rows (q, k, v and the rotated q; the gradients on the way back); TC: of the cache.  kN: elements a vector.
// kBack: from fp32 gradients of the rotated q (rows) and of the cache to those of the rows.
template <typename T, typename TC, bool kPairs, int kN, bool kBack>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeLaunch P) {
  extern __shared__ __attribute__((aligned(16))) f32x2_t s_turn[];  // [rows of the block][R / 2] (cos, sin)
  const int tid = threadIdx.x, half = P.rotary / 2;
  const int block = blockIdx.x / P.chunks, chunk = blockIdx.x - block * P.chunks;
  const int row0 = block * P.block_rows, rows = min(P.block_rows, P.rows - row0);

  // ---- this thread's unit ------------------------------------------------------------------------------------
  const int turning = half / kN;                                        // units of a head that are turned
  const int passing = (P.D - P.rotary + 2 * kN - 1) / (2 * kN);         // that pass through
  const int per_head = turning + passing, per_value = (P.D + 2 * kN - 1) / (2 * kN);
  const int rotated = (P.Hq + P.Hkv) * per_head;
  const int unit = chunk * kRopeThreads + tid;
  const bool used = unit < rotated + P.Hkv * per_value;
  bool turns = false, two = true;
  int head, e0, e1, pair = 0;  // the unit's vectors start at elements e0 and e1 of the head
  if (unit < rotated) {
    head = unit / per_head;
    const int u = unit - head * per_head;
    turns = u < turning;
    if (turns) {
      pair = u * kN;
      e0 = kPairs ? 2 * u * kN : u * kN;
      e1 = kPairs ? e0 + kN : e0 + half;
    } else {
      e0 = P.rotary + (u - turning) * 2 * kN;
      e1 = e0 + kN;
      two = e1 < P.D;
    }
  } else {
    head = (unit - rotated) / per_value;
    e0 = (unit - rotated - head * per_value) * 2 * kN;
    e1 = e0 + kN;
    two = e1 < P.D;
    head += P.Hq + P.Hkv;
  }
  const bool is_q = head < P.Hq, is_v = head >= P.Hq + P.Hkv;
  const int hk = is_q ? 0 : head - P.Hq - (is_v ? P.Hkv : 0);
  if (!two) e1 = e0;
  const bool side = two && e1 == e0 + kN && P.D % (2 * kN) == 0;  // side by side, at an even vector of the pool

  // rows side: q, k or v of a token (read on the way in, written on the way back); the other side: the rotated q's row, or the cache
  T* rows_p = (T*)(is_q ? P.q : is_v ? P.v : P.k);
  const int64_t rows_stride = is_q ? P.q_stride : is_v ? P.v_stride : P.k_stride;
  rows_p += (int64_t)(is_q ? head : hk) * P.D;
  typedef typename std::conditional<kBack, float, T>::type TQ;
  typedef typename std::conditional<kBack, float, TC>::type TP;
  TQ* qo_p = (TQ*)P.q_out + (int64_t)head * P.D;
  TP* pool = (TP*)(is_v ? P.v_pages : P.k_pages);
  float scale = 1.f;
  if constexpr (!kBack && sizeof(TC) == 1) {
    if (used && !is_q) scale = (is_v ? P.v_scale : P.k_scale)[hk];
  }

  // where row r's part of the other side is, or -1: a row behind the last sequence
  auto slot_of = [&](int r) -> int {
    if (!P.slots) return 0;
    const int s = __builtin_amdgcn_readfirstlane(P.slots[row0 + r]);
    return s >= 0 && s < P.num_slots ? s : -1;
  };
  auto pool_at = [&](int slot) -> int64_t {
    const int page = P.page_shift >= 0 ? slot >> P.page_shift : slot / P.page;
    return (((int64_t)page * P.Hkv + hk) * P.page + (slot - page * P.page)) * P.D;
  };
  auto load = [&](int r, int slot, float (&a)[kN], float (&b)[kN]) {
    if constexpr (kBack) {
      const float* p = is_q ? (const float*)qo_p + (int64_t)(row0 + r) * P.q_out_stride : (const float*)pool + pool_at(max(slot, 0));
      load_vec<kN>(p + e0, a);
      load_vec<kN>(p + e1, b);
    } else {
      const T* p = rows_p + (int64_t)(row0 + r) * rows_stride;
      load_vec<kN>(p + e0, a);
      load_vec<kN>(p + e1, b);
    }
  };

  constexpr int kAhead = kRopeAhead;
  float xa[kAhead][kN], xb[kAhead][kN];
  int slot[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    slot[i] = -1;
    if (i < rows) {
      slot[i] = slot_of(i);
      if (used) load(i, slot[i], xa[i], xb[i]);
    }
  }

  // ---- the block's angles ------------------------------------------------------------------------------------
  for (int i = tid; i < rows * half; i += kRopeThreads) {
    const int r = i / half, p = i - r * half;
    const double turn = (double)P.positions[row0 + r] * (P.frequencies[p] * 0.15915494309189533577);  // / 2 pi
    const double part = turn - rint(turn);
    const float hi = (float)(2.0 * part), lo = (float)(2.0 * part - (double)hi);  // half turns
    float s, c;
    sincospif(hi, &s, &c);
    const float d = lo * 3.14159265358979f;
    const float sn = fmaf(d, c, s), cs = fmaf(-d, s, c);
    s_turn[i] = f32x2_t{cs * P.magnitude, (kBack ? -sn : sn) * P.magnitude};
  }
  __syncthreads();
  if (!used) return;

  for (int r0 = 0; r0 < rows; r0 += kAhead) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = r0 + i;
      if (r < rows) {
        float a[kN], b[kN];
        const int sl = slot[i];
#pragma unroll
        for (int e = 0; e < kN; ++e) { a[e] = xa[i][e]; b[e] = xb[i][e]; }
        if (r + kAhead < rows) {
          slot[i] = slot_of(r + kAhead);
          load(r + kAhead, slot[i], xa[i], xb[i]);
        }
        if (turns) {
          const f32x2_t* t = s_turn + r * half + pair;
          if constexpr (kPairs && kN > 1) {
#pragma unroll
            for (int e = 0; e < kN; e += 2) {
              const f32x2_t t0 = t[e / 2], t1 = t[kN / 2 + e / 2];
              const float a0 = a[e], a1 = a[e + 1], b0 = b[e], b1 = b[e + 1];
              a[e] = a0 * t0[0] - a1 * t0[1];
              a[e + 1] = a1 * t0[0] + a0 * t0[1];
              b[e] = b0 * t1[0] - b1 * t1[1];
              b[e + 1] = b1 * t1[0] + b0 * t1[1];
            }
          } else {
#pragma unroll
            for (int e = 0; e < kN; ++e) {
              const f32x2_t t0 = t[e];
              const float x = a[e], y = b[e];
              a[e] = x * t0[0] - y * t0[1];
              b[e] = y * t0[0] + x * t0[1];
            }
          }
        }
        if constexpr (kBack) {
          if (sl < 0) {  // the row had no effect
#pragma unroll
            for (int e = 0; e < kN; ++e) a[e] = b[e] = 0.f;
          }
          T* p = rows_p + (int64_t)(row0 + r) * rows_stride;
          store_vec<kN, true>(p + e0, a);
          if (two) store_vec<kN, true>(p + e1, b);
        } else if (sl >= 0) {
          if (is_q) {
            T* p = (T*)qo_p + (int64_t)(row0 + r) * P.q_out_stride;
            store_vec<kN, sizeof(TC) != 1>(p + e0, a);
            if (two) store_vec<kN, sizeof(TC) != 1>(p + e1, b);
          } else {
            if constexpr (sizeof(TC) == 1) {
#pragma unroll
              for (int e = 0; e < kN; ++e) { a[e] = a[e] / scale; b[e] = b[e] / scale; }
            }
            TC* p = (TC*)pool + pool_at(sl);
            if (sizeof(TC) == 1 && kN == 8 && side) {  // sixteen codes side by side in one store
              *(u32x4_t*)(p + e0) = u32x4_t{e4m3_pack4(a[0], a[1 % kN], a[2 % kN], a[3 % kN]), e4m3_pack4(a[4 % kN], a[5 % kN], a[6 % kN], a[7 % kN]),
                                            e4m3_pack4(b[0], b[1 % kN], b[2 % kN], b[3 % kN]), e4m3_pack4(b[4 % kN], b[5 % kN], b[6 % kN], b[7 % kN])};
            } else {
              store_vec<kN>(p + e0, a);
              if (two) store_vec<kN>(p + e1, b);
            }
          }
        }
      }
    }
  }
}

// workgroups that a row is cut into where a vector has n elements
static int rope_chunks(const RopeLaunch& P, int n) {
  const int units = (P.Hq + P.Hkv) * (P.rotary / 2 / n + (P.D - P.rotary + 2 * n - 1) / (2 * n)) + P.Hkv * ((P.D + 2 * n - 1) / (2 * n));
  return (units + kRopeThreads - 1) / kRopeThreads;
}
// One row a block while the launch would not fill the chip, then as many as are loaded ahead: more only make a block's start longer
// (two a block, four, eight, sixteen: 16384 rows of 32 + 8 + 8 heads of 128 77, 77, 82, 99 us, their gradients 54.5, 58.5, 63, 63).
static int64_t rope_block_rows(const RopeLaunch& P, int chunks) {
  int64_t rows = (int64_t)chunks * P.rows / kRopeAhead >= 2048 ? kRopeAhead : 1;
  while ((P.rows + rows - 1) / rows * chunks > ((int64_t)1 << 32) / kRopeThreads - 1) rows *= 2;  // fewer than 2^32 threads
  return rows;
}
static size_t rope_lds(const RopeLaunch& P, int64_t block_rows) { return (size_t)block_rows * (P.rotary / 2) * sizeof(f32x2_t); }

// (single elements are the most workgroups a row, and so the most rows a block)
bool rope_fits(const RopeLaunch& P) { return rope_lds(P, rope_block_rows(P, rope_chunks(P, 1))) <= 64 * 1024; }

template <typename T, typename TC, bool kPairs, int kN, bool kBack>
static hipError_t launch_rope_k(RopeLaunch P, hipStream_t st) {
  P.page_shift = (P.page & (P.page - 1)) == 0 ? __builtin_ctz(P.page) : -1;
  P.chunks = rope_chunks(P, kN);
  const int64_t rows = rope_block_rows(P, P.chunks);
  P.block_rows = (int)rows;
  hipLaunchKernelGGL((rope_kernel<T, TC, kPairs, kN, kBack>), dim3((unsigned)((P.rows + rows - 1) / rows * P.chunks)), dim3(kRopeThreads),
                     rope_lds(P, rows), st, P);
  return hipGetLastError();
}

template <typename T, typename TC, int kN, bool kBack>
static hipError_t launch_rope_t(const RopeLaunch& P, hipStream_t st) {
  return P.interleaved ? launch_rope_k<T, TC, true, kN, kBack>(P, st) : launch_rope_k<T, TC, false, kN, kBack>(P, st);
}

// Whole vectors: every head, row and half of a head starts at one, in all the arrays (the cache's rows do if the head's size does).
static bool rope_vectors(const RopeLaunch& P, int n) {
  const uintptr_t p = (uintptr_t)P.q | (uintptr_t)P.q_out | (uintptr_t)P.k | (uintptr_t)P.v | (uintptr_t)P.k_pages | (uintptr_t)P.v_pages;
  return (p & 15) == 0 && P.D % n == 0 && P.rotary % (2 * n) == 0 && (P.q_stride | P.q_out_stride | P.k_stride | P.v_stride) % n == 0;
}

hipError_t launch_rope(const RopeLaunch& P, bool back, hipStream_t st) {
  const bool vec = rope_vectors(P, P.bf16 ? 8 : 4);
#define AURORA_ROPE(T, TC, N) (vec ? launch_rope_t<T, TC, N, false>(P, st) : launch_rope_t<T, TC, 1, false>(P, st))
  if (back) {
    if (P.bf16) return vec ? launch_rope_t<bf16_t, bf16_t, 8, true>(P, st) : launch_rope_t<bf16_t, bf16_t, 1, true>(P, st);
    return vec ? launch_rope_t<float, float, 4, true>(P, st) : launch_rope_t<float, float, 1, true>(P, st);
  }
  if (P.kv_fp8) return P.bf16 ? AURORA_ROPE(bf16_t, e4m3_t, 8) : AURORA_ROPE(float, e4m3_t, 4);
  return P.bf16 ? AURORA_ROPE(bf16_t, bf16_t, 8) : AURORA_ROPE(float, float, 4);
#undef AURORA_ROPE
}

}  // namespace aurora
