// Block tables and slot maps of the paged KV cache, built on the GPU from request lengths.  After a verification step (paper
// section 2.1: a prefix of a chain's drafts is kept) only the GPU knows how long each request has become; this plans the pages of
// the next one without a trip to the host.
//
//   pages(n) = ceil(n / page).  A request that holds h tokens and is to hold w gives pages(h) - pages(w) back if w < h, and takes
//   pages(w) - pages(h) if w > h.  All pages given back go on top of the stack of free pages, in order; then pages are taken from the
//   top, in order.  With F given back onto n free ones, the k-th page taken is therefore the (F - 1 - k)-th given back if k < F, and
//   stack entry n - 1 - (k - F) if not - and of the pages given back the first F - taken are all that reaches the stack.
//
// So the state after the call is a function of three prefix sums over the requests (pages given back, pages taken, token rows), and
// no order between writes is needed: cells of the table that are read (pages held, pages given back) are never written, stack
// entries that are read lie below those that are written.  Tokens of a page taken in this call find it the same way, not through
// the table.
//
// Bound by latency: a launch, the lengths, a search and one or two loads in turn - 4.2 us a call in a captured graph for 32 requests of
// five tokens, 5.1 for 256 that grow, shrink, end and begin with 120 000 rows, 7.0 for a million rows, of which writing their positions and
// slots is 1.6 at a copy's rate.  Up to 1024 requests every workgroup forms the prefix sums itself, four requests a thread, and does its
// share of the writing: one launch.  Where more than one workgroup is wanted and an output is the input that the others still read, or there
// are more requests, one workgroup plans into the workspace and a second launch writes: the same three in place 6.6, 8.6 and 10.2 us, 2000
// requests of five tokens 15.4.
#include "launch.hpp"

#include <algorithm>

namespace aurora {

constexpr int kPlanThreads = 256;
constexpr int kPlanPer = 4;                              // requests a thread
constexpr int kPlanChunk = kPlanThreads * kPlanPer;      // requests planned at a time
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanFewRows = 1 << 18;                    // up to here a thread writes one row, beyond four

// What the writing needs: per request the first row, page taken and page given back, the tokens held, and the table column at which
// the pages taken or given back start; then the stack's size and the totals.
struct PlanArrays { int32_t *row, *take, *give, *held, *col; };
struct PlanTotals { int n, freed, taken, rows; };

struct PlanReq { int held, want, col, need, back; unsigned rows; bool grow, shrink, differs; };

// Sums of rows stop at 2^32 - 1, past every limit: no order of adding changes them, and one that stopped is refused.
__device__ __forceinline__ unsigned add_rows(unsigned a, unsigned b) { return __builtin_elementwise_add_sat(a, b); }

// (a division costs as much as the rest of a request: pages of a power of two shift)
__device__ __forceinline__ int page_of(const CachePlanLaunch& P, unsigned token) {
  return (int)(P.page_shift >= 0 ? token >> P.page_shift : token / (unsigned)P.page);
}
__device__ __forceinline__ int pages_of(const CachePlanLaunch& P, int tokens) { return page_of(P, (unsigned)tokens + (unsigned)P.page - 1u); }

__device__ __forceinline__ PlanReq plan_request(const CachePlanLaunch& P, int b) {
  PlanReq r = {};
  if (b >= P.B) return r;
  r.held = P.held_lens ? P.held_lens[b] : 0;
  r.want = P.want_lens[b];
  r.differs = r.want != r.held;
  if (r.held < 0 || r.want < 0) return r;
  const int hp = pages_of(P, r.held), wp = pages_of(P, r.want);
  if (hp > P.max_pages || wp > P.max_pages) return r;
  r.grow = r.want > r.held;
  r.shrink = r.want < r.held;
  r.col = min(hp, wp);
  r.need = r.grow ? wp - hp : 0;
  r.back = r.shrink ? hp - wp : 0;
  r.rows = r.grow ? (unsigned)(r.want - r.held) : 0u;
  return r;
}

struct PlanSums { int back, need; unsigned rows; };

// one step of an inclusive scan over the 64 lanes: adds the sums of the lane that the data-parallel control `kCtl` names
template <int kCtl, int kRows>
__device__ __forceinline__ void scan_step(PlanSums& x) {
  x.back += __builtin_amdgcn_update_dpp(0, x.back, kCtl, kRows, 0xf, false);
  x.need += __builtin_amdgcn_update_dpp(0, x.need, kCtl, kRows, 0xf, false);
  x.rows = add_rows(x.rows, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x.rows, kCtl, kRows, 0xf, false));
}

// exclusive prefix of the threads' sums over the workgroup, and the totals
__device__ __forceinline__ PlanSums plan_scan(const PlanSums& mine, PlanSums& total, PlanSums* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  PlanSums x = mine;
  scan_step<0x111, 0xf>(x);  // within rows of sixteen: from one, two, four, eight lanes below
  scan_step<0x112, 0xf>(x);
  scan_step<0x114, 0xf>(x);
  scan_step<0x118, 0xf>(x);
  scan_step<0x142, 0xa>(x);  // the first row's last lane into the second row, the third's into the fourth
  scan_step<0x143, 0xc>(x);  // the second's into the upper half
  __syncthreads();  // (the last chunk's sums may still be read)
  if (lane == 63) s_wave[wave] = x;
  PlanSums below = {__shfl_up(x.back, 1, kWave), __shfl_up(x.need, 1, kWave), (unsigned)__shfl_up((int)x.rows, 1, kWave)};
  if (lane == 0) below = {0, 0, 0u};
  __syncthreads();
  total = {0, 0, 0u};
  PlanSums before = {0, 0, 0u};
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const PlanSums t = s_wave[w];
    if (w < wave) { before.back += t.back; before.need += t.need; before.rows = add_rows(before.rows, t.rows); }
    total.back += t.back; total.need += t.need; total.rows = add_rows(total.rows, t.rows);
  }
  return {before.back + below.back, before.need + below.need, add_rows(before.rows, below.rows)};
}

// The plan of all requests, by one workgroup; A may lie in LDS (one chunk) or in the workspace.  publish: this workgroup writes
// the results that are not shared out.
template <bool kOneChunk>
__device__ __forceinline__ PlanTotals plan_requests(const CachePlanLaunch& P, const PlanArrays& A, bool publish) {
  __shared__ PlanSums s_wave[kPlanWaves];
  __shared__ int s_cut, s_refused, s_cut_need;
  __shared__ unsigned s_cut_rows;
  const int tid = threadIdx.x;
  const int n = min(max(P.free_count[0], 0), P.num_pages);
  const unsigned most_rows = P.slots ? (unsigned)P.max_rows : UINT32_MAX;
  if (tid == 0) { s_cut = INT32_MAX; s_refused = 0; }

  int freed = 0;
  if constexpr (!kOneChunk) {  // the pages given back, before anyone is granted a page
    PlanSums all = {0, 0, 0u}, t;
    for (int b = tid; b < P.B; b += kPlanThreads) all.back += plan_request(P, b).back;
    plan_scan(all, t, s_wave);
    freed = t.back;
  }
  PlanSums carry = {0, 0, 0u};
  int cut = INT32_MAX, cut_need = 0;
  unsigned cut_rows = 0;
  for (int base = 0; kOneChunk ? base == 0 : base < P.B; base += kPlanChunk) {
    PlanReq r[kPlanPer];
    PlanSums mine = {0, 0, 0u}, total;
    int refused = 0;
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i) {
      r[i] = plan_request(P, base + tid * kPlanPer + i);
      mine.back += r[i].back; mine.need += r[i].need; mine.rows = add_rows(mine.rows, r[i].rows);
      refused += r[i].differs && !r[i].grow && !r[i].shrink;
    }
    PlanSums at = plan_scan(mine, total, s_wave);
    if constexpr (kOneChunk) freed = total.back;
    at.back += carry.back; at.need += carry.need; at.rows = add_rows(at.rows, carry.rows);
    carry.back += total.back; carry.need += total.need; carry.rows = add_rows(carry.rows, total.rows);
    const int64_t pages = (int64_t)n + freed;
    if (carry.need > pages || carry.rows > most_rows) {  // (the whole workgroup)
      // The sums never fall, so those who are refused for want of pages or rows are one run of growing requests up to the last: the
      // first of them is all there is to find.
      PlanSums cum = at, at_first = {0, 0, 0u};
      int first = INT32_MAX;
#pragma unroll
      for (int i = 0; i < kPlanPer; ++i) {
        const PlanSums next = {0, cum.need + r[i].need, add_rows(cum.rows, r[i].rows)};
        if (r[i].grow && (next.need > pages || next.rows > most_rows)) {
          if (first == INT32_MAX) { first = base + tid * kPlanPer + i; at_first = cum; }
          ++refused;
        }
        cum = next;
      }
      if (first != INT32_MAX) atomicMin(&s_cut, first);
      __syncthreads();
      if (first != INT32_MAX && s_cut == first) { s_cut_need = at_first.need; s_cut_rows = at_first.rows; }
      __syncthreads();
      cut = s_cut; cut_need = s_cut_need; cut_rows = s_cut_rows;
    }
    if (refused) atomicAdd(&s_refused, refused);
    PlanSums cum = at;
    int row[kPlanPer], take[kPlanPer], give[kPlanPer];
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i) {
      const int b = base + tid * kPlanPer + i;
      const bool past = b >= cut;
      row[i] = (int)(past ? cut_rows : cum.rows);
      take[i] = past ? cut_need : cum.need;
      give[i] = cum.back;
      if (b < P.B) {
        if constexpr (!kOneChunk) {
          A.row[b] = row[i]; A.take[b] = take[i]; A.give[b] = give[i]; A.held[b] = r[i].held; A.col[b] = r[i].col;
        }
        if (publish) {
          P.seq_lens[b] = r[i].shrink || (r[i].grow && !past) ? r[i].want : r[i].held;
          if (P.row_start) P.row_start[b] = row[i];
        }
      }
      cum.back += r[i].back; cum.need += r[i].need; cum.rows = add_rows(cum.rows, r[i].rows);
    }
    if constexpr (kOneChunk) {  // in LDS, past the last request too: there the sums are the totals
      static_assert(kPlanPer == 4, "one vector an array");
      ((int4*)A.row)[tid] = make_int4(row[0], row[1], row[2], row[3]);
      ((int4*)A.take)[tid] = make_int4(take[0], take[1], take[2], take[3]);
      ((int4*)A.give)[tid] = make_int4(give[0], give[1], give[2], give[3]);
      ((int4*)A.held)[tid] = make_int4(r[0].held, r[1].held, r[2].held, r[3].held);
      ((int4*)A.col)[tid] = make_int4(r[0].col, r[1].col, r[2].col, r[3].col);
    }
  }
  PlanTotals t;
  t.n = n;
  t.freed = freed;
  t.taken = cut != INT32_MAX ? cut_need : carry.need;
  t.rows = (int)(cut != INT32_MAX ? cut_rows : carry.rows);
  if (tid == 0 && (!kOneChunk || P.B == kPlanChunk)) { A.row[P.B] = t.rows; A.take[P.B] = t.taken; A.give[P.B] = t.freed; }
  __syncthreads();
  if (publish && tid == 0) {
    if (P.row_start) P.row_start[P.B] = t.rows;
    P.free_count_out[0] = (int)min((int64_t)n + freed - t.taken, (int64_t)P.num_pages);
    if (P.info) { P.info[0] = t.rows; P.info[1] = t.taken; P.info[2] = t.freed; P.info[3] = s_refused; }
  }
  return t;
}

// the request whose run of `start` holds x: the last b with start[b] <= x (start[0] = 0, x < start[B]); a quarter of the range a step
__device__ __forceinline__ int plan_owner(const int32_t* start, int B, int x) {
  int lo = 0, n = B;
  while (n > 1) {
    const int q = (n + 3) >> 2;  // the pieces start at lo, lo + q, lo + 2q, lo + 3q
    const int a = start[lo + min(q, n)], b = start[lo + min(2 * q, n)], c = start[lo + min(3 * q, n)];
    const int piece = (a <= x) + (b <= x) + (c <= x);
    lo += piece * q;
    n = min(q, n - piece * q);
  }
  return lo;
}

__device__ __forceinline__ int given_page(const CachePlanLaunch& P, const PlanArrays& A, int j) {
  const int b = plan_owner(A.give, P.B, j);
  return P.block_table[(size_t)b * P.max_pages + A.col[b] + (j - A.give[b])];
}
__device__ __forceinline__ int taken_page(const CachePlanLaunch& P, const PlanArrays& A, const PlanTotals& t, int k) {
  return k < t.freed ? given_page(P, A, t.freed - 1 - k) : P.free_pages[t.n - 1 - (k - t.freed)];
}

// kRows rows, with one search and one page for all of them more often than not
template <int kRows>
__device__ __forceinline__ void plan_rows(const CachePlanLaunch& P, const PlanArrays& A, const PlanTotals& t, int64_t r0) {
  int pos[kRows], slot[kRows];
  int b = 0, left = 0, at = 0, pg = 0, off = 0, pid = 0;  // left: rows of request b from here on
#pragma unroll
  for (int e = 0; e < kRows; ++e) {
    if (r0 + e >= t.rows) { pos[e] = 0; slot[e] = -1; continue; }
    const int r = (int)r0 + e;
    const bool enter = left == 0;
    if (enter) {
      b = plan_owner(A.row, P.B, r);
      left = A.row[b + 1] - r;
      at = A.held[b] + (r - A.row[b]);
      pg = page_of(P, at);
      off = at - pg * P.page;
    } else if (off == P.page) {
      ++pg;
      off = 0;
    }
    if (enter || off == 0) {
      const int col = A.col[b];
      pid = pg < col ? P.block_table[(size_t)b * P.max_pages + pg] : taken_page(P, A, t, A.take[b] + pg - col);
    }
    pos[e] = at++;
    slot[e] = (int)((unsigned)pid * (unsigned)P.page + (unsigned)off++);
    --left;
  }
  if (kRows == 4 && P.wide_rows && r0 + 4 <= P.max_rows) {
    *(int4*)(P.positions + r0) = make_int4(pos[0], pos[1 % kRows], pos[2 % kRows], pos[3 % kRows]);
    *(int4*)(P.slots + r0) = make_int4(slot[0], slot[1 % kRows], slot[2 % kRows], slot[3 % kRows]);
  } else {
#pragma unroll
    for (int e = 0; e < kRows; ++e)
      if (r0 + e < P.max_rows) { P.positions[r0 + e] = pos[e]; P.slots[r0 + e] = slot[e]; }
  }
}

// The rows, table cells and stack entries of this workgroup: each is a chain of a search and one or two loads, so they are numbered
// through, and a thread goes through as few of them as the launch allows.
template <int kRows>
__device__ __forceinline__ void plan_write(const CachePlanLaunch& P, const PlanArrays& A, const PlanTotals& t) {
  const int64_t rows = P.slots ? ((int64_t)P.max_rows + kRows - 1) / kRows : 0, takes = rows + t.taken, all = takes + max(0, t.freed - t.taken);
  for (int64_t i = (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; i < all; i += (int64_t)gridDim.x * kPlanThreads) {
    if (i < rows) {
      plan_rows<kRows>(P, A, t, kRows * i);
    } else if (i < takes) {
      const int k = (int)(i - rows), b = plan_owner(A.take, P.B, k);
      P.block_table[(size_t)b * P.max_pages + A.col[b] + (k - A.take[b])] = taken_page(P, A, t, k);
    } else {
      const int j = (int)(i - takes);
      if ((int64_t)t.n + j < P.num_pages) P.free_pages[t.n + j] = given_page(P, A, j);
    }
  }
}

template <int kRows>
__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(CachePlanLaunch P) {
  __shared__ __attribute__((aligned(16))) int32_t s_row[kPlanChunk + 4], s_take[kPlanChunk + 4], s_give[kPlanChunk + 4], s_held[kPlanChunk],
      s_col[kPlanChunk];
  const PlanArrays A = {s_row, s_take, s_give, s_held, s_col};
  const PlanTotals t = plan_requests<true>(P, A, blockIdx.x == 0);
  plan_write<kRows>(P, A, t);
}

__device__ __forceinline__ PlanArrays workspace_arrays(const CachePlanLaunch& P) {
  const size_t n = (size_t)P.B + 1;
  int32_t* w = P.work + 4;
  return {w, w + n, w + 2 * n, w + 3 * n, w + 4 * n};
}
__global__ __launch_bounds__(kPlanThreads) void cache_plan_requests_kernel(CachePlanLaunch P) {
  const PlanTotals t = plan_requests<false>(P, workspace_arrays(P), true);
  if (threadIdx.x == 0) *(int4*)P.work = make_int4(t.n, t.freed, t.taken, t.rows);
}
template <int kRows>
__global__ __launch_bounds__(kPlanThreads) void cache_plan_write_kernel(CachePlanLaunch P) {
  const int4 t = *(const int4*)P.work;
  plan_write<kRows>(P, workspace_arrays(P), PlanTotals{t.x, t.y, t.z, t.w});
}

size_t cache_plan_work_bytes(int batch) { return 16 + 5 * ((size_t)batch + 1) * sizeof(int32_t); }

hipError_t launch_cache_plan(const CachePlanLaunch& plan, hipStream_t st) {
  CachePlanLaunch P = plan;
  P.page_shift = (P.page & (P.page - 1)) == 0 ? __builtin_ctz(P.page) : -1;
  // Few rows are given a thread each: four that belong to two or three requests are as many loads in turn (us with one and with four:
  // 160 rows 4.0 and 6.1, 120 000 5.6 and 9.0, 2^20 9.7 and 7.5, where writes of 16 bytes count; in the second of two launches 160 6.6
  // and 9.0, 120 000 8.6 and 13.0).  A workgroup per 256 or 1024 rows, and per 4096 cells of the table (how many cells change hands
  // only the lengths say).
  const bool few = P.max_rows <= kPlanFewRows;
  const int64_t rows = P.slots ? ((int64_t)P.max_rows + (few ? 255 : 1023)) / (few ? 256 : 1024) : 0;
  const int64_t cells = (int64_t)P.B * P.max_pages / 4096;
  const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(rows + cells, 1024));
  // an output that replaces an input is safe within one workgroup alone: the others read the input too
  const bool in_place = P.free_count_out == P.free_count || P.seq_lens == P.held_lens || P.seq_lens == P.want_lens;
  if (P.B <= kPlanChunk && (grid == 1 || !in_place)) {
    if (few) hipLaunchKernelGGL(cache_plan_kernel<1>, dim3(grid), dim3(kPlanThreads), 0, st, P);
    else hipLaunchKernelGGL(cache_plan_kernel<4>, dim3(grid), dim3(kPlanThreads), 0, st, P);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(cache_plan_requests_kernel, dim3(1), dim3(kPlanThreads), 0, st, P);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (few) hipLaunchKernelGGL(cache_plan_write_kernel<1>, dim3(grid), dim3(kPlanThreads), 0, st, P);
  else hipLaunchKernelGGL(cache_plan_write_kernel<4>, dim3(grid), dim3(kPlanThreads), 0, st, P);
  return hipGetLastError();
}

}  // namespace aurora
