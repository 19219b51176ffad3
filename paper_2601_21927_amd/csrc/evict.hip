// Eviction by accumulated attention weight: of a request's rows the first and the last ones stay, and of those
// between them the heaviest, up to a budget.  What stays keeps its order, because the rows' order is what the
// next-turn step reads (system prompt, Nexus rows, the turn's rows).
//
// select_kernel, one workgroup per request: checks the lengths of every request, so that a call is done for all or
// for none, finds the weight that separates kept from dropped rows by a radix search over the weights' order (up to
// three passes of eleven bits, histograms in LDS; a request's first 8,192 weights stay in registers), and lists the kept
// rows.  It writes to the workspace only.  Bound by round trips that wait for one another (status and length, limits,
// capacity, first row, weights, then three for the other requests' limits; the early returns of evict_check keep the loads
// apart) and by the search's barriers: 9.5 us for 8 requests of 1,328 rows, 12 for 4 of 7,552, 39 for one of 30,000, 102
// for one of 100,000.
// move_kernel, to another cache: every kept row is read and written once, in parallel over rows.  Bound by HBM: 64
// uneven requests of up to 8,192 rows of 8 bf16 heads of 128 (652 MB) 4.7 TB/s.  Small calls are bound by round trips: a
// piece's list entry is waited for before its loads, so the pieces of a thread come one after the other.
// move_in_place_kernel: row j goes down to j from list[j] >= j, so a workgroup that walks the rows upwards, loading a
// batch before it stores it, never overwrites a row it has yet to read; workgroups split the rows' bytes into
// columns.  Rows before the first dropped one are not touched.  64 requests of 4,000 bf16 rows to 2,000: 4.5 TB/s; one
// request has 32 to 64 columns, each a workgroup that waits for its loads and, between a batch's guarded stores, for every
// store: 30,000 bf16 rows to 20,000 62 us (2.6 TB/s).
#include <algorithm>

#include "common.h"
#include "scan.h"

namespace sonic {

constexpr int kSelectThreads = 1024;
constexpr int kSelectRows = 8;                              // consecutive rows of a thread
constexpr int kSelectChunk = kSelectThreads * kSelectRows;
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 8;   // 64 uneven requests of 8,192 rows at most to half of that: 149 us a pass, with 4 158, with 16 206
constexpr int kWalkThreads = 1024;
constexpr int kWalkUnroll = 8;

// A request's rows, cut into head, middle and tail.
struct EvictReq {
  int len, head, tail, kept;
};
__device__ __forceinline__ int evict_check(int j, const EvictCall &c, EvictReq *r) {
  const int len = c.cache_len[j], head = c.keep_head[j], tail = c.keep_tail[j], budget = c.budget[j];
  *r = EvictReq{0, 0, 0, 0};
  if (len < 0 || len > c.max_rows || head < 0 || tail < 0 || budget < 0) return SONIC_ERR_BAD_LAYOUT;
  r->len = len;
  r->head = min(head, len);
  r->tail = min(tail, len - r->head);
  r->kept = len <= budget ? len : max(r->head + r->tail, budget);
  if (c.out_row_cap != nullptr && r->kept > c.out_row_cap[j]) return SONIC_ERR_CAPACITY;
  return 0;
}

// Weights as unsigned integers of the same order; NaN as -infinity, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w == w ? w + 0.f : -INFINITY);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// A pass of the radix search: 2,048 bins, a quarter of the lanes adding to a copy of their own (weights share their
// exponents, and lanes that add to one word take turns).  find_digit adds the copies up and writes the digit that
// holds the `need`-th key from above, how many of its keys are wanted, and how many it has; the copies are clear again.
constexpr int kDigitBits = 11, kBins = 1 << kDigitBits, kCopies = 4;
static_assert(kBins == 2 * kSelectThreads, "a thread adds up two bins");
struct Digit {
  int digit, rest, count;
};
__device__ __forceinline__ void find_digit(int *copies, int need, Digit *found, int *lds) {
  // thread t has the bins kBins - 1 - 2 t and the one below
  int h[2] = {0, 0};
  const int top = kBins - 1 - 2 * threadIdx.x;
#pragma unroll
  for (int c = 0; c < kCopies; ++c) {
    int2 *pair = reinterpret_cast<int2 *>(copies + c * kBins + top - 1);
    const int2 x = *pair;
    *pair = make_int2(0, 0);
    h[0] += x.y;
    h[1] += x.x;
  }
  int total;
  int above = block_int_scan<kSelectThreads>(h[0] + h[1], &total, lds);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (above < need && above + h[i] >= need) *found = Digit{top - i, need - above, h[i]};
    above += h[i];
  }
  __syncthreads();
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictCall c, EvictWs ws) {
  __shared__ int lds[2 * (kSelectThreads / kWave)];
  __shared__ __align__(8) int copies[kCopies * kBins];
  __shared__ int s_first;
  __shared__ Digit s_digit;
  const int b = blockIdx.x;
  // Behind a pending error a length may be anything: no weight is read for it.  Workgroup 0's look at the status word
  // decides for the call; a request whose workgroup saw an error that workgroup 0 did not (the word may change meanwhile)
  // is left as it is.
  const bool pending = __hip_atomic_load(c.status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != 0;
  EvictReq own;
  const int own_code = evict_check(b, c, &own);
  if (pending) own.len = own.head = own.tail = 0;
  const float *w = c.row_weight + c.row_off[b];
  const int lo = own.head, hi = own.len - own.tail;
  // A thread has kSelectRows consecutive rows of a chunk; the first chunk's keys stay in registers.  Head and tail
  // rows are as if heavier than any, rows past the end as if lighter: no weight has their keys.
  const int mine = kSelectRows * threadIdx.x;
  auto load_keys = [&](int base, uint32_t (&key)[kSelectRows]) {
    float x[kSelectRows];
#pragma unroll
    for (int i = 0; i < kSelectRows; ++i) {
      const int r = base + mine + i;
      x[i] = r >= lo && r < hi ? w[r] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kSelectRows; ++i) {
      const int r = base + mine + i;
      key[i] = r >= own.len ? 0u : r < lo || r >= hi ? 0xFFFFFFFFu : weight_key(x[i]);
    }
  };
  uint32_t first_keys[kSelectRows];
  load_keys(0, first_keys);
  int bad = pending;
  for (int j = threadIdx.x; j < c.batch; j += kSelectThreads) {
    EvictReq r;
    bad |= evict_check(j, c, &r) != 0;
  }
  for (int i = threadIdx.x; i < kCopies * kBins; i += kSelectThreads) copies[i] = 0;
  if (threadIdx.x == 0) s_first = own.kept;
  bad = __syncthreads_or(bad);
  if (own_code != 0 && threadIdx.x == 0) raise_status(c.status, own_code);
  if (b == 0 && threadIdx.x == 0) ws.ctrl[0] = !bad;
  if (bad) {
    if (threadIdx.x == 0) ws.req[b] = make_int2(-1, 0);
    return;
  }

  int32_t *list = ws.list + static_cast<size_t>(b) * c.max_rows;
  const int take = own.kept - own.head - own.tail;   // of the middle rows
  // kept are the keys above the threshold, and the first `rest` of those at it
  uint32_t threshold = 0;   // all: every key is above 0
  int rest = 0;
  if (take < hi - lo) {
    threshold = 0xFFFFFFFEu;   // none: only head and tail are above
    int need = take;
    uint32_t prefix = 0;
    int *const copy = copies + (threadIdx.x % kCopies) * kBins;
    for (int shift = 32 - kDigitBits, bits = kDigitBits; need > 0; bits = min(kDigitBits, shift), shift -= bits) {
      const uint32_t mask = (1u << bits) - 1;
      auto add = [&](uint32_t key) {
        if (key - 1u < 0xFFFFFFFEu && (shift + bits == 32 || (key >> (shift + bits)) == prefix)) atomicAdd(&copy[(key >> shift) & mask], 1);
      };
#pragma unroll
      for (int i = 0; i < kSelectRows; ++i) add(first_keys[i]);
      // the rows behind the first chunk, in an order that needs no sorting out: a batch ahead, whole lines
      const int begin = max(lo, kSelectChunk);
      auto load = [&](int base, float (&x)[kSelectRows]) {
#pragma unroll
        for (int i = 0; i < kSelectRows; ++i) {
          const int r = base + i * kSelectThreads + threadIdx.x;
          x[i] = r < hi ? w[r] : 0.f;
        }
      };
      float x[kSelectRows];
      if (begin < hi) load(begin, x);
      for (int base = begin; base < hi; base += kSelectChunk) {
        float ahead[kSelectRows];
        if (base + kSelectChunk < hi) load(base + kSelectChunk, ahead);
#pragma unroll
        for (int i = 0; i < kSelectRows; ++i)
          if (base + i * kSelectThreads + static_cast<int>(threadIdx.x) < hi) add(weight_key(x[i]));
#pragma unroll
        for (int i = 0; i < kSelectRows; ++i) x[i] = ahead[i];
      }
      __syncthreads();
      find_digit(copies, need, &s_digit, lds);
      const Digit d = s_digit;
      prefix = prefix << bits | static_cast<uint32_t>(d.digit);
      threshold = prefix << shift;
      rest = need = d.rest;
      if (d.rest == d.count) {   // all of the digit's keys are kept: no need to tell them apart
        threshold -= 1;          // (not below 0: a key is above 0)
        rest = need = 0;
      }
      if (shift == 0) break;
    }
  }

  // the list, in row order
  int listed = 0, equal = 0;
  for (int base = 0; base < own.len; base += kSelectChunk) {
    uint32_t key[kSelectRows];
#pragma unroll
    for (int i = 0; i < kSelectRows; ++i) key[i] = first_keys[i];
    if (base + kSelectChunk < own.len) load_keys(base + kSelectChunk, first_keys);   // the next chunk's, ahead
    int sure = 0, ties = 0;
#pragma unroll
    for (int i = 0; i < kSelectRows; ++i) {
      sure += key[i] > threshold;
      ties += rest > 0 && key[i] == threshold;
    }
    // a tie is kept while fewer than `rest` come before it
    const int x[2] = {sure, ties};
    int below[2], total[2];
    block_int_scan_n<kSelectThreads, 2>(x, below, total, lds);
    int tie_rank = equal + below[1];
    int at = listed + below[0] + min(tie_rank, rest) - min(equal, rest);
#pragma unroll
    for (int i = 0; i < kSelectRows; ++i) {
      const int r = base + mine + i;
      if (r < own.len) {
        const bool tie = rest > 0 && key[i] == threshold;
        if (key[i] > threshold || (tie && tie_rank < rest)) list[at++] = r;
        else if (at == r) s_first = r;   // the first dropped row: those before it stay where they are
        tie_rank += tie;
      }
    }
    listed += total[0] + min(equal + total[1], rest) - min(equal, rest);
    equal += total[1];
  }
  __syncthreads();
  if (threadIdx.x == 0) ws.req[b] = make_int2(own.kept, s_first);
}

// To another cache.  Grid (chunks of 16-byte units of the kept rows, requests).
template <typename SCALE>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(EvictCall c, EvictWs ws, int row_units, int scale_units) {
  if (ws.ctrl[0] == 0) return;
  const int b = blockIdx.y;
  const int kept = ws.req[b].x;
  if (kept < 0) return;
  const int32_t *list = ws.list + static_cast<size_t>(b) * c.max_rows;
  const size_t src0 = c.row_off[b], dst0 = c.out_row_off[b];
  const long first = static_cast<long>(blockIdx.x) * kMoveThreads + threadIdx.x, step = static_cast<long>(gridDim.x) * kMoveThreads;
  for (long j = first; j < kept; j += step) {
    const int r = list[j];
    c.out_weight[dst0 + j] = c.row_weight[src0 + r];
    if (c.keep_idx != nullptr) c.keep_idx[dst0 + j] = r;
  }
  const u32x4 *k = reinterpret_cast<const u32x4 *>(c.k), *v = reinterpret_cast<const u32x4 *>(c.v);
  u32x4 *ko = reinterpret_cast<u32x4 *>(c.k_out), *vo = reinterpret_cast<u32x4 *>(c.v_out);
  const long total = static_cast<long>(kept) * row_units;
  for (long u0 = first; u0 < total; u0 += step * kMoveUnroll) {
    u32x4 x[kMoveUnroll], y[kMoveUnroll];
#pragma unroll
    for (int i = 0; i < kMoveUnroll; ++i) {
      const long u = u0 + i * step;
      if (u < total) {
        const long j = u / row_units;
        const size_t src = (src0 + list[j]) * row_units + (u - j * row_units);
        x[i] = k[src];
        y[i] = v[src];
      }
    }
#pragma unroll
    for (int i = 0; i < kMoveUnroll; ++i) {
      const long u = u0 + i * step;
      if (u < total) {
        ko[dst0 * row_units + u] = x[i];
        vo[dst0 * row_units + u] = y[i];
      }
    }
  }
  if (scale_units > 0) {
    const SCALE *ks = reinterpret_cast<const SCALE *>(c.ks), *vs = reinterpret_cast<const SCALE *>(c.vs);
    SCALE *kso = reinterpret_cast<SCALE *>(c.ks_out), *vso = reinterpret_cast<SCALE *>(c.vs_out);
    const long n = static_cast<long>(kept) * scale_units;
    for (long u = first; u < n; u += step) {
      const long j = u / scale_units;
      const size_t src = (src0 + list[j]) * scale_units + (u - j * scale_units);
      kso[dst0 * scale_units + u] = ks[src];
      vso[dst0 * scale_units + u] = vs[src];
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) c.out_len[b] = kept;
}

// Rows first .. kept of one column (units [unit0, unit0 + units) of each row of `plane`), downwards in place.
template <typename UNIT>
__device__ __forceinline__ void walk_down(UNIT *plane, size_t row0, int row_units, int unit0, int units, const int32_t *list,
                                          int first, int kept) {
  const int rows = kWalkThreads / units;   // rows that the threads cover at once
  const int i = threadIdx.x / units, u = threadIdx.x % units;
  UNIT *p = plane + row0 * row_units + unit0 + u;
  int from[kWalkUnroll];
  auto look_up = [&](int j0) {
#pragma unroll
    for (int n = 0; n < kWalkUnroll; ++n) {
      const int j = j0 + n * rows + i;
      from[n] = i < rows && j < kept ? list[j] : -1;
    }
  };
  look_up(first);
  for (int j0 = first; j0 < kept; j0 += rows * kWalkUnroll) {
    UNIT x[kWalkUnroll];
    int to[kWalkUnroll];
#pragma unroll
    for (int n = 0; n < kWalkUnroll; ++n) {
      to[n] = from[n] < 0 ? -1 : j0 + n * rows + i;
      if (from[n] >= 0) x[n] = p[static_cast<size_t>(from[n]) * row_units];
    }
    look_up(j0 + rows * kWalkUnroll);
    // Every thread's loads of the batch come before any store behind the barrier (they need not have arrived: a
    // workgroup's accesses keep their order): rows below j0 + rows * kWalkUnroll may be overwritten.
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kWalkUnroll; ++n)
      if (to[n] >= 0) p[static_cast<size_t>(to[n]) * row_units] = x[n];
  }
}

// In place.  Grid (columns, requests): the columns of K, of V, of the scales of K and V, and the weights.
template <typename SCALE>
__global__ __launch_bounds__(kWalkThreads) void move_in_place_kernel(EvictCall c, EvictWs ws, int row_units, int col_units,
                                                                     int scale_units, int scale_col_units) {
  if (ws.ctrl[0] == 0) return;
  const int b = blockIdx.y;
  const int kept = ws.req[b].x, first = ws.req[b].y;
  if (kept < 0) return;
  const int32_t *list = ws.list + static_cast<size_t>(b) * c.max_rows;
  const size_t row0 = c.row_off[b];
  const int cols = (row_units + col_units - 1) / col_units;
  int col = blockIdx.x;
  if (col < 2 * cols) {
    u32x4 *plane = reinterpret_cast<u32x4 *>(const_cast<void *>(col < cols ? c.k : c.v));
    const int unit0 = col % cols * col_units;
    walk_down(plane, row0, row_units, unit0, min(col_units, row_units - unit0), list, first, kept);
    return;
  }
  col -= 2 * cols;
  const int scale_cols = scale_units > 0 ? (scale_units + scale_col_units - 1) / scale_col_units : 0;
  if (col < 2 * scale_cols) {
    SCALE *plane = reinterpret_cast<SCALE *>(const_cast<uint8_t *>(col < scale_cols ? c.ks : c.vs));
    const int unit0 = col % scale_cols * scale_col_units;
    walk_down(plane, row0, scale_units, unit0, min(scale_col_units, scale_units - unit0), list, first, kept);
    return;
  }
  walk_down(c.row_weight, row0, 1, 0, 1, list, first, kept);
  if (c.keep_idx != nullptr)
    for (int j = threadIdx.x; j < kept; j += kWalkThreads) c.keep_idx[row0 + j] = list[j];
  if (threadIdx.x == 0) c.cache_len[b] = kept;
}

template <typename SCALE>
static void launch_moves(const EvictCall &c, const EvictWs &ws, int row_units, int scale_units, hipStream_t stream) {
  if (c.k_out != nullptr) {
    const long units = static_cast<long>(c.max_rows) * row_units;
    const long chunks = std::max(1L, std::min((units + kMoveThreads * kMoveUnroll - 1) / (kMoveThreads * kMoveUnroll),
                                              std::max(16L, 4096L / c.batch)));
    move_kernel<SCALE><<<dim3(chunks, c.batch), dim3(kMoveThreads), 0, stream>>>(c, ws, row_units, scale_units);
  } else {
    // Columns of 128 bytes, or of 64 where that makes fewer than 64 workgroups.  An iteration of a workgroup moves
    // kWalkThreads * kWalkUnroll units and takes its time whatever their number; narrower columns than that have every
    // line fetched several times (1 request of 30,000 bf16 rows of 8 heads of 128 to 20,000: 16 bytes 215 us, 32 134,
    // 64 118, 128 125; 4 of 7,552 rows of 4 heads to 7,000: 131, 79, 55, 49).
    int col_units = 8;
    if (2L * c.batch * ((row_units + col_units - 1) / col_units) < 64) col_units = 4;
    const int scale_col_units = std::max(1, std::min(scale_units, c.batch < 16 ? 2 : 8));
    const int cols = (row_units + col_units - 1) / col_units, scale_cols = (scale_units + scale_col_units - 1) / scale_col_units;
    move_in_place_kernel<SCALE><<<dim3(2 * cols + 2 * scale_cols + 1, c.batch), dim3(kWalkThreads), 0, stream>>>(
        c, ws, row_units, col_units, scale_units, scale_col_units);
  }
}

hipError_t launch_evict(const EvictCall &c, const EvictWs &ws, int Hkv, int D, hipStream_t stream) {
  select_kernel<<<dim3(c.batch), dim3(kSelectThreads), 0, stream>>>(c, ws);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool q4 = c.ks != nullptr;
  const int row_units = Hkv * D / (q4 ? 32 : 8);   // of 16 bytes
  if (D == 128) launch_moves<uint32_t>(c, ws, row_units, q4 ? Hkv : 0, stream);
  else launch_moves<uint16_t>(c, ws, row_units, q4 ? Hkv : 0, stream);
  return hipGetLastError();
}

}  // namespace sonic
