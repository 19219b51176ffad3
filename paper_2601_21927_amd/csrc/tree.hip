// Drafted tokens over the compact cache: which tokens a drafted one sees, their attention, and the path that is kept.
//
// A request's drafted tokens ("nodes") form trees: parent[i] < i, -1 for a root, or a chain.  With r over the cache rows
// and over the nodes on i's path (itself and its ancestors),
//     out[i][h] = softmax_r(scale <q[i][h], k[r][g(h)]>) v[r][g(h)].
//
// A workgroup has a tile of q rows (node i and q-head g of a kv-head are row i G + g) and a range of the request's rows, in
// blocks of 32: first the cache's, then the nodes', so that a block is of one kind and the nodes' visibility in it is one
// word of the plan.  Per block and wave
//   scores   S^T (16 rows x 16 columns) = K . Q^T   v_mfma_f32_16x16x32_bf16
//   softmax  online, fp32, per column in the four lanes that hold it
//   values   O^T (d x 16 columns) += V^T . P^T      v_mfma_f32_16x16x32_bf16, depth 32: the block's rows
// K and V come by direct-to-LDS loads.  Up to 32 rows are one wave's columns, and the waves of a workgroup take blocks in
// turn, each with LDS of its own (tree_kernel); of more rows, waves with 32 each share the blocks (tree_wide_kernel).
// An fp32 output takes a probability in three bf16 values (2^-26 of it is left), a bf16 output in one: its rounding, with
// the sum taken over the rounded ones, is of the size of the output's own (1.2 to 1.3 times that in all).  Two would leave the
// output's alone and cost nothing where HBM bounds the call, but trees of 32 over eight caches of 1,328 rows 20.0 us instead of
// 17.7 and chains of 250 over four of 1,584 53 instead of 43; a caller who wants them takes fp32.
// Ranges of a request are joined by another kernel.
//
// Bound by, trees of 32 over eight caches of 1,328 rows (32 / 8 heads of 128, bf16 out, 17.7 us; the bytes alone 9.5, the
// products 4.6): 2.2 us until the first rows are asked for, eleven blocks a wave with one wave a SIMD, 2 us for the waves'
// join.  Long and wide ones by the sum of what the SIMDs do (chains of 250 over four caches of 1,584, 43 us: matrix cores 14,
// vector instructions 14, LDS 7 and waits for it; they overlap little, two waves a SIMD).  64 caches of 1,500 rows, trees of
// 16: HBM, 5.1 TB/s.
#include <algorithm>

#include "common.h"
#include "q4.h"
#include "scan.h"

namespace sonic {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16_t;
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kTreeBlock = 32;   // rows of a block: the bits of a word of the plan

// ------------------------------------------------------------------ the plan
// One workgroup per request, one thread per node.  A node's words start with itself and take in those of its ancestors
// by doubling: after round k they hold 2^k of them, and `up` is the one behind those.  At most eight rounds.  Up to 64 nodes
// are one wave, whose lanes exchange words and parents without LDS.  Bound by its chain of loads: 4 us.
template <bool WAVE>
__global__ __launch_bounds__(WAVE ? kWave : kMaxNodes) void tree_plan_kernel(const int32_t *__restrict__ cu, const int32_t *__restrict__ parent,
                                                                             int total, int max_nodes, int words, int2 *__restrict__ req,
                                                                             uint32_t *__restrict__ sees, int32_t *status) {
  const int b = blockIdx.x, i = threadIdx.x;
  const int s = cu[b], e = cu[b + 1];
  const int pending = __hip_atomic_load(status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  bool bad = s < 0 || e < s || e > total || e - s > max_nodes || (b == 0 && s != 0);
  const int n = bad ? 0 : e - s;
  int up = -1;
  if (i < n) {
    up = parent != nullptr ? parent[s + i] : i - 1;
    bad = up < -1 || up >= i;
  }
  // (one look for the workgroup: the first thread's)
  const int stop = pending != 0 && pending != SONIC_ERR_CAPACITY && i == 0 ? 2 : 0;
  int any;
  if constexpr (WAVE) any = (__any(bad) ? 1 : 0) | __builtin_amdgcn_readfirstlane(stop);
  else any = (__syncthreads_or(bad) ? 1 : 0) | (__syncthreads_or(stop) ? 2 : 0);
  if (any & 2) return;
  if (any & 1) {
    if (i == 0) {
      raise_step_status(status, SONIC_ERR_BAD_LAYOUT);
      req[b] = int2{0, 0};
    }
    return;
  }
  if (i == 0) req[b] = int2{s, n};
  uint32_t *mine = sees + static_cast<size_t>(s + i) * words;
  if (parent == nullptr) {
    for (int w = 0; i < n && w < words; ++w) mine[w] = i / 32 > w ? ~0u : i / 32 == w ? ~0u >> (31 - i % 32) : 0;
    return;
  }
  if constexpr (WAVE) {
    uint32_t low = i < 32 ? 1u << i : 0, high = i < 32 ? 0 : 1u << (i - 32);
    while (__any(up >= 0)) {
      const int from = max(up, 0);
      const uint32_t l = __shfl(static_cast<int>(low), from), h = __shfl(static_cast<int>(high), from);
      const int next = __shfl(up, from);
      if (up >= 0) low |= l, high |= h, up = next;
    }
    if (i < n) mine[0] = low;
    if (i < n && words > 1) mine[1] = high;
  } else {
    __shared__ uint32_t s_sees[kMaxNodes][kMaxNodes / 32 + 1];
    __shared__ int s_up[kMaxNodes];
    for (int w = 0; w < words; ++w) s_sees[i][w] = i / 32 == w ? 1u << (i % 32) : 0;
    s_up[i] = up;
    while (__syncthreads_or(up >= 0)) {
      const int from = max(up, 0), next = s_up[from];
      uint32_t more[kMaxNodes / 32];
#pragma unroll
      for (int w = 0; w < kMaxNodes / 32; ++w) more[w] = w < words && up >= 0 ? s_sees[from][w] : 0;
      __syncthreads();
      if (up >= 0) {
#pragma unroll
        for (int w = 0; w < kMaxNodes / 32; ++w)
          if (w < words) s_sees[i][w] |= more[w];
        up = next;
        s_up[i] = up;
      }
    }
    for (int w = 0; i < n && w < words; ++w) mine[w] = s_sees[i][w];
  }
}

hipError_t launch_tree_plan(int batch, int total, int max_nodes, const int32_t *cu, const int32_t *parent, TreePlan plan,
                            int32_t *status, hipStream_t stream) {
  int2 *req = const_cast<int2 *>(plan.req);
  uint32_t *sees = const_cast<uint32_t *>(plan.sees);
  if (max_nodes <= kWave) tree_plan_kernel<true><<<dim3(batch), dim3(kWave), 0, stream>>>(cu, parent, total, max_nodes, plan.words, req, sees, status);
  else tree_plan_kernel<false><<<dim3(batch), dim3(kMaxNodes), 0, stream>>>(cu, parent, total, max_nodes, plan.words, req, sees, status);
  return hipGetLastError();
}

// ------------------------------------------------------------------ attention
// What a workgroup of any of this file's kernels looks up of its request; nodes 0 where there is nothing to do.
struct TreeReq {
  int first, nodes, len;
  int64_t base;
};
__device__ __forceinline__ TreeReq tree_request(const TreeCall &c, int b) {
  const int2 r = c.plan.req[b];
  const int len = c.cache_len[b];
  const int64_t base = c.row_off[b];
  TreeReq t;
  t.first = __builtin_amdgcn_readfirstlane(r.x);
  t.nodes = __builtin_amdgcn_readfirstlane(r.y);
  t.len = __builtin_amdgcn_readfirstlane(len);
  t.base = base;
  // a plan of another call, or none: nothing outside of this call's rows
  if (t.first < 0 || t.nodes < 0 || t.nodes > c.max_nodes || t.first > c.total_nodes - t.nodes) t.nodes = 0;
  return t;
}

__device__ __forceinline__ uint32_t finite_halves(uint32_t w) {   // the halves of a word that hold a number
  return ((w & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
}

// Four outputs, d = dd .. dd + 3 of the row at element `at`.
__device__ __forceinline__ void tree_store(const TreeCall &c, size_t at, int dd, f32x4 o) {
  if (c.out_bf16) {
    *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(c.out) + at + dd) = __builtin_convertvector(o, bf16x4);
  } else {
    *reinterpret_cast<f32x4 *>(static_cast<float *>(c.out) + at + dd) = o;
  }
}

// Behind the store of four outputs of node i by this thread, where some output of the workgroup was no number although its
// scores were.  The nodes' V that are none went into the products as zero (tree_only_numbers), since zero times them would
// be none too, also for the nodes that do not see them: here they are looked at again.  And an infinite V of the cache
// comes out of the sums as NaN (a row past a block's end counts zero times, a probability's second value is negative for half
// of the rows): the rows' V are read again.  A column whose only values that are none are infinities of one sign
// gives that infinity.
__device__ __forceinline__ void tree_odd_values(const TreeCall &c, const TreeReq &r, int Hkv, int D, int kvh, int i, size_t at, int dd) {
  const size_t stride = static_cast<size_t>(Hkv) * D;
  const bool q4 = c.ks != nullptr;
  int found[4] = {0, 0, 0, 0};   // 1: +inf, 2: -inf, 4: NaN
  auto look = [&](const uint16_t *x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) found[e] |= x[e] == 0x7F80 ? 1 : x[e] == 0xFF80 ? 2 : (x[e] & 0x7FFF) > 0x7F80 ? 4 : 0;
  };
  bool none = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float o = c.out_bf16 ? bf16_lo(static_cast<const uint16_t *>(c.out)[at + dd + e]) : static_cast<const float *>(c.out)[at + dd + e];
    none = none || o != o;
  }
  if (none && !q4) {   // (4-bit rows hold no infinities)
    const uint16_t *col = static_cast<const uint16_t *>(c.v) + static_cast<size_t>(r.base) * stride + kvh * D + dd;
#pragma unroll 4
    for (int j = 0; j < r.len; ++j) look(col + j * stride);
  }
  const uint16_t *own = c.v_new + static_cast<size_t>(r.first) * stride + kvh * D + dd;
  const uint32_t *sees = c.plan.sees + static_cast<size_t>(r.first + i) * c.plan.words;
#pragma unroll 1
  for (int j = 0; j < r.nodes; ++j) {
    if (((sees[j / 32] >> (j % 32)) & 1) == 0) continue;
    const uint16_t *x = own + j * stride;
    if (!q4) {
      look(x);
    } else {   // all of the value's block is NaN
      x -= dd % kQ4Block;
#pragma unroll 1
      for (int e = 0; e < kQ4Block; ++e)
        if ((x[e] & 0x7F80) == 0x7F80) found[0] = found[1] = found[2] = found[3] = 4;
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (found[e] == 0) continue;
    const float o = found[e] == 1 ? INFINITY : found[e] == 2 ? -INFINITY : NAN;
    if (c.out_bf16) static_cast<uint16_t *>(c.out)[at + dd + e] = static_cast<uint16_t>(__float_as_uint(o) >> 16);
    else static_cast<float *>(c.out)[at + dd + e] = o;
  }
}

// Instruction order of a product of N operands read from LDS (READS reads each) with MFMAS products on each: the reads of
// the first AHEAD operands, then the products of one and the reads of one more at a time, so that the reads' latency passes
// behind the matrix cores (see order_reads_ahead).
template <int N, int READS, int MFMAS, int AHEAD> __device__ __forceinline__ void order_operands() {
  static_assert(AHEAD <= N, "lookahead within the block");
  __builtin_amdgcn_sched_group_barrier(0x100, READS * AHEAD, 0);
#pragma unroll
  for (int i = 0; i < N - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, MFMAS, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, MFMAS * AHEAD, 0);
}
constexpr int kAheadK = 4, kAheadV = 3;   // operands

// A wave's 16 CT columns of the attention: the running softmax and the output.
template <int D, int CT, int PARTS> struct TreeColumns {
  static constexpr int KS = D / 32;              // k steps of the score product
  static constexpr int DB = D / 16;              // 16-wide d blocks of the value product
  static constexpr int DC = D / 8;               // 16-byte chunks per row
  static constexpr int KSWZ = DC - 1;            // K in LDS: 16-byte chunk p of row r at p ^ (r & KSWZ)
  static constexpr int VSWZ = DC / 2 - 1;        // V in LDS: 32-byte segment s of row r at s ^ (r & VSWZ)
  f32x4 oacc[CT][DB];                            // lane (col, quarter): d = 16 db + 4 quarter .. + 3 of column 16 t + col
  float m_run[CT];                               // log2 domain, lagging by at most 8
  f32x4 lacc[CT];                                // the probabilities' sum, in every element: a product with ones, of the same
                                                 // rounded values as the output's (4 % faster than adding them up)

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      // (the lowest number: a block whose scores all passed the range below, -infinity, then weighs exp2(-infinity), 0)
      m_run[t] = -__FLT_MAX__;
      lacc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DB; ++i) oacc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Scores of the 32-row block of K at ktile: s[t][h][i] of row 16 h + 4 quarter + i.
  __device__ __forceinline__ static void scores(const uint16_t *ktile, const bf16x8 (&qf)[CT][KS], int col, int quarter, f32x4 (&s)[CT][2]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int t = 0; t < CT; ++t) s[t][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 a = *reinterpret_cast<const bf16x8 *>(ktile + (16 * h + col) * D + (((4 * ks + quarter) ^ (col & KSWZ)) * 8));
#pragma unroll
        for (int t = 0; t < CT; ++t) s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[t][ks], s[t][h], 0, 0, 0);
      }
    }
  }

  // The scores of NB blocks to probabilities.
  template <int NB>
  __device__ __forceinline__ void soften(const f32x4 (&s)[NB][CT][2], float scale_log2, bf16x8 (&pp)[NB][CT][PARTS]) {
    float top[CT];
    bool grows = false;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      top[t] = -INFINITY;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) top[t] = fmaxf(top[t], s[n][t][h][i]);
      top[t] = pair32_max(pair16_max(top[t])) * scale_log2;
      grows = grows || top[t] > m_run[t] + 8.f;
    }
    if (__any(grows)) {   // rescale only when a max grows by more than 2^8
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        const float m_new = fmaxf(m_run[t], top[t]);
        const float corr = __builtin_amdgcn_exp2f(m_run[t] - m_new);
        m_run[t] = m_new;
        lacc[t] *= corr;
#pragma unroll
        for (int i = 0; i < DB; ++i) oacc[t][i] *= corr;
      }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        f32x8 p;
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[n][t][i / 4][i % 4], scale_log2, -m_run[t]));
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          pp[n][t][k] = __builtin_convertvector(p, bf16x8);
          if (k + 1 < PARTS) less_rounded(p, pp[n][t][k]);
        }
      }
  }

  // p less its rounded values: v_dot2c_f32_bf16 against (-1, 0) and (0, -1) takes one of a pair off a number, exactly.
  __device__ __forceinline__ static void less_rounded(f32x8 &p, bf16x8 r) {
    uint32_t first = 0x0000BF80u, second = 0xBF800000u;
    asm("" : "+s"(first), "+s"(second));   // (as a literal the second one is taken for -1 in 32 bits)
    const bf16x2 low = __builtin_bit_cast(bf16x2, first), high = __builtin_bit_cast(bf16x2, second);
    const bf16x2 pair[4] = {__builtin_shufflevector(r, r, 0, 1), __builtin_shufflevector(r, r, 2, 3), __builtin_shufflevector(r, r, 4, 5),
                            __builtin_shufflevector(r, r, 6, 7)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[2 * i] = __builtin_amdgcn_fdot2_f32_bf16(pair[i], low, p[2 * i], false);
      p[2 * i + 1] = __builtin_amdgcn_fdot2_f32_bf16(pair[i], high, p[2 * i + 1], false);
    }
  }

  // The values of the 32-row block of V at vtile.
  __device__ __forceinline__ void add_values(const uint16_t *vtile, int col, int quarter, const bf16x8 (&pp)[CT][PARTS]) {
    const int tr_row = 4 * quarter + (col >> 2);
    const int tr_off = tr_row * D + 4 * (col & 3), tr_swz = tr_row & VSWZ;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const uint16_t *pa = vtile + tr_off + ((db ^ tr_swz) * 16);
      // C-style cast: the transposing read takes an LDS-qualified pointer
      const v4i16 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)pa);
      const v4i16 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t *)(pa + 16 * D));
      const bf16x8 aa = __builtin_bit_cast(bf16x8, __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int k = 0; k < PARTS; ++k) oacc[t][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aa, pp[t][k], oacc[t][db], 0, 0, 0);
    }
    const u32x4 one = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int k = 0; k < PARTS; ++k)
        lacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, one), pp[t][k], lacc[t], 0, 0, 0);
  }
};

// Scores of what a column does not see, s[t][h][i] of row 16 h + 4 quarter + i of block g: the nodes that are not on its
// node's path, and rows past the cache's end.  Called for blocks from r.len / 32 on.
template <int CT>
__device__ __forceinline__ void tree_mask(const TreeCall &c, const TreeReq &r, int g, int cached, const int (&node)[CT], int quarter,
                                          f32x4 (&s)[CT][2]) {
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    uint32_t word;
    if (g < cached) {
      const int left = r.len - g * kTreeBlock;
      word = left >= kTreeBlock ? ~0u : (1u << left) - 1;
    } else {   // (behind the last block, whose rows are loaded again, nothing is seen)
      word = g - cached < c.plan.words ? c.plan.sees[static_cast<size_t>(r.first + node[t]) * c.plan.words + g - cached] : 0;
    }
    word >>= 4 * quarter;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][h][i] = (word >> (16 * h + i)) & 1 ? s[t][h][i] : -INFINITY;
  }
}

// V of a block of nodes in LDS: what is no number becomes zero (see tree_odd_values).  Returns whether there was any.
template <int D> __device__ __forceinline__ bool tree_only_numbers(uint16_t *vtile, int lane) {
  bool here = false;
#pragma unroll
  for (int i = 0; i < kTreeBlock * D / 8 / kWave; ++i) {
    u32x4 *at = reinterpret_cast<u32x4 *>(vtile + (i * kWave + lane) * 8);
    const u32x4 w = *at;
    const u32x4 keep = {finite_halves(w[0]), finite_halves(w[1]), finite_halves(w[2]), finite_halves(w[3])};
    const bool bad = (keep[0] & keep[1] & keep[2] & keep[3]) != ~0u;
    if (bad) *at = w & keep;
    here = here || bad;
  }
  return __any(here);
}

// The parts of KW waves with the same columns to one, and out: to the output, or to the range's partial.  Each wave takes
// its share of the d blocks and gets the others' through LDS (`lds`: a wave's columns at wave * CT * DB * 64 values of 16
// bytes; `stat`: [wave][CT][16] (max, sum)).  The parts of wave `wave` are those of waves wave % RW + RW k.
// Returns whether an output of the workgroup is no number although its scores were; then, unless `careful`, nothing is
// written.  `odd`: V of a node is no number.
template <int D, int CT, int PARTS, int RW, int KW>
__device__ __forceinline__ bool tree_finish(TreeColumns<D, CT, PARTS> &cols, const TreeCall &c, const TreeReq &r, f32x4 *lds, float2 *stat,
                                            int wave, int lane, int row0, int rows, int Hkv, int G, int kvh, bool whole, bool careful, bool odd,
                                            float *acc, float2 *acc_stat) {
  constexpr int DB = D / 16, MINE = (DB + KW - 1) / KW;   // (of more waves than d blocks, some take none)
  const int col = lane & 15, quarter = lane >> 4, kg = wave / RW, rg = wave % RW;
  float l[CT], weight[CT][KW];
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    l[t] = cols.lacc[t][0];
    weight[t][0] = 1.f;
  }
  if constexpr (KW > 1) {
    __syncthreads();   // every wave is done with its blocks
#pragma unroll
    for (int t = 0; t < CT; ++t) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (db / MINE != kg) lds[((wave * CT + t) * DB + db) * kWave + lane] = cols.oacc[t][db];
      if (quarter == 0) stat[(wave * CT + t) * 16 + col] = float2{cols.m_run[t], l[t]};
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      float2 s[KW];
      float M = -__FLT_MAX__, L = 0.f;
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        s[k] = stat[((rg + RW * k) * CT + t) * 16 + col];
        M = fmaxf(M, s[k].x);
      }
#pragma unroll
      for (int k = 0; k < KW; ++k) {
        weight[t][k] = __builtin_amdgcn_exp2f(s[k].x - M);
        L = fmaf(weight[t][k], s[k].y, L);
      }
      cols.m_run[t] = M;
      l[t] = L;
    }
  }
  bool none = false;
#pragma unroll
  for (int t = 0; t < CT; ++t) {
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
      f32x4 A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KW; ++k)   // the waves in order, so that the sum does not depend on which of them takes the block
#pragma unroll
        for (int own = 0; own < KW && own * MINE < DB; ++own)
          if (own == kg) {
            const int db = own * MINE + m;
            const f32x4 a = k == own ? cols.oacc[t][db] : lds[(((rg + RW * k) * CT + t) * DB + db) * kWave + lane];
            if constexpr (KW > 1) {
#pragma unroll
              for (int e = 0; e < 4; ++e) A[e] = fmaf(weight[t][k], a[e], A[e]);
            } else {
              A = a;
            }
          }
      cols.oacc[t][m] = A;   // (behind the last use of what it held: a wave's blocks come first)
      const float all_of = (A[0] + A[1]) + (A[2] + A[3]);
      none = none || (all_of != all_of && l[t] == l[t] && row0 + 16 * t + col < rows);
    }
  }
  odd = __syncthreads_or(none || odd);
  if (odd && !careful) return true;
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const int cc = 16 * t + col, row = row0 + cc;
    if (row >= rows || kg * MINE >= DB) continue;
    if (whole) {
      const int i = row / G;
      const size_t at = (static_cast<size_t>(r.first + i) * Hkv * G + kvh * G + row % G) * D;
      const float inv = 1.f / l[t];
#pragma unroll
      for (int m = 0; m < MINE; ++m) tree_store(c, at, (kg * MINE + m) * 16 + 4 * quarter, cols.oacc[t][m] * inv);
      if (__builtin_expect(odd, 0) && l[t] == l[t])
#pragma unroll 1
        for (int m = 0; m < MINE; ++m) tree_odd_values(c, r, Hkv, D, kvh, i, at, (kg * MINE + m) * 16 + 4 * quarter);
    } else {
#pragma unroll
      for (int m = 0; m < MINE; ++m) *reinterpret_cast<f32x4 *>(acc + cc * D + (kg * MINE + m) * 16 + 4 * quarter) = cols.oacc[t][m];
      if (kg == 0 && quarter == 0) acc_stat[cc] = float2{cols.m_run[t], odd ? -l[t] : l[t]};   // (it has no sign of its own)
    }
  }
  return false;
}

// What the workgroups of an attention call start with: its place in the call, the request, and what there is to do.
struct TreePlace {
  int kvh, rt, split, rows, cached, blocks, first, last;   // (split, first, last: of a tile of up to 32 rows)
  bool whole;        // the request is one range
  TreeReq r;
  float *acc;        // else the range's partial: the values, ..
  float2 *stat;      // .. and (max, sum), of COLS columns
};
// False: nothing to do.  The row tiles of one range are neighbours on one XCD (workgroup i goes to XCD i % 8): its rows come
// from that L2 after the first.  So are 2^run_log2 of its kv-heads.
template <int D, int COLS>
__device__ __forceinline__ bool tree_begin(const TreeCall &c, const TreeShape &sh, float *part, int Hkv, int G, TreePlace *p) {
  __shared__ int s_stop;
  constexpr bool RANGES = COLS <= 32;   // (tiles of more rows are not cut: see tree_shape)
  const unsigned turn = blockIdx.x / kNumXcd, xcd = blockIdx.x % kNumXcd, splits = RANGES ? sh.splits : 1;
  const unsigned at = turn / sh.tiles, unit = ((((at >> sh.run_log2) * kNumXcd + xcd) << sh.run_log2) + (at & ((1u << sh.run_log2) - 1)));
  if (unit >= static_cast<unsigned>(c.batch) * Hkv * splits) return false;
  p->rt = turn % sh.tiles;
  p->kvh = unit % Hkv;
  p->split = unit / Hkv % splits;
  const int b = unit / Hkv / splits;
  if (threadIdx.x == 0) s_stop = step_stops(c.status);   // one look for the workgroup
  p->r = tree_request(c, b);
  __syncthreads();
  const bool stop = s_stop != 0;
  p->rows = p->r.nodes * G;                              // q rows of the request
  if (p->rt * COLS >= p->rows) return false;
  if (p->r.len < 0 || p->r.len > c.max_ctx) {            // uniform over the request: no output
    if (threadIdx.x == 0 && p->rt == 0 && p->kvh == 0 && p->split == 0) raise_status(c.status, SONIC_ERR_CAPACITY);
    return false;
  }
  p->cached = (p->r.len + kTreeBlock - 1) / kTreeBlock;  // blocks of the cache, then of the nodes
  p->blocks = p->cached + (p->r.nodes + kTreeBlock - 1) / kTreeBlock;
  p->first = 0, p->last = p->blocks;
  p->whole = true;
  p->acc = nullptr, p->stat = nullptr;
  if constexpr (!RANGES) return !stop;
  p->first = p->split * sh.range;
  p->last = min(p->blocks, p->first + sh.range);
  if (p->first >= p->blocks) return false;
  p->whole = p->blocks <= sh.range;
  const size_t slot = ((static_cast<size_t>(b) * Hkv + p->kvh) * sh.tiles + p->rt) * sh.splits + p->split;
  const size_t slots = static_cast<size_t>(c.batch) * Hkv * sh.tiles * sh.splits;
  p->acc = part + slot * (COLS * D);
  p->stat = reinterpret_cast<float2 *>(part + slots * (COLS * D)) + slot * COLS;
  if (stop) {   // another workgroup of the call may have seen no error: what it left is not to be joined with this one's
    if (!p->whole && threadIdx.x < COLS) p->stat[threadIdx.x] = float2{0.f, -INFINITY};
    return false;
  }
  return true;
}

// Q^T fragments (B operand of the scores) of the 16 CT rows from row0 on: lane (col, quarter) has d = 32 ks + 8 quarter .. + 7 of
// its row, or, BY_QUARTERS, d = quarter D / 4 + 8 ks ..; and the rows' nodes.  Rows past the end are the last one again.
template <int D, int CT, bool BY_QUARTERS>
__device__ __forceinline__ void tree_queries(const TreeCall &c, const TreePlace &p, int Hkv, int G, int row0, int lane, bf16x8 (&qf)[CT][D / 32],
                                             int (&node)[CT]) {
  const int col = lane & 15, quarter = lane >> 4;
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const int row = min(row0 + 16 * t + col, p.rows - 1);
    node[t] = row / G;
    const uint16_t *src = c.q + (static_cast<size_t>(p.r.first + node[t]) * Hkv * G + p.kvh * G + row % G) * D +
                          (BY_QUARTERS ? quarter * (D / 4) : 8 * quarter);
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) qf[t][ks] = *reinterpret_cast<const bf16x8 *>(src + (BY_QUARTERS ? 8 : 32) * ks);
  }
}
// The fragments are waited for where this stands: in the loop the wait would drain the loads ahead.
template <int CT, int KS> __device__ __forceinline__ void tree_wait(bf16x8 (&qf)[CT][KS]) {
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[t][ks]));
}

// Up to 32 q rows: the NW waves take the range's blocks in turn, each with K and V of its own in LDS.
template <int D, int CT, int NW, bool Q4, int PARTS>
__global__ __launch_bounds__(NW *kWave, 2) void tree_kernel(TreeCall c, TreeShape sh, float *__restrict__ part, int Hkv, int G) {
  constexpr int KS = D / 32, DB = D / 16, DC = D / 8, BR = kTreeBlock;
  constexpr int NI = BR * DC / kWave;            // direct-to-LDS instructions per tensor and block
  constexpr int KSWZ = TreeColumns<D, CT, PARTS>::KSWZ, VSWZ = TreeColumns<D, CT, PARTS>::VSWZ;
  constexpr int COLS = 16 * CT;
  constexpr int TILE = BR * D;                   // elements of one tensor's block
  constexpr int RING = (Q4 ? 1 : 2) * TILE;      // 4-bit rows: V alone, as bf16
  constexpr int JOIN = CT * DB * kWave * 8;      // a wave's part of the join (in 16-bit elements)
  __shared__ __align__(16) uint16_t lds[NW * (RING > JOIN ? RING : JOIN)];
  __shared__ float2 stat[NW * COLS];
  TreePlace p;
  if (!tree_begin<D, COLS>(c, sh, part, Hkv, G, &p)) return;
  const TreeReq &r = p.r;
  const int cached = p.cached, blocks = p.blocks, kvh = p.kvh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int col = lane & 15, quarter = lane >> 4;
  bf16x8 qf[CT][KS];
  int node[CT];
  tree_queries<D, CT, Q4>(c, p, Hkv, G, p.rt * COLS, lane, qf, node);
  TreeColumns<D, CT, PARTS> cols;
  const size_t row_elems = static_cast<size_t>(Hkv) * D;
  const uint16_t *knew = c.k_new + static_cast<size_t>(r.first) * row_elems + kvh * D;
  const uint16_t *vnew = c.v_new + static_cast<size_t>(r.first) * row_elems + kvh * D;
  uint16_t *const vtile = lds + wave * RING + (Q4 ? 0 : TILE);
  const int full = r.len / BR;                   // blocks without a row that some column does not see
  bool careful = false, odd = false;

  // A block's scores into the output.  `ready`: V of the block is in vtile when it returns.
  auto block = [&](int g, f32x4 (&s)[1][CT][2], auto ready) {
    if (__builtin_expect(g >= full, 0)) tree_mask<CT>(c, r, g, cached, node, quarter, s[0]);
    bf16x8 pp[1][CT][PARTS];
    cols.soften(s, c.scale_log2, pp);
    ready();
    if (__builtin_expect(careful, 0) && g >= cached) odd = tree_only_numbers<D>(vtile, lane) || odd;
    cols.add_values(vtile, col, quarter, pp[0]);
    order_operands<DB, 2, CT * PARTS, kAheadV>();
  };

again:
  cols.clear();
  if constexpr (!Q4) {
    uint16_t *const ktile = lds + wave * RING;
    const uint32_t klds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint16_t *)ktile));
    const uint16_t *kbase = static_cast<const uint16_t *>(c.k) + static_cast<size_t>(r.base) * row_elems + kvh * D;
    const uint16_t *vbase = static_cast<const uint16_t *>(c.v) + static_cast<size_t>(r.base) * row_elems + kvh * D;
    const uint32_t row_bytes = row_elems * 2;
    // Block g's rows to LDS: lane -> (row, 16-byte position) of each instruction; the position holds the row's swizzled
    // chunk.  Rows past the end, and blocks past the last, load a row again: every block issues the same loads, so that
    // the waits can be counted.
    auto issue = [&](int g, const uint16_t *cache, const uint16_t *fresh, uint32_t to, bool is_v) {
      g = min(g, blocks - 1);
      const int r0 = (g < cached ? g : g - cached) * BR;
      const int left = (g < cached ? r.len : r.nodes) - r0;
      const char *src = reinterpret_cast<const char *>(g < cached ? cache : fresh) + static_cast<size_t>(r0) * row_bytes;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int rl = (i * kWave + lane) / DC, pos = (i * kWave + lane) % DC;
        dma_row16_s(src, min(rl, left - 1) * row_bytes + (pos ^ (is_v ? 2 * (rl & VSWZ) : rl & KSWZ)) * 16, to + i * kWave * 16);
      }
    };
    auto issue_k = [&](int g) { issue(g, kbase, knew, klds, false); };
    auto issue_v = [&](int g) { issue(g, vbase, vnew, klds + TILE * 2, true); };
    int g = p.first + wave;
    if (g < p.last) {
      issue_k(g);
      issue_v(g);
      tree_wait(qf);
      for (; g < p.last; g += NW) {
        wait_vm<NI>();   // K is there; V may not be
        f32x4 s[1][CT][2];
        cols.scores(ktile, qf, col, quarter, s[0]);
        order_operands<2 * KS, 1, CT, kAheadK>();
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // lgkmcnt(0): K may be overwritten
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        issue_k(g + NW);
        block(g, s, [&]() {
          wait_vm<NI>();   // V is there; the next K may not be
          __atomic_signal_fence(__ATOMIC_SEQ_CST);
        });
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        issue_v(g + NW);
      }
      wait_vm<0>();   // the loads behind the last block
    }
  } else {
    // K stays in registers: lane (col, quarter) decodes a quarter of row col, D / 4 values, into the operand; V goes through
    // LDS as bf16 for the transposing reads.  A node's row is rounded as its append would.
    constexpr int LV = D / kQ4Block;             // lanes that hold a row of V, a quantisation block each
    constexpr int NV = BR * LV / kWave;          // ... and loads of a block's V
    constexpr int CW = D / 32;                   // words of a lane's K codes, eight each
    typedef uint32_t codes_t __attribute__((ext_vector_type(CW)));
    const size_t row_codes = static_cast<size_t>(Hkv) * (D / 2), row_scales = static_cast<size_t>(Hkv) * (D / kQ4Block);
    auto plane = [&](const void *p, size_t row) { return static_cast<const uint8_t *>(p) + static_cast<size_t>(r.base) * row + kvh * (row / Hkv); };
    const uint8_t *kcode = plane(c.k, row_codes), *vcode = plane(c.v, row_codes);
    const uint8_t *kscale = plane(c.ks, row_scales), *vscale = plane(c.vs, row_scales);
    const int k_blk = quarter * LV / 4, v_blk = lane % LV, v_row = lane / LV;
    struct KRaw { codes_t c[2]; uint32_t s[2]; };
    struct VRaw { u32x4 c[NV]; uint32_t s[NV]; };
    auto fetch_k = [&](int g) {
      KRaw x;
      if (g < cached) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const size_t row = min(g * BR + 16 * h + col, r.len - 1);
          x.c[h] = *reinterpret_cast<const codes_t *>(kcode + row * row_codes + 4 * CW * quarter);
          x.s[h] = kscale[row * row_scales + k_blk];
        }
      } else if (g < blocks) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const size_t row = min((g - cached) * BR + 16 * h + col, r.nodes - 1);
          const uint16_t *src = knew + row * row_elems + quarter * (D / 4);
          uint32_t w[4 * CW];
#pragma unroll
          for (int k = 0; k < CW; ++k) {
            const u32x4 y = *reinterpret_cast<const u32x4 *>(src + 8 * k);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * k + e] = y[e];
          }
          uint32_t top = q4_top(w);
          if (D / 4 < kQ4Block) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16)));   // half a block here
          x.s[h] = q4_scale_byte(top);
#pragma unroll
          for (int k = 0; k < CW; ++k) x.c[h][k] = q4_encode8(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3], x.s[h]);
        }
      }
      return x;
    };
    auto fetch_v = [&](int g) {
      VRaw x;
#pragma unroll
      for (int t = 0; t < NV; ++t) {
        const int at = kWave / LV * t + v_row;
        if (g < cached) {
          const int row = min(g * BR + at, r.len - 1);
          x.c[t] = *reinterpret_cast<const u32x4 *>(vcode + row * row_codes + 16 * v_blk);
          x.s[t] = vscale[row * row_scales + v_blk];
        } else if (g < blocks) {
          const size_t row = min((g - cached) * BR + at, r.nodes - 1);
          const uint16_t *src = vnew + row * row_elems + kQ4Block * v_blk;
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const u32x4 y = *reinterpret_cast<const u32x4 *>(src + 8 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * i + e] = y[e];
          }
          x.s[t] = q4_scale_byte(q4_top(w));
#pragma unroll
          for (int i = 0; i < 4; ++i) x.c[t][i] = q4_encode8(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3], x.s[t]);
        }
      }
      return x;
    };
    int g = p.first + wave;
    if (g < p.last) {
      KRaw k_raw = fetch_k(g);
      VRaw v_raw = fetch_v(g);
      tree_wait(qf);
      for (; g < p.last; g += NW) {
        f32x4 s[1][CT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int t = 0; t < CT; ++t) s[0][t][h] = f32x4{0.f, 0.f, 0.f, 0.f};
          const float scale = q4_scale(k_raw.s[h]);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const bf16x8 a = q4_decode8(k_raw.c[h][ks], scale);
#pragma unroll
            for (int t = 0; t < CT; ++t) s[0][t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[t][ks], s[0][t][h], 0, 0, 0);
          }
        }
        k_raw = fetch_k(g + NW);
        block(g, s, [&]() {
          const int left = (g < cached ? r.len - g * BR : r.nodes - (g - cached) * BR);
#pragma unroll
          for (int t = 0; t < NV; ++t) {
            const int row = kWave / LV * t + v_row;
            const float vs = row < left ? q4_scale(v_raw.s[t]) : 1.f;   // (a NaN would stay one under its weight of zero)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<bf16x8 *>(vtile + row * D + ((2 * v_blk + i / 2) ^ (row & VSWZ)) * 16 + (i & 1) * 8) =
                  q4_decode8(v_raw.c[t][i], vs);
          }
          v_raw = fetch_v(g + NW);
        });
      }
    }
  }

  if (tree_finish<D, CT, PARTS, 1, NW>(cols, c, r, reinterpret_cast<f32x4 *>(lds), stat, wave, lane, p.rt * COLS, p.rows, Hkv, G, kvh,
                                               p.whole, careful, odd, p.acc, p.stat)) {
    careful = true;   // once more, the nodes' V with a look
    __syncthreads();
    goto again;
  }
}

// More than 32 q rows: RW waves with 32 of them each share the blocks in LDS, KW = NW / RW such groups take the NW / 2 blocks of
// a step between them.  While a step is computed the next one's rows stream into the other buffers, NJ direct-to-LDS loads a
// wave and tensor, also past the end (there the last block again).  One barrier a step, before its rows are read: a second one
// behind the scores, with K a step further ahead, left the waves less room (64 requests of 180 .. 4,300 rows: 115 us, this
// way 109).  4-bit rows are decoded on the way: the codes of a step ahead wait in registers, one quantisation block a lane.
template <int D, int RW, int NW, bool Q4, int PARTS>
__global__ __launch_bounds__(NW *kWave, 2) void tree_wide_kernel(TreeCall c, TreeShape sh, int Hkv, int G) {
  typedef TreeColumns<D, 2, PARTS> Columns;
  constexpr int CT = 2, KS = D / 32, DB = D / 16, DC = D / 8, BR = kTreeBlock;
  constexpr int KW = NW / RW, SB = NW / 2, NB = SB / KW;   // key groups; blocks of a step, and of them a wave's
  constexpr int NI = BR * DC / kWave;                // direct-to-LDS instructions per tensor and block
  constexpr int NJ = SB * NI / NW;                   // ... and of a wave per tensor and step
  constexpr int COLS = 32 * RW;
  constexpr int TILE = BR * D;
  static_assert(NB * KW == SB && NI % NJ == 0, "a step is whole blocks; a wave loads from one of them");
  static_assert(NW * CT * DB * kWave * 8 <= 4 * SB * TILE, "the join fits");
  __shared__ __align__(16) uint16_t lds[4 * SB * TILE];   // K of two steps, V of two steps
  __shared__ float2 stat[NW * 32];
  TreePlace p;
  if (!tree_begin<D, COLS>(c, sh, nullptr, Hkv, G, &p)) return;
  const TreeReq &r = p.r;
  const int cached = p.cached, blocks = p.blocks, kvh = p.kvh;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int rg = wave % RW, kg = wave / RW;
  const int col = lane & 15, quarter = lane >> 4;
  const int row0 = p.rt * COLS + 32 * rg;
  const bool rowless = row0 >= p.rows;               // such a wave only stages
  bf16x8 qf[CT][KS];
  int node[CT];
  tree_queries<D, CT, false>(c, p, Hkv, G, row0, lane, qf, node);
  Columns cols;
  const size_t row_elems = static_cast<size_t>(Hkv) * D;
  const uint16_t *knew = c.k_new + static_cast<size_t>(r.first) * row_elems + kvh * D;
  const uint16_t *vnew = c.v_new + static_cast<size_t>(r.first) * row_elems + kvh * D;
  uint16_t *const kbuf = lds, *const vbuf = lds + 2 * SB * TILE;   // [2 steps][SB blocks][32 rows][D]
  const int steps = (blocks + SB - 1) / SB;
  const int full = r.len / BR;                       // blocks without a row that some column does not see
  bool careful = false, odd = false;

  auto compute = [&](int step) {
    if (rowless) return;
    const uint16_t *kt = kbuf + (step & 1) * SB * TILE;
    uint16_t *vt = vbuf + (step & 1) * SB * TILE;
    f32x4 s[NB][CT][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) cols.scores(kt + (KW * n + kg) * TILE, qf, col, quarter, s[n]);
    order_operands<NB * 2 * KS, 1, CT, kAheadK>();
    const int g = SB * step + kg;
    if (__builtin_expect(g + KW * (NB - 1) >= full, 0))
#pragma unroll
      for (int n = 0; n < NB; ++n) tree_mask<CT>(c, r, g + KW * n, cached, node, quarter, s[n]);
    bf16x8 pp[NB][CT][PARTS];
    cols.soften(s, c.scale_log2, pp);
    if (__builtin_expect(careful, 0))
#pragma unroll 1
      for (int n = 0; n < NB; ++n)   // (every wave for itself: the same values)
        if (g + KW * n >= cached) odd = tree_only_numbers<D>(vt + (KW * n + kg) * TILE, lane) || odd;
#pragma unroll
    for (int n = 0; n < NB; ++n) cols.add_values(vt + (KW * n + kg) * TILE, col, quarter, pp[n]);
    order_operands<NB * DB, 2, CT * PARTS, kAheadV>();
  };

again:
  cols.clear();
  if constexpr (!Q4) {
    const uint16_t *kbase = static_cast<const uint16_t *>(c.k) + static_cast<size_t>(r.base) * row_elems + kvh * D;
    const uint16_t *vbase = static_cast<const uint16_t *>(c.v) + static_cast<size_t>(r.base) * row_elems + kvh * D;
    const uint32_t row_bytes = row_elems * 2;
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint16_t *)lds)) +
                        wave * NJ * kWave * 16;
    auto issue = [&](int step, const uint16_t *cache, const uint16_t *fresh, uint32_t to, bool is_v) {
      const int g = min(SB * step + wave * NJ / NI, blocks - 1);
      const int r0 = (g < cached ? g : g - cached) * BR;
      const int left = (g < cached ? r.len : r.nodes) - r0;
      const char *src = reinterpret_cast<const char *>(g < cached ? cache : fresh) + static_cast<size_t>(r0) * row_bytes;
#pragma unroll
      for (int i = 0; i < NJ; ++i) {
        const int rl = ((wave * NJ % NI + i) * kWave + lane) / DC, pos = lane % DC;
        dma_row16_s(src, min(rl, left - 1) * row_bytes + (pos ^ (is_v ? 2 * (rl & Columns::VSWZ) : rl & Columns::KSWZ)) * 16,
                    to + (step & 1) * (2 * SB * TILE) + i * kWave * 16);
      }
    };
    auto issue_k = [&](int step) { issue(step, kbase, knew, at, false); };
    auto issue_v = [&](int step) { issue(step, vbase, vnew, at + 4 * SB * TILE, true); };
    issue_k(0);
    issue_v(0);
    tree_wait(qf);
    for (int step = 0; step < steps; ++step) {
      wait_vm<0>();
      lds_barrier();   // the step's rows are there; every wave is past the one before
      issue_k(step + 1);
      issue_v(step + 1);
      compute(step);
    }
    wait_vm<0>();
  } else {
    constexpr int LV = D / kQ4Block, HALF = D == 64 ? 2 : 1;   // a lane has a block of K and one of V, or (d = 64) one of either
    const size_t row_codes = static_cast<size_t>(Hkv) * (D / 2), row_scales = static_cast<size_t>(Hkv) * LV;
    const int item = threadIdx.x % (NW * kWave / HALF), row = item / LV, blk = item % LV;
    const bool does_v = HALF == 1 || threadIdx.x >= NW * kWave / 2;
    const size_t code0 = static_cast<size_t>(r.base) * row_codes + kvh * (D / 2) + 16 * blk;
    const size_t scale0 = static_cast<size_t>(r.base) * row_scales + kvh * LV + blk;
    struct Raw { u32x4 c; uint32_t s; };
    auto fetch = [&](int step, const void *codes, const uint8_t *scales, const uint16_t *fresh) {
      Raw x;
      const int g = min(SB * step + row / BR, blocks - 1);
      if (g < cached) {
        const size_t at = min(g * BR + row % BR, r.len - 1);
        x.c = *reinterpret_cast<const u32x4 *>(static_cast<const uint8_t *>(codes) + code0 + at * row_codes);
        x.s = scales[scale0 + at * row_scales];
      } else {   // a node's row is rounded as its append would
        const size_t at = min((g - cached) * BR + row % BR, r.nodes - 1);
        const uint16_t *src = fresh + at * row_elems + kQ4Block * blk;
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 y = *reinterpret_cast<const u32x4 *>(src + 8 * i);
#pragma unroll
          for (int e = 0; e < 4; ++e) w[4 * i + e] = y[e];
        }
        x.s = q4_scale_byte(q4_top(w));
#pragma unroll
        for (int i = 0; i < 4; ++i) x.c[i] = q4_encode8(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3], x.s);
      }
      return x;
    };
    Raw kq, vq;
    auto fetch_both = [&](int step) {
      if (HALF == 1 || !does_v) kq = fetch(step, c.k, c.ks, knew);
      if (does_v) vq = fetch(step, c.v, c.vs, vnew);
    };
    auto put = [&](int step) {
      if (HALF == 1 || !does_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<bf16x8 *>(kbuf + (step & 1) * SB * TILE + row * D + ((4 * blk + i) ^ (row & Columns::KSWZ)) * 8) =
              q4_decode8(kq.c[i], q4_scale(kq.s));
      }
      if (does_v) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<bf16x8 *>(vbuf + (step & 1) * SB * TILE + row * D + ((2 * blk + i / 2) ^ (row & Columns::VSWZ)) * 16 + (i & 1) * 8) =
              q4_decode8(vq.c[i], q4_scale(vq.s));
      }
    };
    fetch_both(0);
    put(0);
    fetch_both(1);
    tree_wait(qf);
    for (int step = 0; step < steps; ++step) {
      lds_barrier();   // the step's rows are there; every wave is past the one before
      put(step + 1);
      fetch_both(step + 2);
      compute(step);
    }
  }

  if (tree_finish<D, CT, PARTS, RW, KW>(cols, c, r, reinterpret_cast<f32x4 *>(lds), stat, wave, lane, row0, p.rows, Hkv, G, kvh, true, careful,
                                        odd, nullptr, nullptr)) {
    careful = true;   // once more, the nodes' V with a look
    __syncthreads();
    goto again;
  }
}

// The ranges of a request joined by log-sum-exp.  Grid (rows of a kv-head / rows a workgroup has, kv-heads, requests).  A
// thread has four values of a row and every sh.groups-th range of it; the groups' parts meet in LDS.  The first ranges are
// loaded before the request is looked up: their places do not depend on it.  16 ranges of 52 rows a kv-head: 4.2 us, a launch
// and two round trips.
constexpr int kJoinThreads = 256, kJoinAhead = 4;
template <int D>
__global__ __launch_bounds__(kJoinThreads) void tree_join_kernel(TreeCall c, TreeShape sh, const float *__restrict__ part, int G) {
  constexpr int LANES = D / 4, SLOTS = kJoinThreads / LANES;
  __shared__ f32x4 s_acc[kJoinThreads];
  __shared__ float2 s_stat[SLOTS];
  __shared__ int s_odd;
  const int b = blockIdx.z, kvh = blockIdx.y, Hkv = gridDim.y, COLS = 16 * sh.columns;
  const int place = threadIdx.x / LANES, group = place % sh.groups, dd = 4 * (threadIdx.x % LANES);
  const int row = blockIdx.x * (SLOTS / sh.groups) + place / sh.groups;
  const size_t slot = ((static_cast<size_t>(b) * Hkv + kvh) * sh.tiles + min(row / COLS, sh.tiles - 1)) * sh.splits;
  const size_t slots = static_cast<size_t>(c.batch) * Hkv * sh.tiles * sh.splits;
  const float *acc = part + (slot * COLS + row % COLS) * D + dd;
  const float2 *stat = reinterpret_cast<const float2 *>(part + slots * COLS * D) + slot * COLS + row % COLS;
  float2 ml[kJoinAhead];
  f32x4 a[kJoinAhead];
  auto load = [&](int s0) {
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      const size_t s = min(s0 + i * sh.groups, sh.splits - 1);
      ml[i] = stat[s * COLS];
      a[i] = *reinterpret_cast<const f32x4 *>(acc + s * COLS * D);
    }
  };
  load(group);
  if (threadIdx.x == 0) s_odd = 0;
  const TreeReq r = tree_request(c, b);
  const int blocks = (r.len + kTreeBlock - 1) / kTreeBlock + (r.nodes + kTreeBlock - 1) / kTreeBlock;
  if (blockIdx.x * (SLOTS / sh.groups) >= r.nodes * G || r.len < 0 || r.len > c.max_ctx || blocks <= sh.range) return;
  // (nobody writes the places of rows past the request's last: a thread that stands there has no ranges, whatever they hold)
  const int splits = row < r.nodes * G ? (blocks + sh.range - 1) / sh.range : 0;
  float M = -INFINITY, L = 0.f;
  bool odd = false, stopped = false;
  f32x4 A = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = group; s0 < splits; s0 += kJoinAhead * sh.groups) {
    if (s0 != group) load(s0);
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      if (s0 + i * sh.groups >= splits) break;
      stopped = stopped || ml[i].y == -INFINITY;   // a workgroup that had been stopped
      odd = odd || (__float_as_uint(ml[i].y) >> 31) != 0;
      const float top = fmaxf(M, ml[i].x), old = __builtin_amdgcn_exp2f(M - top), weight = __builtin_amdgcn_exp2f(ml[i].x - top);
      M = top;
      L = fmaf(weight, fabsf(ml[i].y), L * old);
#pragma unroll
      for (int e = 0; e < 4; ++e) A[e] = fmaf(weight, a[i][e], A[e] * old);
    }
  }
  if (__syncthreads_or(stopped)) return;
  if (sh.groups > 1) {
    s_acc[threadIdx.x] = A;
    if (dd == 0) s_stat[place] = float2{M, L};
    if (odd) s_odd = 1;
    __syncthreads();
    if (group != 0) return;
    odd = s_odd != 0;
    for (int g = 1; g < sh.groups; ++g) {
      const float2 x = s_stat[place + g];
      const f32x4 y = s_acc[threadIdx.x + g * LANES];
      if (x.x == -INFINITY) continue;              // no range of its own
      const float top = fmaxf(M, x.x), old = __builtin_amdgcn_exp2f(M - top), weight = __builtin_amdgcn_exp2f(x.x - top);
      M = top;
      L = fmaf(weight, x.y, L * old);
#pragma unroll
      for (int e = 0; e < 4; ++e) A[e] = fmaf(weight, y[e], A[e] * old);
    }
  }
  if (row >= r.nodes * G) return;
  const int i = row / G;
  const size_t at = (static_cast<size_t>(r.first + i) * Hkv * G + kvh * G + row % G) * D;
  tree_store(c, at, dd, A * (1.f / L));
  const float all_of = (A[0] + A[1]) + (A[2] + A[3]);
  if (__builtin_expect((odd || all_of != all_of) && L == L, 0)) tree_odd_values(c, r, Hkv, D, kvh, i, at, dd);
}

// How a call is cut.  Times of a call, 32 / 8 heads of 128, bf16 rows and outputs unless said otherwise.
// - Rows of a tile: the fewest with which the tiles of all requests and kv-heads are at most 256, one a CU: a tile reads
//   its rows from the XCD's L2 again, which costs less than ranges that have to be joined (8 requests of 1,328 rows: trees of
//   16, tiles of 16 rows 14.5 us, of 32 17.0, of 64 in two ranges 21.9; trees of 32, tiles of 16 22.8, of 32 17.7, of 64 in two
//   ranges 23.8, of 128 in four 24.0; 32 of 1,000 rows, trees of 32: tiles of 32 57, of 64 44, of 128 39).  Tiles of 16 rows
//   use the matrix cores half, which long rows show (one request of 8,000 rows, trees of 64: 30.7 us and, of 32, 23.6), and
//   4-bit rows are decoded once for each tile (one request of 100,001, trees of 13: 72.6 us, tiles of 16 rows 88; short ones
//   would be better off with those: 8 of 1,328, trees of 16: 19.2 and 15.5).  4-bit rows in tiles of 128 rows of 128 values
//   spill 2 to 15 registers, and are still better than tiles of 64, which spill none (64 requests of 1,500 rows, trees of 64: 129
//   us, fp32 203; 175 and 242).
// - Ranges: up to 256 workgroups, of 512 rows and more (1,024 from 128 tiles on: the join is a launch of 4 us).  One request
//   of 8,000 rows, trees of 16: 4 ranges 20.8 us, 8 16.1, 16 18.0; 8 of 1,328 rows, trees of 8: one range 14.7, two 16.1.
//   They are those of max_ctx rows, the lengths being on the device: one request of 8,000 rows takes 52 us under a bound of
//   100,000, 15.9 under its own; 6,000 4-bit rows 49 and 16.1; eight of 1,328, trees of 32, 19.9 and 17.6.
//   Uneven lengths are not evened out: 64 requests of 180 .. 4,300 rows, trees of up to 16, gained 5 to 8 us of 114 in three
//   ranges or in ranges shared evenly over the batch, which cost 64 equal ones of 1,500 rows 85 us instead of 77.
// - Eight waves where a CU has one workgroup: of up to 32 rows if it is long (4 requests of 7,552 rows, 28 / 4 heads, trees of
//   61, fp32: 67 us, with four 73; one of 100,001 4-bit rows: 16 ranges of eight waves 73, 32 of four 74, and 16 of four 99),
//   of more rows always (chains of 250 over four requests of 1,584 rows 42.6 and 49.9; trees of 64 over eight of 1,328 24.5
//   and 27.6).  With two workgroups a CU four are better (64 requests of 1,500 rows, trees of 16: 78, with eight 84).  Short
//   ranges are better off with four: trees of 32 over eight of 1,328 rows (44 blocks) 17.4 us, with eight 20.1; 32 of 800 4-bit
//   rows (26 blocks), trees of 8, 16.2 and 17.3, of 1,300 (42) 20.5 and 20.5, of 2,000 (64) 25.3 and 25.1, trees of 4 22.4 and
//   20.3.  For bf16 rows the border is between products and bytes rather than at a length: small trees, which HBM bounds, have
//   four ahead by 0 to 5 % on both sides of it (32 of 2,900 rows, trees of 8: 71.1 and 72.7; of 4,500 104.5 and 107.5).
// - Neighbours: lines of 4-bit rows hold several heads' codes and scales, so up to eight heads of a range go to one XCD, as
//   long as every XCD still gets as many workgroups (64 requests of 1,500 rows, trees of 8: 39.0 us, each head on another XCD
//   46.5; one of 100,001 rows: 114 MB fetched instead of 266, 70.6 us instead of 72).
TreeShape tree_shape(int batch, int Hkv, int G, int D, int max_nodes, int max_ctx, bool q4) {
  TreeShape sh{};
  const long rows = static_cast<long>(max_nodes) * G, pairs = static_cast<long>(batch) * Hkv;
  const long blocks = (static_cast<long>(max_ctx) + kTreeBlock - 1) / kTreeBlock + (max_nodes + kTreeBlock - 1) / kTreeBlock;
  auto tiles = [&](int columns) { return (rows + 16 * columns - 1) / (16 * columns); };
  sh.columns = rows > 16 && (q4 || (blocks > 64 && pairs * tiles(1) > 64)) ? 2 : 1;
  while (sh.columns < 8 && 16 * sh.columns < rows && pairs * tiles(sh.columns) > 256) sh.columns *= 2;
  sh.tiles = static_cast<int>(tiles(sh.columns));
  const long units = pairs * sh.tiles;
  // (tiles of more than 32 rows are taken where half as large ones were more than 256, so they are 129 and more)
  const long splits = sh.columns > 2 ? 1 : std::max(1L, std::min(256 / units, blocks / (units >= 128 ? 32 : 16)));
  sh.range = static_cast<int>((blocks + splits - 1) / splits + 3) / 4 * 4;   // four waves' turns
  sh.splits = static_cast<int>((blocks + sh.range - 1) / sh.range);
  sh.waves = units * sh.splits <= 256 && (sh.columns > 2 || sh.range > (q4 ? 32 : 96)) ? 8 : 4;
  for (sh.run_log2 = 0; q4 && sh.run_log2 < 3 && Hkv % (2 << sh.run_log2) == 0; ++sh.run_log2) {
    const long unit_groups = pairs * sh.splits >> (sh.run_log2 + 1);
    if (unit_groups % kNumXcd != 0 && unit_groups < 8 * kNumXcd) break;
  }
  for (sh.groups = 1; sh.groups < 8 && sh.groups * kJoinAhead < sh.splits; sh.groups *= 2) {}
  sh.part_bytes = sh.splits > 1 ? static_cast<size_t>(units) * sh.splits * 16 * sh.columns * (D + 2) * sizeof(float) : 0;
  return sh;
}

template <int D, bool Q4, int PARTS>
static void launch_tree_rows(const TreeCall &c, const TreeShape &sh, float *part, int Hkv, int G, dim3 grid, hipStream_t stream) {
  const dim3 block(4 * kWave), more(8 * kWave);
  if (sh.columns == 1 && sh.waves == 8) tree_kernel<D, 1, 8, Q4, PARTS><<<grid, more, 0, stream>>>(c, sh, part, Hkv, G);
  else if (sh.columns == 1) tree_kernel<D, 1, 4, Q4, PARTS><<<grid, block, 0, stream>>>(c, sh, part, Hkv, G);
  else if (sh.columns == 2 && sh.waves == 8) tree_kernel<D, 2, 8, Q4, PARTS><<<grid, more, 0, stream>>>(c, sh, part, Hkv, G);
  else if (sh.columns == 2) tree_kernel<D, 2, 4, Q4, PARTS><<<grid, block, 0, stream>>>(c, sh, part, Hkv, G);
  else if (sh.columns == 4 && sh.waves == 8) tree_wide_kernel<D, 2, 8, Q4, PARTS><<<grid, more, 0, stream>>>(c, sh, Hkv, G);
  else if (sh.columns == 4) tree_wide_kernel<D, 2, 4, Q4, PARTS><<<grid, block, 0, stream>>>(c, sh, Hkv, G);
  else if (sh.waves == 8) tree_wide_kernel<D, 4, 8, Q4, PARTS><<<grid, more, 0, stream>>>(c, sh, Hkv, G);
  else tree_wide_kernel<D, 4, 4, Q4, PARTS><<<grid, block, 0, stream>>>(c, sh, Hkv, G);
}

template <int D>
static void launch_tree_d(const TreeCall &c, const TreeShape &sh, float *part, int Hkv, int G, hipStream_t stream) {
  const long units = static_cast<long>(c.batch) * Hkv * sh.splits;
  const long each_xcd = static_cast<long>(kNumXcd) << sh.run_log2;
  const dim3 grid((units + each_xcd - 1) / each_xcd * each_xcd * sh.tiles);
  if (c.ks != nullptr) {
    if (c.out_bf16) launch_tree_rows<D, true, 1>(c, sh, part, Hkv, G, grid, stream);
    else launch_tree_rows<D, true, 3>(c, sh, part, Hkv, G, grid, stream);
  } else {
    if (c.out_bf16) launch_tree_rows<D, false, 1>(c, sh, part, Hkv, G, grid, stream);
    else launch_tree_rows<D, false, 3>(c, sh, part, Hkv, G, grid, stream);
  }
  if (sh.splits > 1) {
    const int each = kJoinThreads / (D / 4) / sh.groups;
    const long rows = static_cast<long>(c.max_nodes) * G;
    tree_join_kernel<D><<<dim3((rows + each - 1) / each, Hkv, c.batch), dim3(kJoinThreads), 0, stream>>>(c, sh, part, G);
  }
}

hipError_t launch_tree(const TreeCall &c, const TreeShape &sh, float *part, int Hkv, int G, int D, hipStream_t stream) {
  if (D == 64) launch_tree_d<64>(c, sh, part, Hkv, G, stream);
  else launch_tree_d<128>(c, sh, part, Hkv, G, stream);
  return hipGetLastError();
}

// ------------------------------------------------------------------ the path that is kept
// One wave per request.  From node 0 on: of the nodes behind the present one whose parent it is and whose token is the one
// chosen there, the lowest; until there is none (a negative choice, as the logits' call makes where nothing is allowed, is no
// token, whatever a padded tree holds).  Lane l looks at nodes l, l + 64, ..: a step is a few ballots.  Bound by the
// round trips before them and the stores behind: 4.3 us for eight trees of 32.
__global__ __launch_bounds__(kWave) void tree_accept_kernel(TreePlan plan, const int32_t *__restrict__ parent, const int32_t *__restrict__ node_token,
                                                            const int32_t *__restrict__ chosen, int32_t *__restrict__ path,
                                                            int32_t *__restrict__ path_len, int32_t *__restrict__ next_token,
                                                            int32_t *__restrict__ tokens, const int64_t *__restrict__ token_off,
                                                            const int32_t *__restrict__ token_cap, int32_t *__restrict__ token_len, int total,
                                                            int max_nodes, int32_t *status) {
  constexpr int PER = kMaxNodes / kWave;
  const int b = blockIdx.x, lane = threadIdx.x;
  if (step_stops(status)) return;
  const int2 r = plan.req[b];
  const int first = __builtin_amdgcn_readfirstlane(r.x), n = __builtin_amdgcn_readfirstlane(r.y);
  if (first < 0 || n < 0 || n > max_nodes || first > total - n) return;
  int up[PER], token[PER], pick[PER], place[PER];   // place: the node's step on the path, or -1
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = k * kWave + lane;
    const bool in = i < n;
    up[k] = !in ? -2 : parent != nullptr ? parent[first + i] : i - 1;
    token[k] = in ? node_token[first + i] : 0;
    pick[k] = in ? chosen[first + i] : 0;
    place[k] = -1;
  }
  int now = n > 0 ? 0 : -1, steps = 0, want = -1;
  while (now >= 0) {
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (now / kWave == k) {
        want = __builtin_amdgcn_readlane(pick[k], now % kWave);
        if (lane == now % kWave) place[k] = steps;
      }
    ++steps;
    int found = -1;
#pragma unroll
    for (int k = PER - 1; k >= 0; --k) {
      const uint64_t m = __ballot(want >= 0 && up[k] == now && token[k] == want && k * kWave + lane > now);
      if (m != 0) found = k * kWave + __builtin_ctzll(m);
    }
    now = found;
  }
  if (tokens != nullptr) {
    const int len = token_len[b], cap = token_cap[b];
    const int64_t off = token_off[b];
    if (len < 0 || cap < len || steps > cap - len) {   // no room: nothing of the request is kept
      if (lane == 0) raise_status(status, SONIC_ERR_CAPACITY);
      steps = 0, want = -1;
#pragma unroll
      for (int k = 0; k < PER; ++k) place[k] = -1;
    } else {
#pragma unroll
      for (int k = 0; k < PER; ++k)
        if (place[k] >= 0) tokens[off + len + place[k]] = token[k];
      if (lane == 0) token_len[b] = len + steps;
    }
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = k * kWave + lane;
    if (place[k] >= 0) path[first + place[k]] = i;
    if (i >= steps && i < n) path[first + i] = -1;
  }
  if (lane == 0) {
    path_len[b] = steps;
    next_token[b] = want;
  }
}

hipError_t launch_tree_accept(int batch, int total, int max_nodes, TreePlan plan, const int32_t *parent, const int32_t *node_token,
                              const int32_t *chosen, int32_t *path, int32_t *path_len, int32_t *next_token, int32_t *tokens,
                              const int64_t *token_off, const int32_t *token_cap, int32_t *token_len, int32_t *status, hipStream_t stream) {
  tree_accept_kernel<<<dim3(batch), dim3(kWave), 0, stream>>>(plan, parent, node_token, chosen, path, path_len, next_token, tokens, token_off,
                                                               token_cap, token_len, total, max_nodes, status);
  return hipGetLastError();
}

}  // namespace sonic
