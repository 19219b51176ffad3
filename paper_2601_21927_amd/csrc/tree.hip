// Drafted tokens over the compact cache: which tokens a drafted one sees, their attention, and the path that is kept.
//
// A request's drafted tokens ("nodes") form trees: parent[i] < i, -1 for a root, or a chain.  With r over the cache rows
// and over the nodes on i's path (itself and its ancestors),
//     out[i][h] = softmax_r(scale <q[i][h], k[r][g(h)]>) v[r][g(h)].
//
// tree_kernel: a workgroup has up to 64 q rows (node i and q-head g of a kv-head are row i G + g) and a range of the
// request's rows, in blocks of 32: first the cache's, then the nodes', so that a block is of one kind and the nodes'
// visibility in it is one word of the plan.  The four waves take blocks in turn, each with its own K and V in LDS
// (direct-to-LDS loads, K of the next block requested when this one's scores are taken, V when its values are), so that
// none waits for another before the end.  Per block
//   scores   S^T (16 rows x 16 columns) = K . Q^T   v_mfma_f32_16x16x32_bf16
//   softmax  online, fp32, per column in the four lanes that hold it
//   values   O^T (d x 16 columns) += V^T . P^T      v_mfma_f32_16x16x32_bf16, depth 32: the block's rows
// An fp32 output takes a probability in three bf16 values (2^-26 of it is left), a bf16 output in one: its rounding, with
// the sum taken over the rounded ones, is of the size of the output's own (1.2 to 1.3 times that in all).
// Ranges of a request are joined by another kernel.
#include <algorithm>

#include "common.h"
#include "q4.h"
#include "scan.h"

namespace sonic {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16_t;
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int kTreeWaves = 4;
constexpr int kTreeBlock = 32;   // rows of a block: the bits of a word of the plan

// ------------------------------------------------------------------ the plan
// One workgroup per request, one thread per node.  A node's word starts with itself and takes in those of its ancestors
// by doubling: after round k it holds 2^k of them, and `up` is the one behind those.  At most eight rounds.
__global__ __launch_bounds__(kMaxNodes) void tree_plan_kernel(const int32_t *__restrict__ cu, const int32_t *__restrict__ parent,
                                                              int total, int max_nodes, int words, int2 *__restrict__ req,
                                                              uint32_t *__restrict__ sees, int32_t *status) {
  __shared__ int s_stop;
  __shared__ uint32_t s_sees[kMaxNodes][kMaxNodes / 32 + 1];
  __shared__ int s_up[kMaxNodes];
  const int b = blockIdx.x, i = threadIdx.x;
  const int s = cu[b], e = cu[b + 1];
  if (i == 0) s_stop = step_stops(status);
  __syncthreads();
  if (s_stop) return;
  bool bad = s < 0 || e < s || e > total || e - s > max_nodes || (b == 0 && s != 0);
  const int n = bad ? 0 : e - s;
  int up = -1;
  if (i < n) {
    up = parent != nullptr ? parent[s + i] : i - 1;
    bad = up < -1 || up >= i;
  }
  if (__syncthreads_or(bad)) {
    if (i == 0) {
      raise_status(status, SONIC_ERR_BAD_LAYOUT);
      req[b] = int2{0, 0};
    }
    return;
  }
  if (i == 0) req[b] = int2{s, n};
  if (parent == nullptr) {
    for (int w = 0; i < n && w < words; ++w)
      sees[static_cast<size_t>(s + i) * words + w] = i / 32 > w ? ~0u : i / 32 == w ? ~0u >> (31 - i % 32) : 0;
    return;
  }
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
  for (int w = 0; i < n && w < words; ++w) sees[static_cast<size_t>(s + i) * words + w] = s_sees[i][w];
}

hipError_t launch_tree_plan(int batch, int total, int max_nodes, const int32_t *cu, const int32_t *parent, TreePlan plan,
                            int32_t *status, hipStream_t stream) {
  tree_plan_kernel<<<dim3(batch), dim3(kMaxNodes), 0, stream>>>(cu, parent, total, max_nodes, plan.words, const_cast<int2 *>(plan.req),
                                                                const_cast<uint32_t *>(plan.sees), status);
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

// Four outputs, d = dd .. dd + 3 of node i's q-head, normalised by L.  `odd`: V of some nodes is no number.  Those went
// into the products as zero, since zero times them would be none either, also for the nodes that do not see them: here they
// are looked at again.  And an infinite V of the cache comes out of the sums as NaN (a row past a block's end counts zero
// times, a probability's second value is negative for half of the rows): where the scores were numbers, the rows' V are
// read again.  A column whose only values that are none are infinities of one sign gives that infinity.
__device__ __forceinline__ void tree_store(const TreeCall &c, const TreeReq &r, int Hkv, int D, int kvh, int i, size_t at, int dd, f32x4 A,
                                           float L, bool odd) {
  f32x4 o = {A[0] / L, A[1] / L, A[2] / L, A[3] / L};
  const float all_of = (o[0] + o[1]) + (o[2] + o[3]);
  const bool q4 = c.ks != nullptr, none = all_of != all_of && L == L && !q4;   // (4-bit rows hold no infinities)
  if (__builtin_expect(odd || none, 0)) {
    const size_t stride = static_cast<size_t>(Hkv) * D;
    int found[4] = {0, 0, 0, 0};   // 1: +inf, 2: -inf, 4: NaN
    auto look = [&](const uint16_t *x) {
#pragma unroll
      for (int e = 0; e < 4; ++e) found[e] |= x[e] == 0x7F80 ? 1 : x[e] == 0xFF80 ? 2 : (x[e] & 0x7FFF) > 0x7F80 ? 4 : 0;
    };
    if (none) {
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
    for (int e = 0; e < 4; ++e)
      if (found[e] != 0) o[e] = found[e] == 1 ? INFINITY : found[e] == 2 ? -INFINITY : NAN;
  }
  if (c.out_bf16) {
    *reinterpret_cast<bf16x4 *>(static_cast<uint16_t *>(c.out) + at + dd) = __builtin_convertvector(o, bf16x4);
  } else {
    *reinterpret_cast<f32x4 *>(static_cast<float *>(c.out) + at + dd) = o;
  }
}

template <int D, int CT, bool Q4, int PARTS>
__global__ __launch_bounds__(kTreeWaves *kWave, 2) void tree_kernel(TreeCall c, TreeShape sh, float *__restrict__ part, int Hkv, int G) {
  constexpr int KS = D / 32;                     // k steps of the score product
  constexpr int DB = D / 16;                     // 16-wide d blocks of the value product
  constexpr int DC = D / 8;                      // 16-byte chunks per row
  constexpr int BR = kTreeBlock;
  constexpr int NI = BR * DC / kWave;            // direct-to-LDS instructions per tensor and block
  constexpr int KSWZ = DC - 1;                   // K: 16-byte chunk p of row r at p ^ (r & KSWZ)
  constexpr int VSWZ = DC / 2 - 1;               // V: 32-byte segment s of row r at s ^ (r & VSWZ)
  constexpr int COLS = 16 * CT;
  constexpr int TILE = BR * D;                   // elements of one tensor's block
  constexpr int HD = D / 2, HP = HD + 4;         // the join of the waves: half of the values at a time
  constexpr int RING = (Q4 ? 1 : 2) * TILE;      // 4-bit rows: V alone, as bf16
  constexpr int JOIN = COLS * HP * 2;            // (in 16-bit elements)
  __shared__ __align__(16) uint16_t lds[kTreeWaves * (RING > JOIN ? RING : JOIN)];
  __shared__ float m_lds[kTreeWaves][COLS], l_lds[kTreeWaves][COLS];
  __shared__ int s_odd[kTreeWaves];

  // The row tiles of one range are neighbours on one XCD (workgroup i goes to XCD i % 8), as are a range's kv-heads
  // in time: the rows come from its L2 after the first.
  const unsigned turn = blockIdx.x / kNumXcd, xcd = blockIdx.x % kNumXcd;
  const unsigned unit = turn / sh.tiles * kNumXcd + xcd;
  const int rt = turn % sh.tiles;
  if (unit >= static_cast<unsigned>(c.batch) * Hkv * sh.splits) return;
  const int kvh = unit % Hkv, split = unit / Hkv % sh.splits, b = unit / Hkv / sh.splits;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int col = lane & 15, quarter = lane >> 4;
  const int Hq = Hkv * G;

  __shared__ int s_stop;
  if (threadIdx.x == 0) s_stop = step_stops(c.status);   // one look for the workgroup
  const TreeReq r = tree_request(c, b);
  __syncthreads();
  const bool stop = s_stop != 0;
  const int rows = r.nodes * G;                  // q rows of the request
  if (rt * COLS >= rows) return;
  if (r.len < 0 || r.len > c.max_ctx) {          // uniform over the request: no output
    if (threadIdx.x == 0 && rt == 0 && kvh == 0 && split == 0) raise_status(c.status, SONIC_ERR_CAPACITY);
    return;
  }
  const int cached = (r.len + BR - 1) / BR;      // blocks of the cache, then of the nodes
  const int blocks = cached + (r.nodes + BR - 1) / BR;
  const int first = split * sh.range, last = min(blocks, first + sh.range);
  if (first >= blocks) return;
  const bool whole = blocks <= sh.range;
  const size_t slot = ((static_cast<size_t>(b) * Hkv + kvh) * sh.tiles + rt) * sh.splits + split;
  const size_t slots = static_cast<size_t>(c.batch) * Hkv * sh.tiles * sh.splits;
  float *const acc_rec = part + slot * (COLS * D);
  float2 *const stat_rec = reinterpret_cast<float2 *>(part + slots * (COLS * D)) + slot * COLS;
  if (stop) {   // another workgroup of the call may have seen no error: what it left is not to be joined with this one's
    if (!whole && threadIdx.x < COLS) stat_rec[threadIdx.x] = float2{0.f, -INFINITY};
    return;
  }

  // Q^T fragments (B operand of the scores): lane (col, quarter) has d = 32 ks + 8 quarter .. + 7 of its row; with 4-bit
  // rows d = quarter D / 4 + 8 ks .., as the lanes hold K.
  bf16x8 qf[CT][KS];
  int node[CT];
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const int row = min(rt * COLS + 16 * t + col, rows - 1);
    node[t] = row / G;
    const uint16_t *src = c.q + (static_cast<size_t>(r.first + node[t]) * Hq + kvh * G + row % G) * D + (Q4 ? quarter * (D / 4) : 8 * quarter);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[t][ks] = *reinterpret_cast<const bf16x8 *>(src + (Q4 ? 8 : 32) * ks);
  }
  // waited for here: not in the loop, where it would drain the loads ahead
#pragma unroll
  for (int t = 0; t < CT; ++t)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[t][ks]));

  f32x4 oacc[CT][DB];
  float m_run[CT], l_run[CT];   // log2 domain, lagging by at most 8; a lane's share of the sum
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    // (the lowest number: a block whose scores all passed the range below, -infinity, then weighs exp2(-infinity), 0)
    m_run[t] = -__FLT_MAX__;
    l_run[t] = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) oacc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const size_t row_elems = static_cast<size_t>(Hkv) * D;
  const uint16_t *knew = c.k_new + static_cast<size_t>(r.first) * row_elems + kvh * D;
  const uint16_t *vnew = c.v_new + static_cast<size_t>(r.first) * row_elems + kvh * D;
  const int tr_row = 4 * quarter + (col >> 2);
  const int tr_off = tr_row * D + 4 * (col & 3);
  const int tr_swz = tr_row & VSWZ;
  uint16_t *const vtile = lds + wave * RING + (Q4 ? 0 : TILE);

  bool odd = false;   // V of a node is no number

  // The scores of a block, s[t][half][i] for row 16 half + 4 quarter + i of column 16 t + col, to probabilities and into
  // the output.  `ready`: V of the block is in vtile when it returns.
  auto block = [&](int g, f32x4 (&s)[CT][2], auto ready) {
    const bool drafted = g >= cached;
    if (drafted) {
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        const uint32_t word = c.plan.sees[static_cast<size_t>(r.first + node[t]) * c.plan.words + (g - cached)] >> (4 * quarter);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][h][i] = (word >> (16 * h + i)) & 1 ? s[t][h][i] : -INFINITY;
      }
    } else if ((g + 1) * BR > r.len) {
      const int left = r.len - g * BR - 4 * quarter;
#pragma unroll
      for (int t = 0; t < CT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][h][i] = 16 * h + i < left ? s[t][h][i] : -INFINITY;
    }
    float top[CT];
    bool grows = false;
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      top[t] = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])),
                     fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
      top[t] = pair32_max(pair16_max(top[t])) * c.scale_log2;
      grows = grows || top[t] > m_run[t] + 8.f;
    }
    if (__any(grows)) {   // rescale only when a max grows by more than 2^8
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        const float m_new = fmaxf(m_run[t], top[t]);
        const float corr = __builtin_amdgcn_exp2f(m_run[t] - m_new);
        m_run[t] = m_new;
        l_run[t] *= corr;
#pragma unroll
        for (int i = 0; i < DB; ++i) oacc[t][i] *= corr;
      }
    }
    bf16x8 pp[CT][PARTS];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      f32x8 p;
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[t][i / 4][i % 4], c.scale_log2, -m_run[t]));
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        pp[t][k] = __builtin_convertvector(p, bf16x8);
        if (k + 1 < PARTS) p -= __builtin_convertvector(pp[t][k], f32x8);
      }
      l_run[t] += rounded_sum(pp[t]);
    }
    ready();
    if (drafted) {   // (see tree_store)
      bool here = false;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        u32x4 *at = reinterpret_cast<u32x4 *>(vtile + (i * kWave + lane) * 8);
        const u32x4 w = *at;
        const u32x4 keep = {finite_halves(w[0]), finite_halves(w[1]), finite_halves(w[2]), finite_halves(w[3])};
        const bool bad = (keep[0] & keep[1] & keep[2] & keep[3]) != ~0u;
        if (bad) *at = w & keep;
        here = here || bad;
      }
      odd = odd || __any(here);
    }
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
  };

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
    int g = first + wave;
    if (g < last) {
      issue_k(g);
      issue_v(g);
      for (; g < last; g += kTreeWaves) {
        wait_vm<NI>();   // K is there; V may not be
        f32x4 s[CT][2];
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
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // lgkmcnt(0): K may be overwritten
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        issue_k(g + kTreeWaves);
        block(g, s, [&]() {
          wait_vm<NI>();   // V is there; the next K may not be
          __atomic_signal_fence(__ATOMIC_SEQ_CST);
        });
        __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));
        __atomic_signal_fence(__ATOMIC_SEQ_CST);
        issue_v(g + kTreeWaves);
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
    int g = first + wave;
    if (g < last) {
      KRaw k_raw = fetch_k(g);
      VRaw v_raw = fetch_v(g);
      for (; g < last; g += kTreeWaves) {
        f32x4 s[CT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int t = 0; t < CT; ++t) s[t][h] = f32x4{0.f, 0.f, 0.f, 0.f};
          const float scale = q4_scale(k_raw.s[h]);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const bf16x8 a = q4_decode8(k_raw.c[h][ks], scale);
#pragma unroll
            for (int t = 0; t < CT; ++t) s[t][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[t][ks], s[t][h], 0, 0, 0);
          }
        }
        k_raw = fetch_k(g + kTreeWaves);
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
          v_raw = fetch_v(g + kTreeWaves);
        });
      }
    }
  }

  // ---- the waves' parts to one: columns across the four quarters, then through LDS, half of the values at a time ----
#pragma unroll
  for (int t = 0; t < CT; ++t) {
    const float l = pair32_add(pair16_add(l_run[t]));
    if (quarter == 0) {
      m_lds[wave][16 * t + col] = m_run[t];
      l_lds[wave][16 * t + col] = l;
    }
  }
  if (lane == 0) s_odd[wave] = odd;
  float *const join = reinterpret_cast<float *>(lds);   // [wave][COLS][HP]
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    __syncthreads();   // every wave is done with its blocks (with the first half)
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int db = 0; db < DB / 2; ++db)
        *reinterpret_cast<f32x4 *>(&join[(wave * COLS + 16 * t + col) * HP + 16 * db + 4 * quarter]) = oacc[t][half * (DB / 2) + db];
    __syncthreads();
    odd = false;
#pragma unroll
    for (int w = 0; w < kTreeWaves; ++w) odd = odd || s_odd[w] != 0;
    for (int u = threadIdx.x; u < COLS * HD / 4; u += kTreeWaves * kWave) {
      const int cc = u / (HD / 4), dd = 4 * (u % (HD / 4));
      const int row = rt * COLS + cc;
      if (row >= rows) break;
      float M = m_lds[0][cc];
#pragma unroll
      for (int w = 1; w < kTreeWaves; ++w) M = fmaxf(M, m_lds[w][cc]);
      float L = 0.f;
      f32x4 A = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kTreeWaves; ++w) {
        const float weight = __builtin_amdgcn_exp2f(m_lds[w][cc] - M);
        L = fmaf(weight, l_lds[w][cc], L);
        const f32x4 a = *reinterpret_cast<const f32x4 *>(&join[(w * COLS + cc) * HP + dd]);
#pragma unroll
        for (int e = 0; e < 4; ++e) A[e] = fmaf(weight, a[e], A[e]);
      }
      if (whole) {
        const int i = row / G;
        tree_store(c, r, Hkv, D, kvh, i, (static_cast<size_t>(r.first + i) * Hq + kvh * G + row % G) * D, half * HD + dd, A, L, odd);
      } else {
        *reinterpret_cast<f32x4 *>(acc_rec + cc * D + half * HD + dd) = A;
        if (half == 0 && dd == 0) stat_rec[cc] = float2{M, odd ? -L : L};   // (L has no sign of its own)
      }
    }
  }
}

// The ranges of a request joined by log-sum-exp.  Grid (rows of a kv-head / rows a workgroup has, kv-heads, requests); a
// thread has four values of a row, eight ranges in flight.
constexpr int kJoinThreads = 256;
template <int D>
__global__ __launch_bounds__(kJoinThreads) void tree_join_kernel(TreeCall c, TreeShape sh, const float *__restrict__ part, int G) {
  constexpr int AHEAD = 8;
  const int b = blockIdx.z, kvh = blockIdx.y, Hkv = gridDim.y;
  const TreeReq r = tree_request(c, b);
  const int row = blockIdx.x * (kJoinThreads / (D / 4)) + threadIdx.x / (D / 4), dd = 4 * (threadIdx.x % (D / 4));
  const int blocks = (r.len + kTreeBlock - 1) / kTreeBlock + (r.nodes + kTreeBlock - 1) / kTreeBlock;
  if (row >= r.nodes * G || r.len < 0 || r.len > c.max_ctx || blocks <= sh.range) return;
  const int splits = (blocks + sh.range - 1) / sh.range;
  const int COLS = 16 * sh.columns;
  const size_t slot = ((static_cast<size_t>(b) * Hkv + kvh) * sh.tiles + row / COLS) * sh.splits;
  const size_t slots = static_cast<size_t>(c.batch) * Hkv * sh.tiles * sh.splits;
  const float *acc = part + (slot * COLS + row % COLS) * D + dd;
  const float2 *stat = reinterpret_cast<const float2 *>(part + slots * COLS * D) + slot * COLS + row % COLS;
  float M = -INFINITY, L = 0.f;
  bool odd = false;
  f32x4 A = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += AHEAD) {
    float2 ml[AHEAD];
    f32x4 a[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const size_t s = min(s0 + i, splits - 1);
      ml[i] = stat[s * COLS];
      a[i] = *reinterpret_cast<const f32x4 *>(acc + s * COLS * D);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (s0 + i >= splits) break;
      if (ml[i].y == -INFINITY) return;   // a workgroup that had been stopped
      odd = odd || (__float_as_uint(ml[i].y) >> 31) != 0;
      const float top = fmaxf(M, ml[i].x), old = __builtin_amdgcn_exp2f(M - top), weight = __builtin_amdgcn_exp2f(ml[i].x - top);
      M = top;
      L = fmaf(weight, fabsf(ml[i].y), L * old);
#pragma unroll
      for (int e = 0; e < 4; ++e) A[e] = fmaf(weight, a[i][e], A[e] * old);
    }
  }
  const int i = row / G;
  tree_store(c, r, Hkv, D, kvh, i, (static_cast<size_t>(r.first + i) * Hkv * G + kvh * G + row % G) * D, dd, A, L, odd);
}

// How a call is cut.
TreeShape tree_shape(int batch, int Hkv, int G, int D, int max_nodes, int max_ctx) {
  TreeShape sh{};
  const long rows = static_cast<long>(max_nodes) * G;
  sh.columns = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  sh.tiles = static_cast<int>((rows + 16 * sh.columns - 1) / (16 * sh.columns));
  const long units = static_cast<long>(batch) * Hkv * sh.tiles;
  const long blocks = (static_cast<long>(max_ctx) + kTreeBlock - 1) / kTreeBlock + (max_nodes + kTreeBlock - 1) / kTreeBlock;
  long splits = std::max(1L, std::min({512 / units, (blocks + 7) / 8, 64L}));
  sh.range = static_cast<int>((blocks + splits - 1) / splits);
  sh.splits = static_cast<int>((blocks + sh.range - 1) / sh.range);
  sh.part_bytes = sh.splits > 1 ? static_cast<size_t>(units) * sh.splits * 16 * sh.columns * (D + 2) * sizeof(float) : 0;
  return sh;
}

template <int D, int CT>
static void launch_tree_ct(const TreeCall &c, const TreeShape &sh, float *part, int Hkv, int G, dim3 grid, hipStream_t stream) {
  const dim3 block(kTreeWaves * kWave);
  if (c.ks != nullptr) {
    if (c.out_bf16) tree_kernel<D, CT, true, 1><<<grid, block, 0, stream>>>(c, sh, part, Hkv, G);
    else tree_kernel<D, CT, true, 3><<<grid, block, 0, stream>>>(c, sh, part, Hkv, G);
  } else {
    if (c.out_bf16) tree_kernel<D, CT, false, 1><<<grid, block, 0, stream>>>(c, sh, part, Hkv, G);
    else tree_kernel<D, CT, false, 3><<<grid, block, 0, stream>>>(c, sh, part, Hkv, G);
  }
}

template <int D>
static void launch_tree_d(const TreeCall &c, const TreeShape &sh, float *part, int Hkv, int G, hipStream_t stream) {
  const long units = static_cast<long>(c.batch) * Hkv * sh.splits;
  const dim3 grid((units + kNumXcd - 1) / kNumXcd * kNumXcd * sh.tiles);
  if (sh.columns == 1) launch_tree_ct<D, 1>(c, sh, part, Hkv, G, grid, stream);
  else if (sh.columns == 2) launch_tree_ct<D, 2>(c, sh, part, Hkv, G, grid, stream);
  else launch_tree_ct<D, 4>(c, sh, part, Hkv, G, grid, stream);
  if (sh.splits > 1) {
    const int each = kJoinThreads / (D / 4);
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
// chosen there, the lowest; until there is none.  Lane l looks at nodes l, l + 64, ..: a step is a few ballots.
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
      const uint64_t m = __ballot(up[k] == now && token[k] == want && k * kWave + lane > now);
      if (m != 0) found = k * kWave + __builtin_ctzll(m);
    }
    now = found;
  }
  if (tokens != nullptr) {
    const int len = token_len[b], cap = token_cap[b];
    const int64_t off = token_off[b];
    if (len < 0 || steps > cap - len) {   // no room: nothing of the request is kept
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
