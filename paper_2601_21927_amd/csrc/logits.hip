// Logits with penalties of repeated tokens, biases and grammar masks, and the best token of every row.
//
// For a row of request b and token t, with `seen` whether t is in b's history or on the row's path (the tokens of its node
// and of that node's ancestors) and c how often it is behind the prompt or on the path:
//     x = logit;  seen: x = x > 0 ? x / repetition : x * repetition;  c > 0: x = x - (presence + frequency * c)
//     biased: x = x + bias;  not allowed: x = -infinity
// every operation rounded to fp32 by itself, so that a best token does not depend on how the compiler joins them.
//
// logits_kernel: a workgroup has a piece of the vocabulary and some rows of one request.  It counts the request's tokens
// that fall into the piece in LDS, a word per token (count, seen, biased) and a bit per token that has one, once for its
// rows; per row the path's tokens are added and taken off again.  A row is then one pass over its logits, 16 bytes a lane,
// in which a thread's tokens that have a word are mended one after the other: there are few, but most waves have some
// among any 256 tokens, and did the penalties' divisions for all of them (256 rows of 128,000 in bf16, written out: 73 us
// so, 62 this way).  The next row's logits, mask words and path are requested ahead of this row's stores, so that a row
// waits for nothing of its own (55 us), and the stores pass the caches, which hold what the program has just computed (45 us;
// 201 MB, 4.5 TB/s).  Where rows are few, a chain of loads is what counts: lengths, then history and logits, then biases, in
// 2.3 rounds of workgroups, and then the histories, which every piece scans again (64 rows of 150,001 with histories of up to
// 9,000 tokens, 41 MB: 25 us, 7 of them the histories').
// logits_best_kernel picks each row's best from the pieces' and raises errors.
#include <algorithm>

#include "common.h"
#include "scan.h"

#pragma clang fp contract(off)

namespace sonic {

constexpr int kLogitThreads = 256;
constexpr int kPiece = 4096;                   // tokens of a workgroup
constexpr uint32_t kBiased = 1u << 31, kSeen = 1u << 30, kCount = kSeen - 1;

struct Best {
  float value;
  int token;       // -1: none; kStopped: the piece was not looked at
};
constexpr int kStopped = -2;

// The rows and the history of request b, checked.
struct LogitsReq {
  int first, rows, len, prompt, bias0, biases;
  int64_t off;
};
__device__ __forceinline__ bool logits_request(const LogitsCall &c, int b, LogitsReq *r) {
  int2 rows = int2{b, 1};
  if (c.plan.req != nullptr) rows = c.plan.req[b];
  *r = LogitsReq{rows.x, rows.y, 0, 0, 0, 0, 0};
  if (rows.x < 0 || rows.y < 0 || rows.y > c.max_rows || rows.x > c.total_rows - rows.y) r->rows = 0;   // (a plan of another call)
  bool bad = false;
  if (c.tokens != nullptr) {
    r->len = c.token_len[b];
    r->prompt = c.prompt_len != nullptr ? c.prompt_len[b] : 0;
    r->off = c.token_off[b];
    bad = r->len < 0 || r->prompt < 0 || r->prompt > r->len;
  }
  if (c.bias_cu != nullptr) {
    r->bias0 = c.bias_cu[b];
    r->biases = c.bias_cu[b + 1] - r->bias0;
    bad = bad || r->bias0 < 0 || c.bias_cu[b + 1] < r->bias0;
  }
  return !bad;
}

// The 16-byte parts of a row that a thread has: part k is tokens first + PE (thread + k * threads) .. + PE - 1.
// What else a row needs of memory comes along: the words of its mask, and of the nodes that it sees.
template <bool BF16> struct RowParts {
  static constexpr int PE = BF16 ? 8 : 4;      // elements of 16 bytes
  static constexpr int STEPS = (kPiece + PE) / (PE * kLogitThreads) + 1;
  u32x4 raw[STEPS];
  uint32_t low[STEPS], high[STEPS];            // of the mask: the words from a part's first token on
  uint32_t sees;

  // First token of the parts: the piece starts up to PE - 1 tokens behind a 16-byte border.
  __device__ __forceinline__ static int first(size_t start, int t0) { return t0 - static_cast<int>((start + t0) % PE); }

  __device__ __forceinline__ void load(const LogitsCall &c, size_t at, int t0, int t1) {
    const size_t start = at * c.vocab;
    const int f = first(start, t0), mask_words = (c.vocab + 31) / 32;
    sees = c.plan.req != nullptr && static_cast<int>(threadIdx.x) < c.max_rows ? c.plan.sees[at * c.plan.words + threadIdx.x / 32] : 0;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int t = f + PE * (static_cast<int>(threadIdx.x) + k * kLogitThreads);
      raw[k] = u32x4{0, 0, 0, 0};
      low[k] = high[k] = ~0u;
      if (t >= t1) continue;
      if (c.allowed != nullptr) {
        const uint32_t *allowed = c.allowed + at * mask_words + max(t, 0) / 32;
        low[k] = allowed[0];
        high[k] = allowed[max(t, 0) / 32 + 1 < mask_words ? 1 : 0];
      }
      if (t >= 0 && t + PE <= c.vocab) {
        raw[k] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(c.logits) + (start + t) * (BF16 ? 2 : 4));
      } else {   // the row's ends
#pragma unroll
        for (int e = 0; e < PE; ++e) {
          if (t + e < 0 || t + e >= c.vocab) continue;
          if constexpr (BF16) raw[k][e / 2] |= static_cast<uint32_t>(static_cast<const uint16_t *>(c.logits)[start + t + e]) << (16 * (e & 1));
          else raw[k][e] = static_cast<const uint32_t *>(c.logits)[start + t + e];
        }
      }
    }
  }
};

// Bits t .. of a bit array whose words t / 32 and one on are low and high; t from -PE + 1 on, low its first word then.
__device__ __forceinline__ uint32_t bits_from(uint32_t low, uint32_t high, int t) {
  return t < 0 ? low << -t : __builtin_amdgcn_alignbit(high, low, t % 32);
}

template <bool BF16>
__global__ __launch_bounds__(kLogitThreads) void logits_kernel(LogitsCall c, int group, int pieces, Best *__restrict__ part) {
  typedef RowParts<BF16> Parts;
  constexpr int PE = Parts::PE, STEPS = Parts::STEPS, AHEAD = 8, WORDS = kPiece / 32;
  __shared__ __align__(16) uint32_t s_word[kPiece];
  __shared__ int s_entry[kPiece];              // the token's bias, as an entry of the request's
  __shared__ uint32_t s_has[WORDS];            // tokens that have a word
  __shared__ float s_max[kLogitThreads / kWave];
  __shared__ int s_token, s_stop;
  const int b = blockIdx.z, t0 = blockIdx.x * kPiece, t1 = min(c.vocab, t0 + kPiece);
  LogitsReq r;
  const bool good = logits_request(c, b, &r);
  if (threadIdx.x == 0) {
    s_stop = step_stops(c.status);
    s_token = INT32_MAX;
  }
  for (int i = threadIdx.x; i < kPiece / 4; i += kLogitThreads) reinterpret_cast<u32x4 *>(s_word)[i] = u32x4{0, 0, 0, 0};
  if (threadIdx.x < WORDS) s_has[threadIdx.x] = 0;
  lds_barrier();
  const int row0 = blockIdx.y * group, row1 = min(r.rows, row0 + group);
  if (!good || row0 >= row1) return;
  if (s_stop) {   // other workgroups of the call may have seen no error: no best is made of this piece and theirs
    for (int row = row0 + threadIdx.x; row < row1; row += kLogitThreads)
      part[static_cast<size_t>(r.first + row) * pieces + blockIdx.x] = Best{0.f, kStopped};
    return;
  }

  auto in_piece = [&](int t) { return t >= t0 && t < t1; };
  auto has = [&](int i) { atomicOr(&s_has[i / 32], 1u << (i % 32)); };
  // thread j has node j of the request, whose token the rows that see it count
  int token = -1;
  if (c.node_token != nullptr && c.plan.req != nullptr && static_cast<int>(threadIdx.x) < r.rows) token = c.node_token[r.first + threadIdx.x];
  int t[AHEAD];
  const unsigned len = r.len, biases = r.biases;   // (unsigned: indexes go past them by up to 2,048)
  auto request = [&](unsigned i0) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const unsigned i = i0 + k * kLogitThreads;
      t[k] = i < len ? c.tokens[r.off + i] : -1;
    }
  };
  // the first tokens of the history, the first biases and the first row are on their way together
  request(threadIdx.x);
  const int bias = threadIdx.x < biases ? c.bias_token[r.bias0 + threadIdx.x] : -1;
  Parts x;
  x.load(c, r.first + row0, t0, t1);
  for (unsigned i0 = threadIdx.x; i0 < len; i0 += AHEAD * kLogitThreads) {
    if (i0 >= AHEAD * kLogitThreads) request(i0);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (in_piece(t[k])) {
        if (i0 + k * kLogitThreads < static_cast<unsigned>(r.prompt)) atomicOr(&s_word[t[k] - t0], kSeen);
        else atomicAdd(&s_word[t[k] - t0], 1u);
        has(t[k] - t0);
      }
  }
  if (biases > 0) {
    for (unsigned i = threadIdx.x; i < biases; i += kLogitThreads) {   // (few tokens of the piece have one: theirs start at -1)
      const int t = i < kLogitThreads ? bias : c.bias_token[r.bias0 + i];
      if (in_piece(t)) {
        atomicOr(&s_word[t - t0], kBiased);
        has(t - t0);
        s_entry[t - t0] = -1;
      }
    }
    lds_barrier();
    for (unsigned i = threadIdx.x; i < biases; i += kLogitThreads) {
      const int t = i < kLogitThreads ? bias : c.bias_token[r.bias0 + i];
      if (in_piece(t)) atomicMax(&s_entry[t - t0], static_cast<int>(i));              // of several entries for a token the last one counts
    }
  }
  const float rep = c.repetition != nullptr ? c.repetition[b] : 1.f;
  const float presence = c.presence != nullptr ? c.presence[b] : 0.f, frequency = c.frequency != nullptr ? c.frequency[b] : 0.f;
  lds_barrier();

  for (int row = row0; row < row1; ++row) {
    const size_t at = static_cast<size_t>(r.first + row), start = at * c.vocab;
    // the path's tokens
    int mine = -1;
    if (c.node_token != nullptr) {
      const int j = threadIdx.x;
      if (c.plan.req == nullptr) {
        if (j == 0) mine = c.node_token[at];
      } else if (j < r.rows && ((x.sees >> (j % 32)) & 1)) {
        mine = token;
      }
      if (in_piece(mine)) {
        atomicAdd(&s_word[mine - t0], 1u);
        has(mine - t0);
      }
      lds_barrier();
    }
    const int f = Parts::first(start, t0) + PE * static_cast<int>(threadIdx.x);   // the thread's first token
    float v[STEPS][PE], top = -INFINITY;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int t = f + k * PE * kLogitThreads;
#pragma unroll
      for (int e = 0; e < PE; ++e) v[k][e] = -INFINITY;
      if (t >= t1) continue;
      uint32_t in = (1u << PE) - 1;            // tokens of the piece
      if (t < t0) in &= ~0u << (t0 - t);
      if (t + PE > t1) in &= ~(~0u << (t1 - t));
      uint32_t ok = in;
      ok &= bits_from(x.low[k], x.high[k], t);   // (all ones without a mask)
#pragma unroll
      for (int e = 0; e < PE; ++e) {
        if constexpr (BF16) v[k][e] = e & 1 ? bf16_hi(x.raw[k][e / 2]) : bf16_lo(x.raw[k][e / 2]);
        else v[k][e] = __uint_as_float(x.raw[k][e]);
      }
      for (uint32_t left = bits_from(s_has[max(t - t0, 0) / 32], s_has[min(max(t - t0, 0) / 32 + 1, WORDS - 1)], t - t0) & ok; left != 0; left &= left - 1) {
        const int e = __builtin_ctz(left);
        const uint32_t word = s_word[t + e - t0];
        float y = v[k][0];
#pragma unroll
        for (int i = 1; i < PE; ++i) y = e == i ? v[k][i] : y;
        if (word & (kSeen | kCount)) y = y > 0.f ? y / rep : y * rep;
        if (word & kCount) {
          const float off = frequency * static_cast<float>(word & kCount);
          y = y - (presence + off);
        }
        if (word & kBiased) y = y + c.bias_value[r.bias0 + s_entry[t + e - t0]];
#pragma unroll
        for (int i = 0; i < PE; ++i) v[k][i] = e == i ? y : v[k][i];
      }
#pragma unroll
      for (int e = 0; e < PE; ++e) {
        v[k][e] = (ok >> e) & 1 ? v[k][e] : -INFINITY;
        top = fmaxf(top, v[k][e]);
      }
    }
    if (row + 1 < row1) x.load(c, at + 1, t0, t1);   // on their way (ahead of the stores) while the rest is done
    if (c.out != nullptr) {
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const int t = f + k * PE * kLogitThreads;
        float *o = c.out + start + t;
        if (t >= t0 && t + PE <= t1) {
#pragma unroll
          for (int e = 0; e < PE; e += 4)
            __builtin_nontemporal_store(f32x4{v[k][e], v[k][e + 1], v[k][e + 2], v[k][e + 3]}, reinterpret_cast<f32x4 *>(o + e));
        } else {
#pragma unroll
          for (int e = 0; e < PE; ++e)
            if (t + e >= t0 && t + e < t1) o[e] = v[k][e];
        }
      }
    }
    // the piece's greatest value (a NaN is passed over), then the lowest token that has it
    float most = top;
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    if (threadIdx.x % kWave == 0) s_max[threadIdx.x / kWave] = most;
    lds_barrier();
    if (in_piece(mine) && atomicSub(&s_word[mine - t0], 1u) == 1) atomicAnd(&s_has[(mine - t0) / 32], ~(1u << ((mine - t0) % 32)));
#pragma unroll
    for (int w = 0; w < kLogitThreads / kWave; ++w) most = fmaxf(most, s_max[w]);
    if (most > -INFINITY) {
      if (top == most) {
        int lowest = INT32_MAX;
#pragma unroll
        for (int k = STEPS - 1; k >= 0; --k)
#pragma unroll
          for (int e = PE - 1; e >= 0; --e)
            if (v[k][e] == most) lowest = f + k * PE * kLogitThreads + e;
        atomicMin(&s_token, lowest);
      }
    }
    lds_barrier();
    if (threadIdx.x == 0) {
      part[at * pieces + blockIdx.x] = Best{most, most > -INFINITY ? s_token : -1};
      s_token = INT32_MAX;                     // (the next row's are behind a barrier)
    }
  }
}

// One wave per row: the best of its pieces.  The first row's wave of a request raises what is wrong with it (here, where no
// other workgroup looks at the status word any more).
__global__ __launch_bounds__(kWave) void logits_best_kernel(LogitsCall c, int pieces, const Best *__restrict__ part) {
  const int b = blockIdx.y, row = blockIdx.x, lane = threadIdx.x;
  LogitsReq r;
  const bool good = logits_request(c, b, &r);
  if (!good) {
    if (row == 0 && lane == 0) raise_step_status(c.status, SONIC_ERR_BAD_LAYOUT);
    return;
  }
  if (row >= r.rows) return;
  const size_t at = static_cast<size_t>(r.first + row);
  Best best{-INFINITY, -1};
  bool stopped = false;
  for (int i = lane; i < pieces; i += kWave) {
    const Best x = part[at * pieces + i];
    stopped = stopped || x.token == kStopped;
    if (x.token >= 0 && (x.value > best.value || best.token < 0)) best = x;
  }
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) {
    const float v = __shfl_xor(best.value, o);
    const int t = __shfl_xor(best.token, o);
    if (t >= 0 && (best.token < 0 || v > best.value || (v == best.value && t < best.token))) best = Best{v, t};
  }
  if (__any(stopped)) return;
  if (lane == 0) {
    if (c.best != nullptr) c.best[at] = best.token;
    if (c.best_value != nullptr) c.best_value[at] = best.value;
  }
}

int logits_pieces(int vocab) { return (vocab + kPiece - 1) / kPiece; }

hipError_t launch_logits(const LogitsCall &c, void *workspace, hipStream_t stream) {
  const int pieces = logits_pieces(c.vocab);
  // rows of a workgroup: its table is made once for them, so as many as leave about four workgroups a CU
  const long units = static_cast<long>(pieces) * c.batch;
  const int group = static_cast<int>(std::max(1L, std::min(static_cast<long>(c.max_rows), units * c.max_rows / 1024)));
  const dim3 grid(pieces, (c.max_rows + group - 1) / group, c.batch);
  Best *part = static_cast<Best *>(workspace);
  if (c.bf16) logits_kernel<true><<<grid, dim3(kLogitThreads), 0, stream>>>(c, group, pieces, part);
  else logits_kernel<false><<<grid, dim3(kLogitThreads), 0, stream>>>(c, group, pieces, part);
  logits_best_kernel<<<dim3(c.max_rows, c.batch), dim3(kWave), 0, stream>>>(c, pieces, part);
  return hipGetLastError();
}

}  // namespace sonic
