// Logits with penalties of repeated tokens, biases and grammar masks, and the best token of every row.
//
// For a row of request b and token t, with `seen` whether t is in b's history or on the row's path (the tokens of its node
// and of that node's ancestors) and c how often it is behind the prompt or on the path:
//     x = logit;  seen: x = x > 0 ? x / repetition : x * repetition;  c > 0: x = x - (presence + frequency * c)
//     biased: x = x + bias;  not allowed: x = -infinity
// every operation rounded to fp32 by itself, so that a best token does not depend on how the compiler joins them.
//
// logits_kernel: a workgroup has a piece of the vocabulary and some rows of one request.  It counts the request's tokens
// that fall into the piece in LDS, a word per token (count, seen, biased), once for its rows; per row the path's tokens are
// added and taken off again.  The row is then one pass over its logits, 16 bytes a lane; nearly all words are zero and cost
// a compare.  Bound by the bytes of the logits.  logits_best_kernel picks each row's best from the pieces' and raises errors.
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

template <bool BF16>
__global__ __launch_bounds__(kLogitThreads) void logits_kernel(LogitsCall c, int group, int pieces, Best *__restrict__ part) {
  constexpr int PE = BF16 ? 8 : 4;             // elements of 16 bytes
  constexpr int STEPS = (kPiece + PE) / (PE * kLogitThreads) + 1;
  __shared__ __align__(16) uint32_t s_word[kPiece];
  __shared__ int s_entry[kPiece];              // the token's bias, as an entry of the request's
  __shared__ Best s_best[kLogitThreads / kWave];
  __shared__ int s_stop;
  const int b = blockIdx.z, t0 = blockIdx.x * kPiece, t1 = min(c.vocab, t0 + kPiece);
  LogitsReq r;
  const bool good = logits_request(c, b, &r);
  if (threadIdx.x == 0) s_stop = step_stops(c.status);
  __syncthreads();
  const int row0 = blockIdx.y * group, row1 = min(r.rows, row0 + group);
  if (!good || row0 >= row1) return;
  if (s_stop) {   // other workgroups of the call may have seen no error: no best is made of this piece and theirs
    for (int row = row0 + threadIdx.x; row < row1; row += kLogitThreads)
      part[static_cast<size_t>(r.first + row) * pieces + blockIdx.x] = Best{0.f, kStopped};
    return;
  }

  for (int i = threadIdx.x; i < kPiece; i += kLogitThreads) {
    s_word[i] = 0;
    s_entry[i] = -1;
  }
  __syncthreads();
  auto in_piece = [&](int t) { return t >= t0 && t < t1; };
  for (int i = threadIdx.x; i < r.len; i += kLogitThreads) {
    const int t = c.tokens[r.off + i];
    if (in_piece(t)) {
      if (i < r.prompt) atomicOr(&s_word[t - t0], kSeen);
      else atomicAdd(&s_word[t - t0], 1u);
    }
  }
  for (int i = threadIdx.x; i < r.biases; i += kLogitThreads) {
    const int t = c.bias_token[r.bias0 + i];
    if (in_piece(t)) {
      atomicOr(&s_word[t - t0], kBiased);
      atomicMax(&s_entry[t - t0], i);           // of several entries for a token the last one counts
    }
  }
  const float rep = c.repetition != nullptr ? c.repetition[b] : 1.f;
  const float presence = c.presence != nullptr ? c.presence[b] : 0.f, frequency = c.frequency != nullptr ? c.frequency[b] : 0.f;
  __syncthreads();

  for (int row = row0; row < row1; ++row) {
    const size_t at = static_cast<size_t>(r.first + row);
    // the path's tokens: thread j has node j
    int mine = -1;
    if (c.node_token != nullptr) {
      const int j = threadIdx.x;
      if (c.plan.req == nullptr) {
        if (j == 0) mine = c.node_token[at];
      } else if (j < r.rows && ((c.plan.sees[at * c.plan.words + j / 32] >> (j % 32)) & 1)) {
        mine = c.node_token[r.first + j];
      }
      if (in_piece(mine)) atomicAdd(&s_word[mine - t0], 1u);
      __syncthreads();
    }
    const size_t start = at * c.vocab;
    const int skew = static_cast<int>((start + t0) % PE);   // the piece starts that far behind a 16-byte border
    const uint32_t *allowed = c.allowed != nullptr ? c.allowed + at * ((c.vocab + 31) / 32) : nullptr;
    u32x4 raw[STEPS];
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int t = t0 - skew + PE * (static_cast<int>(threadIdx.x) + k * kLogitThreads);
      raw[k] = u32x4{0, 0, 0, 0};
      if (t >= t1) continue;
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
    Best best{-INFINITY, -1};
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      const int t = t0 - skew + PE * (static_cast<int>(threadIdx.x) + k * kLogitThreads);
      if (t >= t1) continue;
      uint32_t bits = ~0u;
      if (allowed != nullptr) {
        const int w0 = max(t, 0) / 32, w1 = min(t + PE - 1, c.vocab - 1) / 32;
        const uint64_t both = static_cast<uint64_t>(allowed[w1]) << 32 | allowed[w0];
        bits = static_cast<uint32_t>(t < 0 ? both << -t : w1 > w0 ? both >> (t % 32) : (both & 0xFFFFFFFFu) >> (t % 32));
      }
      float x[PE];
#pragma unroll
      for (int e = 0; e < PE; ++e) {
        if constexpr (BF16) x[e] = e & 1 ? bf16_hi(raw[k][e / 2]) : bf16_lo(raw[k][e / 2]);
        else x[e] = __uint_as_float(raw[k][e]);
        const bool in = t + e >= t0 && t + e < t1;
        const uint32_t word = s_word[in ? t + e - t0 : 0];
        if (in && word != 0) {
          if (word & (kSeen | kCount)) x[e] = x[e] > 0.f ? x[e] / rep : x[e] * rep;
          if (word & kCount) {
            const float off = frequency * static_cast<float>(word & kCount);
            x[e] = x[e] - (presence + off);
          }
          if (word & kBiased) x[e] = x[e] + c.bias_value[r.bias0 + s_entry[t + e - t0]];
        }
        if (((bits >> e) & 1) == 0) x[e] = -INFINITY;
        if (in && x[e] > best.value) best = Best{x[e], t + e};
      }
      if (c.out != nullptr) {
        float *o = c.out + start + t;
        if (t >= t0 && t + PE <= t1) {
#pragma unroll
          for (int e = 0; e < PE; e += 4) *reinterpret_cast<f32x4 *>(o + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        } else {
#pragma unroll
          for (int e = 0; e < PE; ++e)
            if (t + e >= t0 && t + e < t1) o[e] = x[e];
        }
      }
    }
    // the piece's best: a thread's tokens ascend, so the greatest value's first is its lowest; between threads the lower token
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) {
      const float v = __shfl_xor(best.value, o);
      const int t = __shfl_xor(best.token, o);
      if (t >= 0 && (v > best.value || (v == best.value && t < best.token))) best = Best{v, t};
    }
    if (threadIdx.x % kWave == 0) s_best[threadIdx.x / kWave] = best;
    __syncthreads();
    if (in_piece(mine)) atomicSub(&s_word[mine - t0], 1u);
    if (threadIdx.x == 0) {
#pragma unroll
      for (int w = 1; w < kLogitThreads / kWave; ++w) {
        const Best o = s_best[w];
        if (o.token >= 0 && (o.value > best.value || (o.value == best.value && o.token < best.token))) best = o;
      }
      part[at * pieces + blockIdx.x] = best;
    }
    __syncthreads();
  }
}

// One wave per row: the best of its pieces.  The first row's wave of a request raises what is wrong with it (here, where no
// other workgroup looks at the status word any more).
__global__ __launch_bounds__(kWave) void logits_best_kernel(LogitsCall c, int pieces, const Best *__restrict__ part) {
  const int b = blockIdx.y, row = blockIdx.x, lane = threadIdx.x;
  LogitsReq r;
  const bool good = logits_request(c, b, &r);
  if (!good) {
    if (row == 0 && lane == 0) raise_status(c.status, SONIC_ERR_BAD_LAYOUT);
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
