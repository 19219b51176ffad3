// Cache rows read back and weighed: 4-bit rows to bf16, the prefill's key weights to the rows they were
// compacted to, and the attention weights of a decode step added to its rows.
#include <algorithm>

#include "common.h"
#include "q4.h"

namespace sonic {

constexpr int kRowThreads = 256;
constexpr int kExpandUnroll = 4;

// Request b's rows row_begin[b] .. row_end[b] to rows out_off[b] .. of k and v.  Grid (chunks of units, requests);
// a unit is eight values, four bytes of codes in and sixteen out, so that loads and stores are both whole lines.
__global__ __launch_bounds__(kRowThreads) void expand_q4_kernel(
    const uint32_t *__restrict__ kc, const uint8_t *__restrict__ kscale, const uint32_t *__restrict__ vc,
    const uint8_t *__restrict__ vscale, const int64_t *__restrict__ row_off, const int32_t *__restrict__ row_cap,
    const int32_t *__restrict__ row_begin, const int32_t *__restrict__ row_end, bf16x8 *__restrict__ k, bf16x8 *__restrict__ v,
    const int64_t *__restrict__ out_off, const int32_t *__restrict__ out_cap, int max_rows, int row_units, int32_t *status) {
  __shared__ int s_ok;
  const int b = blockIdx.y;
  const int r0 = row_begin[b], r1 = row_end[b], cap = row_cap[b], room = out_cap[b];
  const int64_t off = row_off[b], out0 = out_off[b];
  if (!block_status_clear(status, &s_ok)) return;
  if (r0 < 0 || r1 < r0 || r1 > cap || r1 - r0 > room || r1 - r0 > max_rows) {
    if (blockIdx.x == 0 && threadIdx.x == 0)
      raise_status(status, r0 < 0 || r1 < r0 || r1 > cap ? SONIC_ERR_BAD_LAYOUT
                           : r1 - r0 > room              ? SONIC_ERR_CAPACITY
                                                         : SONIC_ERR_INVALID_ARG);
    return;
  }
  const long total = static_cast<long>(r1 - r0) * row_units;
  const size_t src0 = static_cast<size_t>(off + r0) * row_units, dst0 = static_cast<size_t>(out0) * row_units;
  const long step = static_cast<long>(gridDim.x) * kRowThreads;
  for (long u0 = static_cast<long>(blockIdx.x) * kRowThreads + threadIdx.x; u0 < total; u0 += step * kExpandUnroll) {
    uint32_t ck[kExpandUnroll], cv[kExpandUnroll], sk[kExpandUnroll], sv[kExpandUnroll];
#pragma unroll
    for (int i = 0; i < kExpandUnroll; ++i) {
      const long u = u0 + i * step;
      if (u < total) {
        ck[i] = kc[src0 + u];
        cv[i] = vc[src0 + u];
        sk[i] = kscale[(src0 + u) / 4];
        sv[i] = vscale[(src0 + u) / 4];
      }
    }
#pragma unroll
    for (int i = 0; i < kExpandUnroll; ++i) {
      const long u = u0 + i * step;
      if (u < total) {
        k[dst0 + u] = q4_decode8(ck[i], q4_scale(sk[i]));
        v[dst0 + u] = q4_decode8(cv[i], q4_scale(sv[i]));
      }
    }
  }
}

// row_weight of request b's row j = the key weight of the prompt position keep_idx holds for it.
__global__ __launch_bounds__(kRowThreads) void compact_weights_kernel(
    const int32_t *__restrict__ cu, const float *__restrict__ key_weight, const int64_t *__restrict__ row_off,
    const int32_t *__restrict__ cache_len, const int32_t *__restrict__ keep_idx, float *__restrict__ row_weight,
    int total_tokens, int max_rows, int32_t *status) {
  __shared__ int s_ok;
  const int b = blockIdx.y;
  const int s = cu[b], e = cu[b + 1], len = cache_len[b];
  const int64_t off = row_off[b];
  if (!block_status_clear(status, &s_ok)) return;
  if (s < 0 || e < s || e > total_tokens || len < 0 || len > max_rows) {
    if (blockIdx.x == 0 && threadIdx.x == 0)
      raise_status(status, len > max_rows ? SONIC_ERR_INVALID_ARG : SONIC_ERR_BAD_LAYOUT);
    return;
  }
  const int j = blockIdx.x * kRowThreads + threadIdx.x;
  if (j >= len) return;
  const int p = keep_idx[off + j];
  if (p < 0 || p >= e - s) raise_status(status, SONIC_ERR_BAD_LAYOUT);
  else row_weight[off + j] = key_weight[s + p];
}

// After a decode step that kept its scores: row r's weight grows by the mean over the q-heads of
// exp2(score - normaliser); the appended row's starts there.  Requests the step did not advance (fresh 0) are left
// alone.  A workgroup has 64 rows, a wave a quarter of the heads (kHeadUnroll of them in flight, requested before the
// request's length is known: every row of the grid has room), and the waves' sums are added in order, so they do not
// depend on timing.
constexpr int kWeightRows = kWave, kWeightWaves = 4, kHeadUnroll = 8;
__global__ __launch_bounds__(kWeightRows *kWeightWaves) void add_weights_kernel(const int64_t *__restrict__ row_off, DecodeRows rows,
                                                                                float *__restrict__ row_weight, int Hq,
                                                                                float inv_heads) {
  __shared__ float part[kWeightWaves][kWeightRows];
  const int b = blockIdx.y;
  const int n = rows.fresh[b];
  const int64_t off = row_off[b];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = blockIdx.x * kWeightRows + lane;
  // (with many workgroups the traffic of those past the request's end counts for more than the round trip)
  if (gridDim.x * gridDim.y > 2048 && static_cast<int>(blockIdx.x) * kWeightRows >= n) return;
  const float *score = rows.scores + static_cast<size_t>(b) * Hq * rows.stride + min(static_cast<size_t>(r), rows.stride - 1);
  const float *lse = rows.lse + static_cast<size_t>(b) * Hq;
  const int per = (Hq + kWeightWaves - 1) / kWeightWaves, h0 = wave * per, h1 = min(Hq, h0 + per);
  float sum = 0.f;
  for (int h = h0; h < h1; h += kHeadUnroll) {
    float s[kHeadUnroll], l[kHeadUnroll];
#pragma unroll
    for (int i = 0; i < kHeadUnroll; ++i) {
      const int hh = min(h + i, h1 - 1);
      s[i] = score[hh * rows.stride];
      l[i] = lse[hh];
    }
#pragma unroll
    for (int i = 0; i < kHeadUnroll; ++i)
      if (h + i < h1) sum += __builtin_amdgcn_exp2f(s[i] - l[i]);
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave > 0 || r >= n) return;
  float *w = row_weight + off + r;
  const float old = r == n - 1 ? 0.f : *w;
#pragma unroll
  for (int i = 1; i < kWeightWaves; ++i) sum += part[i][lane];
  *w = fmaf(sum, inv_heads, old);
}

hipError_t launch_expand_q4(int batch, int max_rows, int Hkv, int D, const uint8_t *kc, const uint8_t *ks, const uint8_t *vc,
                            const uint8_t *vs, const int64_t *row_off, const int32_t *row_cap, const int32_t *row_begin,
                            const int32_t *row_end, uint16_t *k, uint16_t *v, const int64_t *out_off, const int32_t *out_cap,
                            int32_t *status, hipStream_t stream) {
  const int row_units = Hkv * D / 8;
  const long units = static_cast<long>(max_rows) * row_units;
  const long chunks = std::max(1L, std::min((units + kRowThreads * kExpandUnroll - 1) / (kRowThreads * kExpandUnroll),
                                            std::max(16L, 4096L / batch)));
  expand_q4_kernel<<<dim3(chunks, batch), dim3(kRowThreads), 0, stream>>>(
      reinterpret_cast<const uint32_t *>(kc), ks, reinterpret_cast<const uint32_t *>(vc), vs, row_off, row_cap, row_begin, row_end,
      reinterpret_cast<bf16x8 *>(k), reinterpret_cast<bf16x8 *>(v), out_off, out_cap, max_rows, row_units, status);
  return hipGetLastError();
}

hipError_t launch_compact_weights(int batch, int total_tokens, int max_rows, const int32_t *cu, const float *key_weight,
                                  const int64_t *row_off, const int32_t *cache_len, const int32_t *keep_idx, float *row_weight,
                                  int32_t *status, hipStream_t stream) {
  compact_weights_kernel<<<dim3(std::max(1, (max_rows + kRowThreads - 1) / kRowThreads), batch), dim3(kRowThreads), 0, stream>>>(
      cu, key_weight, row_off, cache_len, keep_idx, row_weight, total_tokens, max_rows, status);
  return hipGetLastError();
}

hipError_t launch_add_weights(int batch, int Hq, int max_ctx, const int64_t *row_off, const DecodeRows &rows, float *row_weight,
                              hipStream_t stream) {
  add_weights_kernel<<<dim3((max_ctx + kWeightRows - 1) / kWeightRows, batch), dim3(kWeightRows * kWeightWaves), 0, stream>>>(
      row_off, rows, row_weight, Hq, 1.f / static_cast<float>(Hq));
  return hipGetLastError();
}

}  // namespace sonic
