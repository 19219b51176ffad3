// Cache rows read back and weighed: 4-bit rows to bf16 (bound by HBM: 30,208 rows of 4 heads of 128, 78 MB, 14.4 us, 5.4
// TB/s, and 1.2 for the launch that raises errors), the prefill's key weights to the rows they were compacted to (three
// dependent round trips, 3.6 us, and 2.1 for the errors), and the attention weights of a decode step added to its rows (4 to
// 8 us).
#include <algorithm>

#include "common.h"
#include "q4.h"

namespace sonic {

constexpr int kRowThreads = 256;
constexpr int kExpandUnroll = 4;

// What is wrong with request b's range, or 0.
__device__ __forceinline__ int range_error(int r0, int r1, int cap, int room, int max_rows) {
  if (r0 < 0 || r1 < r0 || r1 > cap) return SONIC_ERR_BAD_LAYOUT;
  return r1 - r0 > room ? SONIC_ERR_CAPACITY : r1 - r0 > max_rows ? SONIC_ERR_INVALID_ARG : 0;
}

// Errors are raised by a kernel of their own, behind the one that writes: a workgroup that starts late takes a status word
// for one that was pending before the call, and would leave out its rows when another request's error is already in it.
__global__ __launch_bounds__(kRowThreads) void expand_errors_kernel(const int32_t *__restrict__ row_begin,
                                                                    const int32_t *__restrict__ row_end,
                                                                    const int32_t *__restrict__ row_cap,
                                                                    const int32_t *__restrict__ out_cap, int batch, int max_rows,
                                                                    int32_t *status) {
  const int b = blockIdx.x * kRowThreads + threadIdx.x;
  if (b >= batch) return;
  const int code = range_error(row_begin[b], row_end[b], row_cap[b], out_cap[b], max_rows);
  if (code != 0) raise_status(status, code);
}

// Request b's rows row_begin[b] .. row_end[b] to rows out_off[b] .. of k and v.  Grid (chunks of units, requests);
// a unit is eight values, four bytes of codes in and sixteen out, so that loads and stores are both whole lines.
__global__ __launch_bounds__(kRowThreads) void expand_q4_kernel(
    const uint32_t *__restrict__ kc, const uint8_t *__restrict__ kscale, const uint32_t *__restrict__ vc,
    const uint8_t *__restrict__ vscale, const int64_t *__restrict__ row_off, const int32_t *__restrict__ row_cap,
    const int32_t *__restrict__ row_begin, const int32_t *__restrict__ row_end, bf16x8 *__restrict__ k, bf16x8 *__restrict__ v,
    const int64_t *__restrict__ out_off, const int32_t *__restrict__ out_cap, int max_rows, int row_units, const int32_t *status) {
  __shared__ int s_ok;
  const int b = blockIdx.y;
  const int r0 = row_begin[b], r1 = row_end[b], cap = row_cap[b], room = out_cap[b];
  const int64_t off = row_off[b], out0 = out_off[b];
  if (!block_status_clear(status, &s_ok)) return;
  if (range_error(r0, r1, cap, room, max_rows) != 0) return;
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

// row_weight of request b's row j = the key weight of the prompt position keep_idx holds for it.  ERRORS: raises what is
// wrong, behind the launch that writes (see expand_errors_kernel); a word that holds an error keeps it.
template <bool ERRORS>
__global__ __launch_bounds__(kRowThreads) void compact_weights_kernel(
    const int32_t *__restrict__ cu, const float *__restrict__ key_weight, const int64_t *__restrict__ row_off,
    const int32_t *__restrict__ cache_len, const int32_t *__restrict__ keep_idx, float *__restrict__ row_weight,
    int total_tokens, int max_rows, int32_t *status) {
  __shared__ int s_ok;
  const int b = blockIdx.y;
  const int s = cu[b], e = cu[b + 1], len = cache_len[b];
  const int64_t off = row_off[b];
  if (!ERRORS && !block_status_clear(status, &s_ok)) return;
  if (s < 0 || e < s || e > total_tokens || len < 0 || len > max_rows) {
    if (ERRORS && blockIdx.x == 0 && threadIdx.x == 0)
      raise_status(status, len > max_rows ? SONIC_ERR_INVALID_ARG : SONIC_ERR_BAD_LAYOUT);
    return;
  }
  for (unsigned j = blockIdx.x * kRowThreads + threadIdx.x; j < static_cast<unsigned>(len); j += gridDim.x * kRowThreads) {
    const int p = keep_idx[off + j];
    const bool in = p >= 0 && p < e - s;
    if (ERRORS) {
      if (!in) raise_status(status, SONIC_ERR_BAD_LAYOUT);
    } else if (in) {
      row_weight[off + j] = key_weight[s + p];
    }
  }
}

// After a decode step that kept its scores: row r's weight grows by the mean over the q-heads of
// exp2(score - normaliser); the appended row's starts there.  Requests the step did not advance (fresh 0) are left
// alone.  A wave takes K blocks of 16 rows: lane l has rows 4 (l % 4) .. + 3 of heads l / 4, l / 4 + 16, .., and the
// lanes' sums are added by exchanges in a fixed order, so they do not depend on timing.  Bound by the launch and its
// round trips, one after the other (scores and normalisers of 16 heads at a time, K = 1: then the length, the old weight):
// 8 requests of 1,328 rows, 32 heads, 4 us with K = 1, 5 with K = 4.
constexpr int kWeightWaves = 4;
template <int K>
__global__ __launch_bounds__(kWave *kWeightWaves) void add_weights_kernel(const int64_t *__restrict__ row_off, DecodeRows rows,
                                                                          float *__restrict__ row_weight, int Hq, float inv_heads) {
  const int b = blockIdx.y;
  const int n = rows.fresh[b];
  const int64_t off = row_off[b];
  const int lane = threadIdx.x % kWave;
  const int r0 = (blockIdx.x * kWeightWaves + static_cast<int>(threadIdx.x) / kWave) * (16 * K);
  // K = 1, few workgroups: the scores are requested before the request's length is known (its blocks have room)
  if (K > 1 && r0 >= n) return;
  const float *lse = rows.lse + static_cast<size_t>(b) * Hq;
  const float *scores = rows.scores + static_cast<size_t>(b) * Hq * rows.stride + 4 * (lane % 4);
  f32x4 sum[K] = {};
  for (int h0 = 0; h0 < Hq; h0 += 16) {
    const bool in = h0 + lane / 4 < Hq;
    const int h = in ? h0 + lane / 4 : 0;
    const float l = lse[h];
    f32x4 s[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const size_t blk = min(static_cast<size_t>(r0 / 16 + k), rows.stride / 16 - 1);
      s[k] = *reinterpret_cast<const f32x4 *>(scores + (blk * Hq + h) * 16);
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[k][e] += in ? __builtin_amdgcn_exp2f(s[k][e] - l) : 0.f;
  }
  if (r0 >= n) return;
  const int r = r0 + lane;   // lane 16 k + 4 i + e: element e of the lanes i of block k
  const bool mine = lane < 16 * K && r < n;
  float *w = row_weight + off + r;
  const float old = mine && r < n - 1 ? *w : 0.f;
  float total = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x = sum[k][e];
      x += __shfl_xor(x, 4);
      x += __shfl_xor(x, 8);
      x = pair32_add(pair16_add(x));
      const float y = __shfl(x, lane / 4 % 4);
      if (lane / 16 == k && lane % 4 == e) total = y;
    }
  if (mine) *w = fmaf(total, inv_heads, old);
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
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  expand_errors_kernel<<<dim3((batch + kRowThreads - 1) / kRowThreads), dim3(kRowThreads), 0, stream>>>(row_begin, row_end, row_cap,
                                                                                                        out_cap, batch, max_rows, status);
  return hipGetLastError();
}

hipError_t launch_compact_weights(int batch, int total_tokens, int max_rows, const int32_t *cu, const float *key_weight,
                                  const int64_t *row_off, const int32_t *cache_len, const int32_t *keep_idx, float *row_weight,
                                  int32_t *status, hipStream_t stream) {
  // (max_rows is the caller's bound, and may be any number)
  const long chunks = (static_cast<long>(max_rows) + kRowThreads - 1) / kRowThreads;
  const dim3 grid(std::max(1L, std::min(chunks, std::max(16L, 4096L / batch))), batch);
  compact_weights_kernel<false><<<grid, dim3(kRowThreads), 0, stream>>>(cu, key_weight, row_off, cache_len, keep_idx, row_weight,
                                                                        total_tokens, max_rows, status);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  compact_weights_kernel<true><<<grid, dim3(kRowThreads), 0, stream>>>(cu, key_weight, row_off, cache_len, keep_idx, row_weight,
                                                                       total_tokens, max_rows, status);
  return hipGetLastError();
}

hipError_t launch_add_weights(int batch, int Hq, int max_ctx, const int64_t *row_off, const DecodeRows &rows, float *row_weight,
                              hipStream_t stream) {
  const float inv = 1.f / static_cast<float>(Hq);
  auto blocks = [&](long k) { return (max_ctx + 16 * k * kWeightWaves - 1) / (16 * k * kWeightWaves); };
  if (blocks(1) * batch <= 1024)
    add_weights_kernel<1><<<dim3(blocks(1), batch), dim3(kWave * kWeightWaves), 0, stream>>>(row_off, rows, row_weight, Hq, inv);
  else
    add_weights_kernel<4><<<dim3(blocks(4), batch), dim3(kWave * kWeightWaves), 0, stream>>>(row_off, rows, row_weight, Hq, inv);
  return hipGetLastError();
}

}  // namespace sonic
