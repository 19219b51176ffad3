// Decode over bf16 rows: how a call is cut into workgroups, the workspaces, and the kernel's variants
// without weights (decode_kernel.h; decode_q4.hip and decode_weighted.hip hold the others).
#include "decode_kernel.h"

#include <algorithm>

namespace sonic {

// Splits per (request, kv-head).  With fewer than 256 pairs the grid takes as many splits
// as give every CU a workgroup (64 pairs of 1.3k rows: 4 splits took 13.7 us per call and 5
// took 18.3, with eight waves a workgroup), each of at least 256 rows, and at most 16 (the
// merging split loads sixteen partials per memory round trip; 16 pairs of ~8k rows: 8 splits
// took 19.0 us per call and 16 took 18.5, 22.6 against 24.6 us with the caches cold).  With
// 256 pairs or more, unless the rows are shared (see decode_shape), one split, or three when
// the longest context reaches 2048 rows, so that the longest pairs do not outlast the rest
// of the call when lengths are uneven (512 pairs of 180 .. 4,300 rows: 1 split took 127.7
// us, 2 117.1, 3 111.4, 4 121.3 per call).
static int decode_splits(int batch, int Hkv, int max_ctx) {
  const long pairs = static_cast<long>(batch) * Hkv;
  if (pairs >= 256) return max_ctx >= 2048 ? 3 : 1;
  long s = 256 / pairs;
  const long by_rows = (static_cast<long>(max_ctx) + 255) / 256;
  if (s > by_rows) s = by_rows;
  if (s > kMaxSplits) s = kMaxSplits;
  return static_cast<int>(s < 1 ? 1 : s);
}

// How a call is cut into workgroups.
DecodeShape decode_shape(int batch, int Hkv, int G, int D, int max_ctx, bool masked, size_t part_bytes) {
  DecodeShape sh{decode_splits(batch, Hkv, max_ctx), 0, 8, 0};
  const long pairs = static_cast<long>(batch) * Hkv;
  auto part = [&](long slots) { return static_cast<size_t>(slots) * G * (D + 2) * sizeof(float); };
  // what a call needs, however it is cut: a smaller workspace is refused
  const size_t least = sh.splits > 1 ? part(pairs * sh.splits) : 0;
  // Evenly shared rows (see the kernel) where a call fills the GPU several times over and
  // contexts may be long and uneven.  512 four-wave workgroups are resident, `target` is whole
  // rounds of them: two for 256 pairs, a round more for every 256 pairs (half as many again
  // where contexts may pass 6k rows: a finer cut costs 2 us of 14 with short ranges and gains
  // 10 of 260 with long ones).  Measured against three splits a pair, 32 / 8 heads: 64 contexts
  // of 100 .. 4,000 rows 51.8 us and 58.7, 32 of 100 .. 8,000 47.3 and 51.7, 64 of 4,000 195
  // and 197, 64 of 100 (under a bound of 8,192) 17.2 and 20.5.  From 1,024 pairs on three
  // splits do as well or better (16 / 16 heads, 64 of 100 .. 4,000 rows 117 and, shared, 145).
  // Fewer than 256 pairs keep a split per pair and range: there the plan and the count over
  // the whole call cost 2.4 us of 12 and evenness gains less.
  if (!masked && batch <= kWave && pairs >= 256 && pairs < 1024 && max_ctx >= 2048) {
    const long rounds = std::max(2L, max_ctx < 6144 ? (pairs + 255) / 256 : (3 * pairs + 511) / 512);
    const long target = 512 * rounds / Hkv, launched = target + (batch + 15) / 16;
    if (std::max(least, part(launched * Hkv)) <= part_bytes) {
      sh.target = static_cast<int>(target);
      sh.splits = static_cast<int>(launched);
    }
  }
  const long slots = sh.target > 0 ? static_cast<long>(sh.splits) * Hkv : pairs * sh.splits;
  sh.part_bytes = std::max(least, sh.target > 0 ? part(slots) : 0);
  // Four waves, two workgroups per CU, or eight, one per CU.  Of two workgroups one starts and
  // merges while the other streams; eight waves keep more loads in flight where a CU has one
  // workgroup, and even out contexts of uneven length.  D = 128, 32 / 8 heads, four and eight
  // waves: 512 pairs of 200 rows 13.7 and 18.1 us, 64 of 1.3k rows in four ranges each 12.1 and
  // 13.0, 64 of 64 rows 5.1 and 5.5; 8 pairs of 8k rows 13.0 and 11.8, 400 of 80 .. 1,900 rows
  // 33.0 and 28.0.  Between 256 and 768 workgroups equal contexts would gain from four (400
  // pairs of 500 rows 21.7 and 24.6, 576 of 1,000 55.1 and 60.6) what uneven ones lose, so
  // four are taken there only for short ranges and where one round of 512 is nearly full.
  // D = 64 fits twice on a CU with eight (64 pairs of 4k rows 13.0, with four 13.4).
  const bool tiny = max_ctx <= 256L * sh.splits;
  const bool two = (slots >= 480 && slots <= 512) || slots > 768;
  const bool brief = slots >= 256 && slots < 480 && max_ctx <= 512L * sh.splits;
  if (sh.target > 0 || (!masked && (tiny || (D == 128 && (two || brief))))) sh.waves = 4;
  return sh;
}

// The same for 4-bit rows.  A row is a quarter of the bytes, so a call is sooner short of work than of bandwidth: ranges
// are longer and waves fewer.  Times of a step, 32 / 8 heads of 128.
// - Fewer than 256 pairs: about as many ranges as give every CU a workgroup, of 256 rows and more, and one up to 448 rows
//   (the hand-over between workgroups costs 1.3 us of 6.8: 8 requests of 100 rows, one range and two; 400 rows, one range
//   8.8 us and four 8.7; 1,328 rows, two ranges 11.8, four 10.0, eight 11.7; one request of 8,000 rows, 16 ranges 11.2
//   and 32 11.8, and of 100,001 rows, 16 ranges 44 and 32 30).
// - Four waves up to 512 rows a range, eight above, which keep more loads in flight and divide the work finer
//   (8 requests of 1,328 rows in four ranges, four waves 10.0 and eight 10.4; of 4,000 rows 14.6 and 14.1; 24 of 4,000
//   rows in one range 30.3 and 26.4).
// - 256 pairs and more with long contexts share the rows evenly (see decode_shape) among 1,024 workgroups of four waves,
//   all of them resident: 64 of 180 .. 4,300 rows 36.7 us, with 768 workgroups 39.9, 1,536 38.1 and a range
//   per pair and 512 rows 39.  More requests or pairs than that, or shorter contexts, keep a range per pair, which evens out
//   by itself: 128 of 180 .. 4,300 rows 69 us a step and in three ranges each (what bf16 rows take) 89, 128 of 4,000 142 and
//   156, 512 of 100 .. 2,500 155 and 263, 64 of 180 .. 4,300 with 16 kv-heads 68 and 81, 128 of 100 under a bound of 4,096
//   20 and 52, 70 of 100 .. 8,000 69 and 69.
DecodeShape decode_shape_q4(int batch, int Hkv, int G, int D, int max_ctx) {
  DecodeShape sh{1, 0, 4, 0};
  const long pairs = static_cast<long>(batch) * Hkv;
  long slots = pairs;
  if (pairs >= 256 && pairs < 1024 && batch <= kWave && max_ctx >= 2048) {
    sh.target = static_cast<int>(std::max(1024L / Hkv, static_cast<long>(batch)));   // (a request takes one at least)
    sh.splits = sh.target + (batch + 15) / 16;
    slots = static_cast<long>(sh.splits) * Hkv;
  } else {
    const long by_rows = max_ctx <= 448 ? 1 : (static_cast<long>(max_ctx) + 255) / 256;
    long most = 256 / pairs;
    if (most > kMaxSplits && max_ctx < 512L * most) most = kMaxSplits;
    sh.splits = static_cast<int>(std::max(1L, std::min({most, by_rows, static_cast<long>(kMaxSplitsQ4)})));
    slots = pairs * sh.splits;
    if (max_ctx > 512L * sh.splits) sh.waves = 8;
  }
  sh.part_bytes = sh.splits > 1 ? static_cast<size_t>(slots) * G * (D + 2) * sizeof(float) : 0;
  return sh;
}

// Fixed layout of a scratch array shared by calls of different shapes: the counters
// sit at the same offsets for every call (each call leaves them at zero), the partial
// records after them.  Returns the bytes a call needs, or 0 when its requests or
// (request, kv-head) pairs exceed the fixed counter regions.
size_t decode_scratch_layout(int batch, int Hkv, size_t part_bytes, DecodeWs *ws, char *base) {
  if (batch > kScratchMaxRequests || static_cast<long>(batch) * Hkv > kScratchMaxPairs) return 0;
  if (ws) {
    ws->done = reinterpret_cast<int32_t *>(base);
    ws->arrive = reinterpret_cast<int32_t *>(base + kScratchMaxRequests * sizeof(int32_t));
    ws->part = reinterpret_cast<float *>(base + kScratchCounterBytes);
  }
  return kScratchCounterBytes + part_bytes;
}

size_t decode_ws_layout(int batch, int Hkv, size_t part_bytes, DecodeWs *ws, char *base) {
  const size_t dbytes = (static_cast<size_t>(batch) * sizeof(int32_t) + 255) / 256 * 256;
  const size_t abytes = (static_cast<size_t>(batch) * Hkv * sizeof(int32_t) + 255) / 256 * 256;
  if (ws) {
    ws->done = reinterpret_cast<int32_t *>(base);
    ws->arrive = reinterpret_cast<int32_t *>(base + dbytes);
    ws->part = reinterpret_cast<float *>(base + dbytes + abytes);
  }
  return dbytes + abytes + part_bytes;
}

hipError_t launch_decode(int batch, int Hq, int Hkv, int D, int max_ctx, const DecodeShape &sh, const DecodeCall &c,
                         const DecodeWs &ws, hipStream_t stream) {
  return launch_decode_rows<false, false>(batch, Hq, Hkv, D, max_ctx, sh, c, DecodeRows{}, ws, stream);
}

}  // namespace sonic
