// Decode over bf16 rows that keeps the scores for the rows' weights (decode_kernel.h; rows.hip adds them up).
#include "decode_kernel.h"

namespace sonic {

hipError_t launch_decode_weighted(int batch, int Hq, int Hkv, int D, int max_ctx, const DecodeShape &sh, const DecodeCall &c,
                                  const DecodeRows &rows, const DecodeWs &ws, hipStream_t stream) {
  return launch_decode_rows<false, true>(batch, Hq, Hkv, D, max_ctx, sh, c, rows, ws, stream);
}

}  // namespace sonic
