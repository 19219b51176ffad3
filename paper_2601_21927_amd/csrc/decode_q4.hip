// Decode over 4-bit rows, with and without the scores for the rows' weights (decode_kernel.h).
#include "decode_kernel.h"

namespace sonic {

hipError_t launch_decode_q4(int batch, int Hq, int Hkv, int D, int max_ctx, const DecodeShape &sh, const DecodeCall &c,
                            const DecodeRows &rows, const DecodeWs &ws, hipStream_t stream) {
  return rows.scores != nullptr ? launch_decode_rows<true, true>(batch, Hq, Hkv, D, max_ctx, sh, c, rows, ws, stream)
                                : launch_decode_rows<true, false>(batch, Hq, Hkv, D, max_ctx, sh, c, rows, ws, stream);
}

}  // namespace sonic
