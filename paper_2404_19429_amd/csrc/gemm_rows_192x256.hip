// The wide bf16 kernel on 192 x 256 tiles: products of groups that share one buffer of
// rows, and the cross entropy's (see gemm.hip).
#include "gemm_wide.h"

namespace lmoe {

void run_rows_192x256(const WideCall& w, hipStream_t s) {
  if (w.kind >= WK_LSE && w.kind < WK_DW) run_xent_m<Tile192>(w, s);
  else run_rows_m<Tile192>(w, s);
}

}  // namespace lmoe
