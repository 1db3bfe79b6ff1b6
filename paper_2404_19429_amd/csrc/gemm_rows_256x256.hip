// The wide bf16 kernel on 256 x 256 tiles: products of groups that share one buffer of
// rows, and the cross entropy's (see gemm.hip).
#include "gemm_wide.h"

namespace lmoe {

void run_rows_256x256(const WideCall& w, hipStream_t s) {
  if (w.kind >= WK_LSE && w.kind < WK_DW) run_xent_m<Tile256>(w, s);
  else if (w.kind < WK_DW) run_rows_m<Tile256>(w, s);
  else run_rows_k<Tile256>(w, s);
}

}  // namespace lmoe
