// The wide bf16 kernel on 128 x 128 tiles: products of groups that share one buffer of
// rows, and the cross entropy's (see gemm.hip).
#include "gemm_wide.h"

namespace lmoe {

void run_rows_128x128(const WideCall& w, hipStream_t s) {
  if (w.kind >= WK_LSE && w.kind < WK_DW) run_xent_m<Tile128>(w, s);
  else if (w.kind < WK_DW) run_rows_m<Tile128>(w, s);
  else run_rows_k<Tile128K>(w, s);
}

}  // namespace lmoe
