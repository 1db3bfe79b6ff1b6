// The wide bf16 kernel on 64 x 64 tiles: products of groups that share one buffer of
// rows, and the cross entropy's (see gemm.hip).
#include "gemm_wide.h"

namespace lmoe {

void run_rows_64x64(const WideCall& w, hipStream_t s) {
  if (w.kind >= WK_LSE && w.kind < WK_DW) run_xent_m<Tile64>(w, s);
  else run_rows_m<Tile64>(w, s);
}

}  // namespace lmoe
