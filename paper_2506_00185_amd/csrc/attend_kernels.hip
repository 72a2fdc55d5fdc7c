// The attention kernels of one element type (RB_AT_TYPE) and one format of the cache (RB_AT_FMT): built once for each.
#include "token_host.h"

#include <type_traits>

#include "token_attend.h"

namespace rb {

template <typename TT, int FMT>
int launch_attend(const AttendArgs &a, int dp, int mt, int64_t blocks, hipStream_t stream) {
  int rc;
  if (dp == 64) {
    if constexpr (FMT == 16) rc = launch(mt == 1 ? k_attend<TT, FMT, 64, 1> : k_attend<TT, FMT, 64, 2>, blocks, 1, 256, a, stream);
    else rc = launch(k_attend<TT, FMT, 64, 1>, blocks, 1, 256, a, stream);
  }
  else if (dp == 128) rc = launch(mt == 1 ? k_attend<TT, FMT, 128, 1> : k_attend<TT, FMT, 128, 2>, blocks, 1, 256, a, stream);
  else rc = launch(k_attend<TT, FMT, 256, 1>, blocks, 1, 256, a, stream);
  if (rc || a.splits == 1) return rc;
  const int rows = 256 / (a.c.dim / 4 * a.join_shares);
  return launch(k_attend_join<TT>, ((int64_t)a.B * a.c.heads * a.rows + rows - 1) / rows, 1, 256, a, stream);
}

template int launch_attend<RB_AT_TYPE, RB_AT_FMT>(const AttendArgs &, int, int, int64_t, hipStream_t);

}  // namespace rb
