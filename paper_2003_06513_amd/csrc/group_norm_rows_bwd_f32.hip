// Group normalisation in NCHW, backward, fp32.
#include "group_norm_rows.h"

namespace psc {
namespace gn {
template void rows_bwd<DT_F32>(const Plan&, int64_t, const void*, const void*, const Params&, const float*, const float*, void*,
                               const Sums&, float2*, Tail, hipStream_t);
}  // namespace gn
}  // namespace psc
