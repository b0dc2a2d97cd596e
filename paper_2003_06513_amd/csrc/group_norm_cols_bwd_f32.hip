// Group normalisation with the channels last, backward, fp32.
#include "group_norm_cols.h"

namespace psc {
namespace gn {
template void cols_bwd<DT_F32>(const Plan&, int, const void*, const void*, const Params&, const float*, const float*, void*,
                               const Sums&, float2*, Tail, hipStream_t);
}  // namespace gn
}  // namespace psc
