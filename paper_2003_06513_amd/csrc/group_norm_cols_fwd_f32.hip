// Group normalisation with the channels last, forward, fp32.
#include "group_norm_cols.h"

namespace psc {
namespace gn {
template void cols_fwd<DT_F32>(const Plan&, int, const void*, const Params&, float, void*, float*, float*, float4*,
                               hipStream_t);
}  // namespace gn
}  // namespace psc
