// Group normalisation in NCHW, forward, fp32.
#include "group_norm_rows.h"

namespace psc {
namespace gn {
template void rows_fwd<DT_F32>(const Plan&, int64_t, const void*, const Params&, float, void*, float*, float*, float4*,
                               hipStream_t);
}  // namespace gn
}  // namespace psc
