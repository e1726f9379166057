// Block-scaled products with what stands behind them, for few rows.
#include "cdl_act_thin.h"

namespace cdl {

int launch_thin_any(const ThinJob &job, int qt, bool gated, int y_type, int a_format, int b_format, hipStream_t stream)
{
    if (gated) return y_type == CDL_BF16 ? launch_thin<true, bf16_t>(job, qt, a_format, b_format, stream) : launch_thin<true, float>(job, qt, a_format, b_format, stream);
    return y_type == CDL_BF16 ? launch_thin<false, bf16_t>(job, qt, a_format, b_format, stream) : launch_thin<false, float>(job, qt, a_format, b_format, stream);
}

}  // namespace cdl
