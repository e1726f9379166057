// The tiles with an activation of the block-scaled product, results in bf16.
#include "cdl_act_ring.h"

namespace cdl {

int launch_act_bf16(ActForm form, const RingJob &job, const ActTarget &to, int a_format, int b_format, hipStream_t stream)
{
    return launch_act_ring<false, bf16_t>(form, job, to, a_format, b_format, stream);
}

}  // namespace cdl
