// The gated tiles of the block-scaled product, results in fp32.
#include "cdl_act_ring.h"

namespace cdl {

int launch_gated_f32(ActForm form, const RingJob &job, const ActTarget &to, int a_format, int b_format, hipStream_t stream)
{
    return launch_act_ring<true, float>(form, job, to, a_format, b_format, stream);
}

}  // namespace cdl
