// Attention over a paged cache of half or bfloat16 values.
#include "attend_launch.h"

namespace ngpu {

size_t attend_workspace(const ngpu_kv_cache_t &c, const ngpu_attend_t &a) {
    return c.dtype == NGPU_F16 ? workspace_of<F16>(c, a) : workspace_of<Bf16>(c, a);
}

hipError_t launch_attend(const ngpu_kv_cache_t &c, const ngpu_attend_t &a, void *workspace, hipStream_t stream) {
    const Attend p{c, a};
    return c.dtype == NGPU_F16 ? launch<F16, F16>(p, workspace, stream) : launch<Bf16, Bf16>(p, workspace, stream);
}

}  // namespace ngpu
