// Attention over a paged cache in 8 bits with a scale for each block of tokens and head.
#include "attend_launch.h"

namespace ngpu {

size_t attend8_workspace(const ngpu_kv_cache8_t &c, const ngpu_attend_t &a) { return workspace_of<E4m3>(c.cache, a); }

hipError_t launch_attend8(const ngpu_kv_cache8_t &c, const ngpu_attend_t &a, void *workspace, hipStream_t stream) {
    const unsigned block = unsigned(c.block);
    const Attend8 p{{c.cache, a}, c.k_scale, c.v_scale, c.k_scale_stride_page, c.k_scale_stride_block, c.k_scale_stride_head,
                    c.v_scale_stride_page, c.v_scale_stride_block, c.v_scale_stride_head, block,
                    block == 1 ? UINT32_MAX : unsigned((uint64_t(1) << 32) / block)};
    return c.cache.dtype == NGPU_F16 ? launch<F16, E4m3>(p, workspace, stream) : launch<Bf16, E4m3>(p, workspace, stream);
}

}  // namespace ngpu
