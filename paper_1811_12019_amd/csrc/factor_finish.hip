// Second pass of the factor builds.
#include "factor_reduce.h"

namespace kfac {

// The second pass of a call's builds.  GROUPS 1: few row ranges, and factors from the parts that their tap pairs share; 4: many
// ranges.
template <int GROUPS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4, 8))) void factor_tile_reduce_kernel(FBatch b) {
    __shared__ __attribute__((aligned(16))) float lds[GROUPS == 1 ? SH_BLOCK_FLOATS : RD_MANY_FLOATS];
    int local;
    const int m = fbatch_locate(b, blockIdx.x, local);
    kfac_factor_item it;
    Unfold u;
    View v;
    fbatch_item(b, m, it, u, v);
    const float scale = it.scale == 0.f ? 1.0f / (float)u.R : it.scale;
    if constexpr (GROUPS == 1) {
        if (v.shared) {
            assemble_blocks(v, plan_shared(v, b.share[m]), shared_ws(v, it.ws), out_spec(it), scale, local, lds);
            return;
        }
    }
    const FactorPlan pl = plan_tiles(v, b.share[m]);
    reduce_partials<GROUPS>(v, pl, partial_of(v, pl, it.ws), out_spec(it), scale, local, lds);
}

// The same for shared parts in (channel, tap) order.
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4, 8))) void factor_channels_kernel(FBatch b) {
    __shared__ __attribute__((aligned(16))) float lds[SH_CHANNEL_FLOATS];
    int local;
    const int m = fbatch_locate(b, blockIdx.x, local);
    kfac_factor_item it;
    Unfold u;
    View v;
    fbatch_item(b, m, it, u, v);
    const float scale = it.scale == 0.f ? 1.0f / (float)u.R : it.scale;
    assemble_channels(v, plan_shared(v, b.share[m]), shared_ws(v, it.ws), out_spec(it), scale, local, lds);
}

int launch_factor_finish(const FBatch& b, int list, hipStream_t stream) {
    if (b.count == 0) return KFAC_OK;
    const dim3 grid(b.prefix[b.count]);
    if (list == FINISH_FEW) KFAC_LAUNCH(factor_tile_reduce_kernel<1>, grid, dim3(256), stream, b);
    else if (list == FINISH_MANY) KFAC_LAUNCH(factor_tile_reduce_kernel<4>, grid, dim3(256), stream, b);
    else KFAC_LAUNCH(factor_channels_kernel, grid, dim3(256), stream, b);
    return KFAC_OK;
}

}  // namespace kfac
