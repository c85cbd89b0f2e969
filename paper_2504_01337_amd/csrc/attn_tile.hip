// The launches of prompt attention in bf16 (attn_tile.h).
#include "attn_tile.h"

namespace c2r {

template <int D, bool ALIGNED, bool ANY_SCALE>
__global__ __launch_bounds__(256, D == 128 ? 2 : 4) void attn_tile_kernel(AttnCall a) {
    __shared__ __align__(1024) TileLds<D> lds;
    attn_tile_block<D, ALIGNED, ANY_SCALE, false>(a, blockIdx.x, lds);
}

int launch_attn_tile(const AttnCall &a, int D, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.splits * a.kv.kv_heads * a.row_blocks * (a.by_rows ? 1 : a.kv.batch))), block(256);
    const bool aligned = tile_aligned(a.kv);
    if (!(a.scale_log2 > 0.0f)) D == 128 ? attn_tile_kernel<128, false, true><<<grid, block, 0, st>>>(a) : attn_tile_kernel<64, false, true><<<grid, block, 0, st>>>(a);
    else if (D == 128) aligned ? attn_tile_kernel<128, true, false><<<grid, block, 0, st>>>(a) : attn_tile_kernel<128, false, false><<<grid, block, 0, st>>>(a);
    else aligned ? attn_tile_kernel<64, true, false><<<grid, block, 0, st>>>(a) : attn_tile_kernel<64, false, false><<<grid, block, 0, st>>>(a);
    const int rc = launch_status();
    return rc == C2R_OK && a.splits > 1 ? launch_attn_join(a, true, D, st) : rc;
}

}  // namespace c2r
