// Whole layers (layer.cu) on rows of f16; a file of its own for each type because it takes long to compile.
#include "layer_pairs.cuh"

RTMA_BOUNDS_TU()

int32_t launch_layer_f16(rtma_ctx* ctx, LayerArgs& a, bool gated, bool gradient, unsigned grid, cudaStream_t stream) {
    const bool resident = a.d_in <= RESIDENT_TERMS;
    if (gated) return resident ? launch_pairs<__half, true, true>(ctx, a, gradient, grid, stream) : launch_pairs<__half, true, false>(ctx, a, gradient, grid, stream);
    return resident ? launch_pairs<__half, false, true>(ctx, a, gradient, grid, stream) : launch_pairs<__half, false, false>(ctx, a, gradient, grid, stream);
}
