// Whole layers on rows of f16 (layer.cu); a file of its own for each type because it takes long to compile.
#include "layer_kernels.cuh"

int32_t launch_layer_f16(rtma_ctx* ctx, grouped::LayerArgs& a, int loading, bool gated, bool gradient, unsigned grid, cudaStream_t stream) {
    return launch_of_type<__half>(ctx, a, loading, gated, gradient, grid, stream);
}
