// Whole layers on rows of bf16 (layer.cu); a file of its own for each type because it takes long to compile.
#include "layer_kernels.cuh"

int32_t launch_layer_bf16(rtma_ctx* ctx, grouped::LayerArgs& a, int loading, bool gated, bool gradient, unsigned grid, cudaStream_t stream) {
    return launch_of_type<__nv_bfloat16>(ctx, a, loading, gated, gradient, grid, stream);
}
