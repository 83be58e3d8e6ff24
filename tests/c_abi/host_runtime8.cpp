// The kernels of the 8-bit calls, counted instead of run: beside host_runtime.cpp, for tests of their argument checks without a GPU.
#include "speca_layer_internal.h"

namespace {
int norms = 0, products = 0;
int vectors = 0;
}  // namespace

extern "C" {
int host_norms() { return norms; }
int host_products() { return products; }
int host_vectors() { return vectors; }
}

namespace speca {
cudaError_t launch_norm8(const Norm8Params&, int, bool v, cudaStream_t) {
    ++norms;
    vectors = v;
    return cudaSuccess;
}
cudaError_t launch_matmul8(const Matmul8Params& p, int, int, cudaStream_t) {
    ++products;
    vectors = p.vectors;
    return cudaSuccess;
}
}  // namespace speca
