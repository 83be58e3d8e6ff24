// The choice of the 8-bit products' kernel, for tests without a GPU: built together with speca_matmul8_plan.cpp.
#include "speca_layer_internal.h"

extern "C" void host_plan_matmul8(int m, int n, int k, int dtype, int eight, int vectors, int masked, int sm_count, int* kernel, int* rows, int* ranks) {
    static char out;
    static uint8_t mask;
    speca::Matmul8Params p{};
    p.m = m, p.n = n, p.k = k, p.vectors = vectors;
    p.out = eight ? nullptr : &out;
    p.dev_mask = masked ? &mask : nullptr;
    const speca::Matmul8Plan plan = speca::plan_matmul8(p, dtype, sm_count);
    *kernel = plan.kernel, *rows = plan.few.rows, *ranks = plan.few.ranks;
}
