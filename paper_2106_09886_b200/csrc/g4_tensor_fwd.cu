// Forward instantiations of the grouped product on tensor memory.
#include "g4_tensor_run.cuh"

int qnn_g4_tensor_fwd(const void *x, int type, int64_t ldx, const G4TensorArgs &a, cudaStream_t st) {
    return g4_tensor_run<G4_FWD>(x, type, ldx, a, st);
}
