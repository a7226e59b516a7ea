// The chains of keys of 65 to 128 values.
#include "luna_delta_chain.cuh"

namespace luna {

cudaError_t launch_delta_chain128(const DeltaArgs &a, bool reverse, cudaStream_t s) { return chain_of<128>(a, reverse, s); }

}  // namespace luna
