// The chains of keys up to 64 wide.
#include "luna_delta_chain.cuh"

namespace luna {

cudaError_t launch_delta_chain64(const DeltaArgs &a, bool reverse, cudaStream_t s) { return chain_of<64>(a, reverse, s); }

}  // namespace luna
