// Scan of requests with many rows: operands in three parts, for outputs of 32 bits.
#include "chunk_scan_tc.cuh"

namespace hspec {

cudaError_t scan_long_wide_launch(const LongArgs& a, cudaStream_t stream) { return launch_long<true>(a, stream); }

}  // namespace hspec
