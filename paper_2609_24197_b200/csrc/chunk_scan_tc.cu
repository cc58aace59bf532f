// Scan of requests with many rows: operands in two parts, for outputs of 16 bits and for states alone.
#include "chunk_scan_tc.cuh"

namespace hspec {

cudaError_t scan_long_launch(const LongArgs& a, cudaStream_t stream) { return scan_wide(a.c) ? scan_long_wide_launch(a, stream) : launch_long<false>(a, stream); }

}  // namespace hspec
