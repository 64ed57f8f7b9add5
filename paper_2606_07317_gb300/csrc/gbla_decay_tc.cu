// Decayed linear attention on tensor cores: not covered yet, every scan runs on
// CUDA cores (gbla_decay.cu).
#include "gbla_internal.cuh"

namespace gbla {

bool tc_scan_supports(const ScanArgs &) { return false; }
size_t tc_scan_floats(const ScanArgs &) { return 0; }
cudaError_t tc_scan(const ScanArgs &, float *, cudaStream_t) { return cudaErrorNotSupported; }
unsigned decay_device_error(bool) { return 0; }

}  // namespace gbla
