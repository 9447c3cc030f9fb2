// Linear attention step by step on f16 tensors.
#include "k_attend_scan.cuh"

namespace mf {

mf_status attend_scan_f16(const AttendPass& p, int64_t rows, cudaStream_t s) { return run<__half>(p, rows, s); }

}  // namespace mf
