// Linear attention step by step on bf16 tensors.
#include "k_attend_scan.cuh"

namespace mf {

mf_status attend_scan_bf16(const AttendPass& p, int64_t rows, cudaStream_t s) { return run<__nv_bfloat16>(p, rows, s); }

}  // namespace mf
