// Linear attention step by step on fp32 tensors, and the choice of the type.
#include "k_attend_scan.cuh"

namespace mf {

mf_status attend_scan(int type, const AttendPass& p, int64_t rows, cudaStream_t s) {
  if (type == MF_TYPE_F32) return run<float>(p, rows, s);
  return type == MF_TYPE_BF16 ? attend_scan_bf16(p, rows, s) : attend_scan_f16(p, rows, s);
}

}  // namespace mf
