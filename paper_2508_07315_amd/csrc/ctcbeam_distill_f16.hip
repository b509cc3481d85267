// Instantiation unit: distillation kernels for fp16 rows.
#include "ctcbeam_distill.inl"

namespace ctcbeam {
hipError_t launch_distill_f16(const DistillParams& p, void* workspace, hipStream_t s) { return rows::launch_distill_impl<rows::F16>(p, workspace, s); }
}  // namespace ctcbeam
