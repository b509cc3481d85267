// Instantiation unit: distillation kernels for fp32 rows.
#include "ctcbeam_distill.inl"

namespace ctcbeam {
hipError_t launch_distill_f32(const DistillParams& p, void* workspace, hipStream_t s) { return rows::launch_distill_impl<float>(p, workspace, s); }
}  // namespace ctcbeam
