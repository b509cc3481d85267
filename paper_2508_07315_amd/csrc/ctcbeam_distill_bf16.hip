// Instantiation unit: distillation kernels for bf16 rows.
#include "ctcbeam_distill.inl"

namespace ctcbeam {
hipError_t launch_distill_bf16(const DistillParams& p, void* workspace, hipStream_t s) { return rows::launch_distill_impl<rows::BF16>(p, workspace, s); }
}  // namespace ctcbeam
