// Instantiation unit: top-logit kernels for fp32 rows.
#include "ctcbeam_top.inl"

namespace ctcbeam {
hipError_t launch_top_f32(const TopParams& p, void* workspace, hipStream_t s) { return rows::launch_top_impl<float>(p, workspace, s); }
}  // namespace ctcbeam
