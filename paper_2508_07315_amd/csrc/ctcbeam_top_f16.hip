// Instantiation unit: top-logit kernels for fp16 rows.
#include "ctcbeam_top.inl"

namespace ctcbeam {
hipError_t launch_top_f16(const TopParams& p, void* workspace, hipStream_t s) { return rows::launch_top_impl<rows::F16>(p, workspace, s); }
}  // namespace ctcbeam
