// Instantiation unit: top-logit kernels for bf16 rows.
#include "ctcbeam_top.inl"

namespace ctcbeam {
hipError_t launch_top_bf16(const TopParams& p, void* workspace, hipStream_t s) { return rows::launch_top_impl<rows::BF16>(p, workspace, s); }
}  // namespace ctcbeam
