// Instantiation unit: row processing kernels for fp32 rows.
#include "ctcbeam_process.inl"

namespace ctcbeam {
hipError_t launch_process_f32(const ProcessParams& p, void* workspace, hipStream_t s) { return rows::launch_process_impl<float>(p, workspace, s); }
}  // namespace ctcbeam
