// Instantiation unit: row processing kernels for fp16 rows.
#include "ctcbeam_process.inl"

namespace ctcbeam {
hipError_t launch_process_f16(const ProcessParams& p, void* workspace, hipStream_t s) { return rows::launch_process_impl<rows::F16>(p, workspace, s); }
}  // namespace ctcbeam
