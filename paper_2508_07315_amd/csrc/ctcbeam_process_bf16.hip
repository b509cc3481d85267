// Instantiation unit: row processing kernels for bf16 rows.
#include "ctcbeam_process.inl"

namespace ctcbeam {
hipError_t launch_process_bf16(const ProcessParams& p, void* workspace, hipStream_t s) { return rows::launch_process_impl<rows::BF16>(p, workspace, s); }
}  // namespace ctcbeam
