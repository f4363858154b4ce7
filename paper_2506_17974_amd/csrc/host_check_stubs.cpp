// Stand-ins for the kernel launchers, for the host-only sanitizer build: the planner and the
// argument checking of the C ABI are linked without any device code.  Nothing here is part of
// the library; every launcher reports that it cannot run.
#include "lqsgd_block_kernels.h"
#include "lqsgd_kernels.h"
#include "lqsgd_linear_kernels.h"

namespace lqsgd {

const char* last_launched_kernel() { return ""; }
hipError_t launch_add_project(int, const DevArgs&, const Tile*, int, int, int, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_orth(int, int, int, int64_t, const DevArgs&, CoopState*, bool*, hipStream_t) { return hipErrorNotSupported; }
int chol_entries(int) { return 0; }
hipError_t launch_exchange(int, int, const DevArgs&, const XTile*, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_back_project(int, const DevArgs&, const Tile*, int, const VTile*, int, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_back_project_mfma(int, const DevArgs&, const Tile*, int, const VTile*, int, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_reduce_q(int, const DevArgs&, const RTile*, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_residual(int, int, const DevArgs&, const Tile*, int, int, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_pad_factor(int, int, const DevArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_mfma_sweep(int, int, const DevArgs&, const Tile*, int, int, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t static_scratch(int, void**, void**, void**) { return hipErrorNotSupported; }
hipError_t launch_fill_zero(void*, size_t, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_write_pointers(const void**, const void* const*, size_t, hipStream_t) { return hipErrorNotSupported; }

namespace linear {

hipError_t launch_product(int, int, const ProductArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_checkpoint_save(int, int64_t, int32_t, const void*, int64_t, Codes, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_checkpoint_load(int, int64_t, int32_t, Codes, void*, int64_t, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_prepare(float*, int*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_activation_backward(int, int, int64_t, int32_t, const void*, int64_t, Codes, void*, int64_t, float*, int, void*, const float*,
                                      hipStream_t) {
  return hipErrorNotSupported;
}
hipError_t launch_rows_save(int, int64_t, int32_t, const void*, int64_t, Rows, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_rows_load(int, int64_t, int32_t, Rows, void*, int64_t, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_rms_norm(int, const NormArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_rms_norm_backward(int, const NormBackwardArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_dropout(int, const DropoutArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_int8_product(int, const Int8Args&, hipStream_t) { return hipErrorNotSupported; }

}  // namespace linear
}  // namespace lqsgd
