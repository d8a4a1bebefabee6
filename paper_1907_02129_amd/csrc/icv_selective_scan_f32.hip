// The scan's kernels (icv_selective_scan_kernel.h) for rows of float; its own translation unit for the build's parallelism.
#include "icv_selective_scan_kernel.h"

namespace icv {

int launch_scan_f32(const ScanArgs& a, const ScanPlan& plan, bool step, hipStream_t s) { return launch_scan<float>(a, plan, step, s); }

}  // namespace icv
