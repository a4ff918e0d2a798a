// The scan kernels on f32 activations.
#include "scan_kernel.h"

namespace mg3m {

ScanFn scan_kernel_f32(int P, int F, bool ends) { return scan_kernel<float>(P, F, ends); }

}  // namespace mg3m
