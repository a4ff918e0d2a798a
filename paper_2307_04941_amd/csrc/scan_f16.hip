// The scan kernels on f16 activations.
#include "scan_kernel.h"

namespace mg3m {

ScanFn scan_kernel_f16(int P, int F, bool ends) { return scan_kernel<_Float16>(P, F, ends); }

}  // namespace mg3m
