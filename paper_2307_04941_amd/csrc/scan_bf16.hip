// The scan kernels on bf16 activations.
#include "scan_kernel.h"

namespace mg3m {

ScanFn scan_kernel_bf16(int P, int F, bool ends) { return scan_kernel<__bf16>(P, F, ends); }

}  // namespace mg3m
