// Linear layers of fp32 numbers.
#include "pcsr_linear_kernels.h"

template struct pcsr::LinearOf<float>;
