// Linear layers of bf16 numbers.
#include "pcsr_linear_kernels.h"

template struct pcsr::LinearOf<pcsr::bfloat_t>;
