// Linear layers of fp16 numbers.
#include "pcsr_linear_kernels.h"

template struct pcsr::LinearOf<pcsr::half_t>;
