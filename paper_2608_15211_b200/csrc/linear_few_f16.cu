// The product for a few rows for fp16 activations: the same source, compiled with the fp16 element operations.
#define TERRA_ELEM_F16 1
#include "linear_few.cu"
