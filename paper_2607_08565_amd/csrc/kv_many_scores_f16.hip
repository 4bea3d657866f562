// Capped and biased scores' kernels of F16, compiled beside the plain ones.
#define SCORED F16
#include "kv_many.hip"
