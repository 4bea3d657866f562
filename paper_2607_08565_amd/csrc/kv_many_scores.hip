// Capped and biased scores' kernels of BF16, compiled beside the plain ones.
#define SCORED Bf16
#include "kv_many.hip"
