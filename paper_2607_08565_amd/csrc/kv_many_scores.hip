// The kernels of kv_many.hip with scores that are capped or have a bias by distance, compiled apart.
#define SCORED
#include "kv_many.hip"
