// The kernels of attention over the 4-bit cache for f32.
#include "cache_attention.h"
CACHE_ATTENTION_OF(float)
