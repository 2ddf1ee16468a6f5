// The kernels of attention over the 4-bit cache for bf16.
#include "cache_attention.h"
CACHE_ATTENTION_OF(cache_bf16)
