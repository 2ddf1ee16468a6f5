#include "attention_backward.h"

template sp_status attn_backward<attn_f16>(const sp_tensor *, grad_args &, const grad_choice &, hipStream_t);
