#include "attention_forward.h"

template sp_status attn_forward<attn_f16>(const sp_attn_plan *, forward_args &, const forward_choice &, hipStream_t);
