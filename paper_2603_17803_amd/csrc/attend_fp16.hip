// Attention of drafted tokens over a paged cache: the kernels for fp16 (attend_core.h).
#include "attend_core.h"

void launch_attend_fp16(const attend_args& a, hipStream_t stream) { launch_attend_type<false>(a, stream); }
