// The kernels of rel_attention_mfma.h for bf16 storage.
#include "rel_attention_mfma.h"

template int rel_mfma_fwd<bf16_t>(const RelArgs&, const bf16_t*, bf16_t*, float*, hipStream_t);
template int rel_mfma_bwd<bf16_t>(const RelArgs&, const bf16_t*, const bf16_t*, const bf16_t*, const float*, bf16_t*, float*, float*, int, bool*, hipStream_t);
