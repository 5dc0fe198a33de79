// The kernels of rel_attention_mfma.h for fp32 storage.
#include "rel_attention_mfma.h"

template int rel_mfma_fwd<float>(const RelArgs&, const float*, float*, float*, hipStream_t);
template int rel_mfma_bwd<float>(const RelArgs&, const float*, const float*, const float*, const float*, float*, float*, float*, int, bool*, hipStream_t);
