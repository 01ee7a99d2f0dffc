// The launches of the kernels for few rows a request (cache_rows.cu), as the entry points use them.
#pragma once
#include "../../include/hyperattn.h"

namespace hyperattn {

// whether these kernels take the call, and their workspace
bool few_rows_attention(const hyperattn_chunk_params& p, size_t* bytes);
int launch_few_rows_attention(const hyperattn_chunk_params& p, int* status);
bool few_rows_weights(const hyperattn_weights_params& p);
int launch_few_rows_weights(const hyperattn_weights_params& p, int* status);

}  // namespace hyperattn
