// The launches of the kernels for few rows a request (cache_rows.cu), as the entry points use them.
#pragma once
#include "../../include/hyperattn.h"

namespace hyperattn {

// whether these kernels take the call, and their workspace
bool few_rows_attention(const hyperattn_chunk_params& p, size_t* bytes);
int launch_few_rows_attention(const hyperattn_chunk_params& p, int* status);
bool few_rows_weights(const hyperattn_weights_params& p);
int launch_few_rows_weights(const hyperattn_weights_params& p, int* status);
int few_rows_unit(int d);                // tokens that it takes at a time: what is beyond a request's last ones it does not write

}  // namespace hyperattn
