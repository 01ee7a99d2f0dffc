// The launches of the kernels for few rows a request (cache_rows.cu), as the entry points use them.
#pragma once
#include "../../include/hyperattn.h"

namespace hyperattn {

// whether these kernels can take the call, and their workspace; most: requests with more rows are left out
bool few_rows_attention(const hyperattn_chunk_params& p, size_t* bytes);
int launch_few_rows_attention(const hyperattn_chunk_params& p, int most, int* status);
bool few_rows_weights(const hyperattn_weights_params& p);
int launch_few_rows_weights(const hyperattn_weights_params& p, int most, int* status);

// Which kernels a call needs: these for requests of up to `most` rows, the tcgen05 ones for those with more.  The host knows the average alone.  If that is not more, these take the
// whole call; but one request may have nearly all of its rows (every other one has one at least, it is assumed): a part of a prompt beside single tokens.  Where that could be more than 256
// rows, both run, each for the requests that suit it; likewise where the average is more and there are 16 requests and more, which are then hardly all large.  us, 512 rows
// and 63 single tokens, 8000 tokens each, 32 heads of 64: attention 696 (these alone) -> 422, weights 6820 -> 347; 32 / 8 heads of 128: 622 (the others alone) -> 304, 490 -> 206.  What it costs where no
// request has many rows: 64 requests of 4 tokens, 32 / 8 heads of 128, over 8000 tokens: 297 -> 310, 111 -> 126.
struct Kinds { bool few, many; };
// Rows of a request up to which these kernels are the faster ones.  Attention, us here / there, up to 8000 tokens, 8 requests: 8 heads of 128, 32 rows 60 / 79, 48 rows 94 / 91, 64 rows 106 / 74; 32 heads
// of 64, 32 rows 129 / 161, 48 rows 157 / 157, 64 rows 173 / 143.  Tables of no more than 1024 tokens (there the first and the last launch take as long as the work), 64 rows: 21 / 25.
inline int most_of(const hyperattn_chunk_params& p) { return (long long)p.table_width * p.cache.page_tokens <= 1024 ? 64 : 32; }
inline int most_of(const hyperattn_weights_params&) { return 16; }
template <class P>
Kinds kinds_of(const P& p, int most) {
  const long long group = p.q_heads / p.cache.kv_heads, all = p.rows * group, largest = all - (p.requests - 1) * group;
  const bool average = all <= (long long)most * p.requests;
  return {average || (largest > 256 && p.requests >= 16), !average || largest > 256};
}

}  // namespace hyperattn
