// The launches of the kernels for few rows a request (cache_rows.cu), as the entry points use them.
#pragma once
#include "../../include/hyperattn.h"

namespace hyperattn {

// whether these kernels can take the call, and their workspace; both: the tcgen05 ones take the requests with more rows than most_of()
bool few_rows_attention(const hyperattn_chunk_params& p, bool both, size_t* bytes);
int launch_few_rows_attention(const hyperattn_chunk_params& p, bool both, int* status);
bool few_rows_weights(const hyperattn_weights_params& p, bool both);
int launch_few_rows_weights(const hyperattn_weights_params& p, bool both, int* status);

// Which kernels a call needs: these for requests of up to `most` rows, the tcgen05 ones for those with more.  The host knows the average alone, and, if the caller says so, the most new tokens that a
// request has.
//   The average is not more than `most`: these, and if a request could have more than 256 rows, both, each for the requests that suit it - all rows may be those of one request, a part of a prompt beside
// places without a request, or single tokens.  us, attention / weights: 64 places, one part of 300 tokens over 8000, 32 heads of 64: 199 / 140 with these alone, 97 / 76 with both; 128 tokens, 32 / 8 heads
// of 128: 158 / 197, 86 / 48.  512 rows and 63 single tokens, 8000 tokens each, 32 heads of 64: 696 / 6820, 422 / 347.  What it costs where no request has many rows, and nobody says so: 128 single
// tokens over up to 4000, 32 / 8 heads of 128, 146 / 50 -> 160 / 62.
//   The average is more: the tcgen05 ones, and if the other requests could have as much in the cache as makes up for the launches, both.  One part of 300 tokens and single tokens over 8000 each, 32 heads
// of 64: 4 requests 139 / 122 -> 113 / 78, 8 222 / 210 -> 133 / 104; 32 / 8 heads of 128: 4 requests 115 / 81 -> 128 / 74, 8 145 / 107 -> 142 / 82, 15 206 / 147 -> 156 / 99; one part of 1024 tokens, single ones
// over 100000: 2 requests 310 / 230 -> 285 / 179, 8 833 / 709 -> 412 / 291.  Where all have many rows it costs 6 to 9.
struct Kinds { bool few, many; };
// Rows of a request up to which these kernels are the faster ones.  Attention, us here / there, up to 8000 tokens, 8 requests: 8 heads of 128, 32 rows 60 / 79, 48 rows 94 / 91, 64 rows 106 / 74; 32 heads
// of 64, 32 rows 129 / 161, 48 rows 157 / 157, 64 rows 173 / 143.  Tables of no more than 1024 tokens (there the first and the last launch take as long as the work), 64 rows: 21 / 25.
inline int most_of(const hyperattn_chunk_params& p) { return (long long)p.table_width * p.cache.page_tokens <= 1024 ? 64 : 32; }
inline int most_of(const hyperattn_weights_params&) { return 16; }
constexpr long long kWorthBoth = 1 << 26;        // numbers of K that the others could have in the cache
// most_new: new tokens that a request has at most (0: not known)
template <class P>
Kinds kinds_of(const P& p, int most_new) {
  const long long group = p.q_heads / p.cache.kv_heads, all = p.rows * group, one = most_new * group;
  if (all <= (long long)most_of(p) * p.requests) return {true, (most_new && one < all ? one : all) > 256};
  return {all > 256 && (double)(p.requests - 1) * p.table_width * p.cache.page_tokens * p.cache.kv_heads * p.cache.d >= (double)kWorthBoth, true};
}

}  // namespace hyperattn
