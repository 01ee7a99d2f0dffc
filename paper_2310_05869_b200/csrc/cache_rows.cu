// Few rows a request over the paged 4-bit cache - drafted tokens, single tokens - and the weight that cached tokens get from them: the launches of the warp-level kernels
// (cache_attn.cuh) with some rows in the place of a key head's query heads.
#include "cache_attn.cuh"
#include "cache_rows.cuh"
#include "cache_tiles.cuh"

namespace hyperattn {

namespace {

// What a call's launches look like: rows of a chunk (0: four, twice in a tile), CTAs, bytes of the workspace
struct RowsShape { int tiles, per_chunk, ctas; long long slots; size_t starts, bytes; };
template <int D, Mode MODE>
RowsShape rows_shape(int requests, int rows, int group, int kv_heads, long long tokens, bool both) {
  RowsShape s;
  const long long all = (long long)rows * group;
  // Rows in a tile: attention four (and what the rounding of their weights loses beside them) where requests have that many on average, two tiles of eight where they have more than eight
  // and d = 64, else eight.  us for four / eight / sixteen: 16 rows over 4000 tokens, 8 heads of 128, 8 requests 51 / 43 / 47, 32 rows 91 / 65 / 72; 2 x 30000 tokens, 32 heads of 64,
  // 16 rows 309 / 190 / 184, 32 rows 556 / 316 / 288; weights of 16 rows over 300 tokens - / 10.8 / 9.4.
  // (Both kinds of kernels: the average is not these requests', whose tokens may be single ones.  Weights have two tiles all the same: requests of more rows than a tile's load their queries anew for
  // every unit, 16 rows 242 us instead of 127.)
  s.tiles = MODE == kSomeRows && all <= 4ll * requests ? 0 : all <= 8ll * requests || (MODE == kSomeRows && (both || D == 128)) ? 1 : 2;
  s.per_chunk = s.tiles == 0 ? 4 : 8 * s.tiles;
  s.slots = chunk_slots(rows, requests, group, s.per_chunk) + 1;
  constexpr int unit = Ring<D, MODE>::kUnitTokens;
  const long long units = (MODE == kWeights ? requests : s.slots) * kv_heads * ((tokens + unit - 1) / unit), ctas = (units + kWarps - 1) / kWarps;
  const int memory = ctas_by_memory<D, MODE>(requests), registers = ctas_by_registers(s.tiles == 2 ? 2 : 1);
  const int most = kSms * (memory < registers ? memory : registers);
  s.ctas = (int)(ctas < most ? ctas : most);
  s.starts = ((size_t)(requests + 2) * 4 + 255) / 256 * 256;
  s.bytes = MODE == kWeights ? 0 : s.starts + (size_t)s.ctas * kWarps * 2 * s.per_chunk * (D + 2) * 4;
  return s;
}
// units are counted in ints
template <int D, Mode MODE>
bool countable(const RowsShape& s, int requests, int kv_heads, long long tokens) {
  return (MODE == kWeights ? (long long)requests : s.slots) * kv_heads <= 0x7fffffffLL / (tokens / Ring<D, MODE>::kUnitTokens + 2 + kBegin) && s.slots * kv_heads <= 0x7fffffffLL;
}
template <Mode MODE>
KernelArgs<MODE> rows_args(const ChunkArgs& c, int most) {
  KernelArgs<MODE> a = {};
  a.cache = c.cache; a.q = c.q; a.q_row = c.q_row; a.q_head = c.q_head; a.table = c.table; a.lengths = c.lengths; a.cu_q = c.cu_q;
  a.requests = c.requests; a.width = c.width; a.q_heads = c.q_heads; a.rows = c.rows; a.causal = c.causal; a.most = most; a.scale_log2 = c.scale_log2; a.chunks = 1;
  return a;
}
template <class F>
auto of_dim(int d, F f) { return d == 64 ? f(std::integral_constant<int, 64>{}) : f(std::integral_constant<int, 128>{}); }

}  // namespace

bool few_rows_attention(const hyperattn_chunk_params& p, bool both, size_t* bytes) {
  const int group = p.q_heads / p.cache.kv_heads;
  const long long tokens = (long long)p.table_width * p.cache.page_tokens;
  return of_dim(p.cache.d, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    const RowsShape s = rows_shape<D, kSomeRows>(p.requests, p.rows, group, p.cache.kv_heads, tokens, both);
    *bytes = s.bytes;
    return countable<D, kSomeRows>(s, p.requests, p.cache.kv_heads, tokens);
  });
}

int launch_few_rows_attention(const hyperattn_chunk_params& p, bool both, int* status) {
  const int group = p.q_heads / p.cache.kv_heads;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p.stream);
  KernelArgs<kSomeRows> a = rows_args<kSomeRows>(chunk_args(p), both ? most_of(p) : INT_MAX);
  a.out = p.out; a.lse = p.lse; a.out_kind = p.out_dtype;
  return of_dim(p.cache.d, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    using R = Ring<D, kSomeRows>;
    const RowsShape s = rows_shape<D, kSomeRows>(p.requests, p.rows, group, p.cache.kv_heads, (long long)p.table_width * p.cache.page_tokens, both);
    a.starts = reinterpret_cast<int*>(p.workspace);
    a.part = reinterpret_cast<float*>(reinterpret_cast<char*>(p.workspace) + s.starts);
    a.part_heads = s.per_chunk;
    auto go = [&](auto tiles, auto type, auto fine) {
      constexpr int NT = decltype(tiles)::value > 1 ? 2 : 1;
      constexpr bool PAIR = decltype(tiles)::value == 0;
      constexpr auto kernel = cache_attn_kernel<D, NT, PAIR, decltype(type), kSomeRows, decltype(fine)::value>;
      cudaError_t e = allow_smem<kernel>(R::bytes(kMaxRequests));
      if (e == cudaSuccess) e = launch(kernel, dim3((unsigned)s.ctas), dim3(32 * kWarps), R::bytes(p.requests), st, a, status);
      const long long segments = s.slots * p.cache.kv_heads;
      // few segments: a CTA for a row or some (8 requests of 16 rows, 8 heads: 13 us with two, of 25 in all)
      int split = (int)((16 * kSms + segments - 1) / segments);
      if (split > s.per_chunk) split = s.per_chunk;
      const int heads = (s.per_chunk + split - 1) / split;
      if (e == cudaSuccess) e = launch(join_kernel<D, kSomeRows>, dim3((unsigned)segments, (unsigned)((s.per_chunk + heads - 1) / heads)), dim3(kJoinThreads), 0, st, a, heads);
      return status_of(e, "chunk attention");
    };
    auto of_type = [&](auto tiles) {
      return p.dtype != HYPERATTN_BF16 ? go(tiles, __half(), std::true_type()) : p.out_dtype == HYPERATTN_FP32 ? go(tiles, __nv_bfloat16(), std::true_type()) : go(tiles, __nv_bfloat16(), std::false_type());
    };
    // (d = 128: never two tiles, see rows_shape)
    if constexpr (D == 64)
      if (s.tiles == 2) return of_type(std::integral_constant<int, 2>{});
    return s.tiles == 0 ? of_type(std::integral_constant<int, 0>{}) : of_type(std::integral_constant<int, 1>{});
  });
}

bool few_rows_weights(const hyperattn_weights_params& p, bool both) {
  const int group = p.q_heads / p.cache.kv_heads;
  const long long tokens = (long long)p.table_width * p.cache.page_tokens;
  return of_dim(p.cache.d, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    return countable<D, kWeights>(rows_shape<D, kWeights>(p.requests, p.rows, group, p.cache.kv_heads, tokens, both), p.requests, p.cache.kv_heads, tokens);
  });
}

int launch_few_rows_weights(const hyperattn_weights_params& p, bool both, int* status) {
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p.stream);
  KernelArgs<kWeights> a = rows_args<kWeights>(chunk_args(p), both ? most_of(p) : INT_MAX);
  a.lse_in = p.lse; a.before = p.weights; a.weights = p.weights_out; a.decay = p.decay;
  return of_dim(p.cache.d, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    using R = Ring<D, kWeights>;
    const int subs = p.cache.page_tokens / kBlockTokens;
    a.run = subs % R::kUnit == 0 ? R::kUnit : subs & -subs;
    const long long blocks = (long long)p.cache.num_pages * p.cache.kv_heads * subs;
    if (!encode_words_map(&a.maps.codes, p.cache.pages, blocks, 5 * D, 2 * D, a.run) || !encode_words_map(&a.maps.scales, p.cache.pages, blocks, 5 * D, D / 2, a.run)) return (int)HYPERATTN_UNSUPPORTED_SHAPE;
    const RowsShape s = rows_shape<D, kWeights>(p.requests, p.rows, p.q_heads / p.cache.kv_heads, p.cache.kv_heads, (long long)p.table_width * p.cache.page_tokens, both);
    auto go = [&](auto tiles, auto type) {
      constexpr auto kernel = cache_attn_kernel<D, decltype(tiles)::value, false, decltype(type), kWeights>;
      cudaError_t e = allow_smem<kernel>(R::bytes(kMaxRequests));
      if (e == cudaSuccess) e = launch(kernel, dim3((unsigned)s.ctas), dim3(32 * kWarps), R::bytes(p.requests), st, a, status);
      return status_of(e, "cache weights");
    };
    auto of_type = [&](auto tiles) { return p.dtype == HYPERATTN_BF16 ? go(tiles, __nv_bfloat16()) : go(tiles, __half()); };
    return s.tiles == 1 ? of_type(std::integral_constant<int, 1>{}) : of_type(std::integral_constant<int, 2>{});
  });
}

}  // namespace hyperattn
