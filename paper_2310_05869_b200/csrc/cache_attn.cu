// Attention of one query token a request over the paged 4-bit cache: the launches (the kernels are in cache_attn.cuh).
#include "cache_attn.cuh"

namespace hyperattn {
namespace {

// What a call's launches look like: heads of a chunk, CTAs, bytes of the workspace (which follow from the call's arguments alone)
struct Shape { bool two; int chunks, part_heads, ctas; size_t starts, bytes; };
Shape shape_of(const hyperattn_cache_attention_params& p) {
  Shape s;
  const int per_kv = p.q_heads / p.cache.kv_heads, d = p.cache.d;
  s.two = per_kv > 8;
  s.chunks = (per_kv + (s.two ? 15 : 7)) / (s.two ? 16 : 8);
  s.part_heads = s.two ? 16 : 8;
  if (s.part_heads > per_kv) s.part_heads = per_kv;
  const int unit = d == 64 ? Ring<64, kOneQuery>::kUnitTokens : Ring<128, kOneQuery>::kUnitTokens;
  const long long units = (long long)p.requests * p.cache.kv_heads * s.chunks * (((long long)p.table_width * p.cache.page_tokens + unit - 1) / unit);
  const long long ctas = (units + kWarps - 1) / kWarps;
  const int memory = d == 64 ? ctas_by_memory<64, kOneQuery>(p.requests) : ctas_by_memory<128, kOneQuery>(p.requests), registers = ctas_by_registers(s.two ? 2 : 1);
  const int most = kSms * (memory < registers ? memory : registers);
  s.ctas = (int)(ctas < most ? ctas : most);
  s.starts = ((size_t)(p.requests + 2) * 4 + 255) / 256 * 256;
  s.bytes = s.starts + (size_t)s.ctas * kWarps * 2 * s.part_heads * (d + 2) * 4;
  return s;
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

namespace {
int check(const hyperattn_cache_attention_params* p) {
  int rc;
  if (!p || p->requests < 0 || p->table_width <= 0 || p->q_heads <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_cache(p->cache, &rc)) return rc;
  if (p->dtype != HYPERATTN_BF16 && p->dtype != HYPERATTN_FP16) return p->dtype == HYPERATTN_FP32 ? HYPERATTN_UNSUPPORTED_SHAPE : HYPERATTN_INVALID_ARGUMENT;
  if (p->out_dtype != p->dtype && p->out_dtype != HYPERATTN_FP32) return HYPERATTN_INVALID_ARGUMENT;
  if (p->q_heads % p->cache.kv_heads || bad_stride(p->q_row_stride) || bad_stride(p->q_head_stride) || p->requests > kMaxRequests) return HYPERATTN_UNSUPPORTED_SHAPE;
  if ((long long)p->table_width * p->cache.page_tokens > 0x7fffffffLL || (long long)p->requests * p->q_heads * ((long long)p->table_width * p->cache.page_tokens / 32 + 1) > 0x7fffffffLL ||
      (long long)p->requests * p->q_heads > 0x7fffffffLL || (long long)p->cache.num_pages * (p->cache.page_tokens / kBlockTokens) * p->cache.kv_heads > 0x7fffffffLL)
    return HYPERATTN_UNSUPPORTED_SHAPE;
  return HYPERATTN_OK;
}
}  // namespace

extern "C" int hyperattn_cache_attention_workspace_bytes(const hyperattn_cache_attention_params* p, size_t* bytes) {
  if (!bytes) return HYPERATTN_INVALID_ARGUMENT;
  if (int rc = check(p)) return rc;
  *bytes = p->requests ? shape_of(*p).bytes : 0;
  return HYPERATTN_OK;
}

extern "C" int hyperattn_cache_attention(const hyperattn_cache_attention_params* p) {
  if (int rc = check(p)) return rc;
  if (p->requests == 0) return HYPERATTN_OK;
  if (!p->q || !p->out || !p->lse || !p->table || !p->lengths || !p->workspace) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->q) || misaligned(p->out) || misaligned(p->workspace)) return HYPERATTN_MISALIGNED;
  const Shape s = shape_of(*p);
  if (p->workspace_bytes < s.bytes) return HYPERATTN_WORKSPACE_TOO_SMALL;
  KernelArgs<kOneQuery> a = {};
  a.cache = {reinterpret_cast<uint8_t*>(p->cache.pages), p->cache.num_pages, p->cache.page_tokens, p->cache.kv_heads};
  a.q = p->q; a.q_row = p->q_row_stride; a.q_head = p->q_head_stride;
  a.out = p->out; a.lse = p->lse; a.table = p->table; a.lengths = p->lengths;
  a.requests = p->requests; a.width = p->table_width; a.q_heads = p->q_heads; a.out_kind = p->out_dtype; a.chunks = s.chunks;
  const int d = p->cache.d;
  a.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.f / sqrtf((float)d)) * 1.4426950408889634f;
  a.starts = reinterpret_cast<int*>(p->workspace);
  a.part = reinterpret_cast<float*>(reinterpret_cast<char*>(p->workspace) + s.starts);
  a.part_heads = s.part_heads;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  int* status = nullptr;
  if (int rc = device_status_word(st, &status)) return rc;
  const int segments = p->requests * p->cache.kv_heads * s.chunks;
  auto go = [&](auto dim, auto kernel) {
    constexpr int D = decltype(dim)::value;
    cudaError_t e = launch(kernel, dim3((unsigned)s.ctas), dim3(32 * kWarps), Ring<D, kOneQuery>::bytes(p->requests), st, a, status);
    // few segments: a CTA for a head or some
    int split = (4 * kSms + segments - 1) / segments;
    if (split > s.part_heads) split = s.part_heads;
    const int heads = (s.part_heads + split - 1) / split;
    if (e == cudaSuccess) e = launch(join_kernel<D, kOneQuery>, dim3((unsigned)segments, (unsigned)((s.part_heads + heads - 1) / heads)), dim3(kJoinThreads), 0, st, a, heads);
    if (e == cudaSuccess) return (int)HYPERATTN_OK;
    std::fprintf(stderr, "hyperattn: cache attention failed: %s\n", cudaGetErrorString(e));
    return (int)HYPERATTN_CUDA_ERROR;
  };
  auto build = [&](auto dim, auto tiles, auto type) {
    constexpr int D = decltype(dim)::value, NT = decltype(tiles)::value > 1 ? 2 : 1;
    constexpr bool PAIR = decltype(tiles)::value == 0;
    using T = decltype(type);
    if (allow_smem<cache_attn_kernel<D, NT, PAIR, T, kOneQuery>>(Ring<D, kOneQuery>::bytes(kMaxRequests)) != cudaSuccess) return (int)HYPERATTN_CUDA_ERROR;
    return go(dim, cache_attn_kernel<D, NT, PAIR, T, kOneQuery>);
  };
  auto of_type = [&](auto dim, auto tiles) { return p->dtype == HYPERATTN_BF16 ? build(dim, tiles, __nv_bfloat16()) : build(dim, tiles, __half()); };
  // (four heads or fewer: both halves of a tile, see add_values)
  auto of_tiles = [&](auto dim) { return s.part_heads <= 4 ? of_type(dim, std::integral_constant<int, 0>{}) : s.two ? of_type(dim, std::integral_constant<int, 2>{}) : of_type(dim, std::integral_constant<int, 1>{}); };
  return d == 64 ? of_tiles(std::integral_constant<int, 64>{}) : of_tiles(std::integral_constant<int, 128>{});
}
