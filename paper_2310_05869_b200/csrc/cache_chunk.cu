// Attention of several new tokens a request over the paged 4-bit cache, and the weight that cached tokens get from them.
// Simple forms: a warp takes a query row and head (attention), or a token and key head (weights), a token of the other side at a time.
#include "serving.cuh"
#include "tc_util.cuh"

namespace hyperattn {
namespace {

struct ChunkArgs {
  CacheView cache;
  const void* q;
  long long q_row, q_head;
  void* out;
  const float* lse_in;
  float* lse;
  const float* weights;
  float* weights_out;
  const int32_t *table, *lengths, *cu_q;
  int requests, rows, width, q_heads, causal, out_kind;
  float scale_log2, decay;
};
struct Span { int first, rows, len; };   // a request's query rows and tokens
__device__ __forceinline__ Span span_of(const ChunkArgs& a, int r) {
  Span s;
  s.first = a.cu_q ? min(max(a.cu_q[r], 0), a.rows) : r;
  s.rows = a.cu_q ? min(max(a.cu_q[r + 1], s.first), a.rows) - s.first : 1;
  s.len = min(max(a.lengths[r], 0), a.width * a.cache.page);
  return s;
}
// coordinates lane, lane + 32, ... of K (which = 0) or V (1) of token t
template <int D>
__device__ __forceinline__ void values_of(const uint8_t* block, int t, int which, float (&x)[D / 32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int w = 0; w < D / 32; ++w) {
    const int c = 32 * w + lane;
    uint32_t code;
    if (which == 0) {
      const int ln = t % 8 * 4 + c / 8 % 4, e = c % 8, nib = e % 2 * 4 + e / 2;
      code = block[(D == 128 ? t / 8 * 512 + ln * 16 : ln * 16 + t / 8 * 8) + c / 32 * 4 + nib / 2] >> (nib % 2 * 4) & 15u;
    } else {
      const int u = c / 16;
      code = block[8 * D + u / 4 * 512 + (c % 8 * 4 + t % 8 / 2) * 16 + u % 4 * 4 + t % 2 * 2 + t / 8] >> (c % 16 >= 8 ? 4 : 0) & 15u;
    }
    const __half* at = reinterpret_cast<const __half*>(block + 16 * D + which * 2 * D + (t / 2 * (D / 32) + w) * 8 + t % 2 * 2);
    x[w] = fmaf(__half2float(at[0]), (float)code, __half2float(at[2]));
  }
}
template <int D, class T>
__device__ __forceinline__ void query_of(const ChunkArgs& a, int row, int head, float (&q)[D / 32]) {
#pragma unroll
  for (int w = 0; w < D / 32; ++w) q[w] = (float)(reinterpret_cast<const T*>(a.q) + (long long)row * a.q_row + (long long)head * a.q_head)[32 * w + (threadIdx.x & 31)];
}
template <int N>
__device__ __forceinline__ float dot(const float (&x)[N], const float (&y)[N]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s = fmaf(x[i], y[i], s);
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

template <int D, class T>
__global__ void __launch_bounds__(128) chunk_kernel(const __grid_constant__ ChunkArgs a) {
  wait_for_stream();
  const long long u = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int row = (int)(u / a.q_heads), head = (int)(u % a.q_heads), lane = threadIdx.x & 31, kv = head / (a.q_heads / a.cache.heads);
  if (row >= a.rows) return;
  int r = 0;
  Span s = {};
  for (; r < a.requests; ++r) { s = span_of(a, r); if (row >= s.first && row < s.first + s.rows) break; }
  if (r == a.requests) return;
  const int seen = a.causal ? min(s.len, s.len - s.rows + row - s.first + 1) : s.len;
  float q[D / 32], o[D / 32] = {}, ref = -INFINITY, sum = 0.f;
  query_of<D, T>(a, row, head, q);
  for (int t = 0; t < seen; ++t) {
    const int page = a.table[(size_t)r * a.width + t / a.cache.page];
    if (page < 0 || page >= a.cache.num_pages) continue;
    const uint8_t* block = block_at<D>(a.cache, page, kv, t % a.cache.page / kBlockTokens);
    float k[D / 32], v[D / 32];
    values_of<D>(block, t % kBlockTokens, 0, k);
    values_of<D>(block, t % kBlockTokens, 1, v);
    const float x = dot(q, k) * a.scale_log2;
    if (!(x <= ref)) {
      const float f = x == x ? exp2f(ref - x) : NAN;
      sum *= f;
#pragma unroll
      for (int w = 0; w < D / 32; ++w) o[w] *= f;
      ref = x;
    }
    const float p = x == -INFINITY && ref == -INFINITY ? 0.f : exp2f(x - ref);
    sum += p;
#pragma unroll
    for (int w = 0; w < D / 32; ++w) o[w] = fmaf(p, v[w], o[w]);
  }
  const size_t at = (size_t)row * a.q_heads + head;
#pragma unroll
  for (int w = 0; w < D / 32; ++w) {
    const float x = sum == 0.f ? 0.f : o[w] / sum;
    const size_t i = at * D + 32 * w + lane;
    if (a.out_kind == HYPERATTN_FP32) reinterpret_cast<float*>(a.out)[i] = x; else reinterpret_cast<T*>(a.out)[i] = static_cast<T>(x);
  }
  if (lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
}

template <class P>
int check(const P* p) {
  int rc;
  if (!p || p->requests < 0 || p->rows < 0 || p->table_width <= 0 || p->q_heads <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_cache(p->cache, &rc)) return rc;
  if (p->dtype != HYPERATTN_BF16 && p->dtype != HYPERATTN_FP16) return p->dtype == HYPERATTN_FP32 ? HYPERATTN_UNSUPPORTED_SHAPE : HYPERATTN_INVALID_ARGUMENT;
  if (p->q_heads % p->cache.kv_heads || bad_stride(p->q_row_stride) || bad_stride(p->q_head_stride) || p->requests > HYPERATTN_PLAN_MAX_REQUESTS) return HYPERATTN_UNSUPPORTED_SHAPE;
  if ((long long)p->table_width * p->cache.page_tokens > 0x7fffffffLL || (long long)p->rows * p->q_heads > 0x7fffffffLL ||
      (long long)p->cache.num_pages * (p->cache.page_tokens / kBlockTokens) * p->cache.kv_heads > 0x7fffffffLL)
    return HYPERATTN_UNSUPPORTED_SHAPE;
  return HYPERATTN_OK;
}
template <class P>
ChunkArgs args_of(const P& p) {
  ChunkArgs a = {};
  a.cache = view_of(p.cache);
  a.q = p.q; a.q_row = p.q_row_stride; a.q_head = p.q_head_stride;
  a.table = p.table; a.lengths = p.lengths; a.cu_q = p.cu_q;
  a.requests = p.requests; a.rows = p.rows; a.width = p.table_width; a.q_heads = p.q_heads; a.causal = p.causal != 0;
  a.scale_log2 = (p.softmax_scale > 0.f ? p.softmax_scale : 1.f / sqrtf((float)p.cache.d)) * 1.4426950408889634f;
  return a;
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_cache_chunk_attention_workspace_bytes(const hyperattn_chunk_params* p, size_t* bytes) {
  if (!bytes) return HYPERATTN_INVALID_ARGUMENT;
  if (int rc = check(p)) return rc;
  *bytes = 0;
  return HYPERATTN_OK;
}

extern "C" int hyperattn_cache_chunk_attention(const hyperattn_chunk_params* p) {
  if (int rc = check(p)) return rc;
  if (p->out_dtype != p->dtype && p->out_dtype != HYPERATTN_FP32) return HYPERATTN_INVALID_ARGUMENT;
  if (!p->cu_q && p->rows != p->requests) return HYPERATTN_INVALID_ARGUMENT;
  if (p->requests == 0 || p->rows == 0) return HYPERATTN_OK;
  if (!p->q || !p->out || !p->lse || !p->table || !p->lengths) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->q) || misaligned(p->out)) return HYPERATTN_MISALIGNED;
  ChunkArgs a = args_of(*p);
  a.out = p->out; a.lse = p->lse; a.out_kind = p->out_dtype;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  const dim3 grid((unsigned)(((long long)p->rows * p->q_heads + 3) / 4)), block(128);
  const bool bf16 = p->dtype == HYPERATTN_BF16;
  if (p->cache.d == 64) return status_of(bf16 ? launch(chunk_kernel<64, __nv_bfloat16>, grid, block, 0, st, a) : launch(chunk_kernel<64, __half>, grid, block, 0, st, a), "chunk attention");
  return status_of(bf16 ? launch(chunk_kernel<128, __nv_bfloat16>, grid, block, 0, st, a) : launch(chunk_kernel<128, __half>, grid, block, 0, st, a), "chunk attention");
}
