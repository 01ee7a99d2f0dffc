// Exact attention over packed prompts with grouped heads.
#include <cstdio>
#include "serving.cuh"

namespace hyperattn {
namespace {

struct PromptArgs {
  const void *q, *k, *v;
  long long q_row, q_head, k_row, k_head, v_row, v_head;
  void* out;
  float* lse;
  const int32_t *cu_q, *cu_k;
  int requests, q_rows, k_rows, q_heads, kv_heads, causal, out_kind;
  float scale_log2;
};

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A warp and one query row of one head: a lane has D / 32 coordinates, the keys follow each other.
template <int D, class T>
__device__ __forceinline__ void attend_row(const PromptArgs& a, int row, int head, int key0, int keys) {
  constexpr int E = D / 32;                                // coordinates of a lane
  const int lane = threadIdx.x & 31, kv = head / (a.q_heads / a.kv_heads);
  auto load = [&](const void* base, size_t at, float (&x)[E]) {
    const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const T*>(base) + at) + lane * (E / 2);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) { const float2 f = to_float2<T>(src[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
  };
  float q[E], o[E], ref = -INFINITY, sum = 0.f;
  load(a.q, (size_t)row * a.q_row + (size_t)head * a.q_head, q);
#pragma unroll
  for (int i = 0; i < E; ++i) o[i] = 0.f;
  for (int j = 0; j < keys; ++j) {
    float k[E], v[E], s = 0.f;
    load(a.k, (size_t)(key0 + j) * a.k_row + (size_t)kv * a.k_head, k);
    load(a.v, (size_t)(key0 + j) * a.v_row + (size_t)kv * a.v_head, v);
#pragma unroll
    for (int i = 0; i < E; ++i) s = fmaf(q[i], k[i], s);
#pragma unroll
    for (int w = 16; w; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
    s *= a.scale_log2;
    if (s > ref) {
      const float f = ex2f(ref - s);
      sum *= f; ref = s;
#pragma unroll
      for (int i = 0; i < E; ++i) o[i] *= f;
    }
    const float p = ex2f(s - (ref == -INFINITY ? 0.f : ref));
    sum += p;
#pragma unroll
    for (int i = 0; i < E; ++i) o[i] = fmaf(p, v[i], o[i]);
  }
  const size_t at = (size_t)row * a.q_heads + head;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float x = sum == 0.f ? 0.f : o[i] / sum;
    const size_t e = at * D + lane * E + i;
    if (a.out_kind == HYPERATTN_FP32) reinterpret_cast<float*>(a.out)[e] = x;
    else if (a.out_kind == HYPERATTN_BF16) reinterpret_cast<__nv_bfloat16*>(a.out)[e] = __float2bfloat16_rn(x);
    else reinterpret_cast<__half*>(a.out)[e] = __float2half_rn(x);
  }
  if (lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
}

template <int D, class T>
__global__ void __launch_bounds__(256) prompt_rows_kernel(PromptArgs a) {
  wait_for_stream();
  const int head = threadIdx.x / 32 + 8 * blockIdx.y, row = blockIdx.x;
  const int r = upper_bound(a.cu_q + 1, a.requests, row);
  if (head >= a.q_heads || r >= a.requests) return;
  const int nq = a.cu_q[r + 1] - a.cu_q[r], nk = a.cu_k[r + 1] - a.cu_k[r];
  attend_row<D, T>(a, row, head, a.cu_k[r], a.causal ? max(0, nk - (nq - 1 - (row - a.cu_q[r]))) : nk);
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_prompt_attention(const hyperattn_prompt_params* p) {
  if (!p || p->requests < 0 || p->q_rows < 0 || p->k_rows < 0 || p->q_heads <= 0 || p->kv_heads <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (p->dtype != HYPERATTN_BF16 && p->dtype != HYPERATTN_FP16) return p->dtype == HYPERATTN_FP32 ? HYPERATTN_UNSUPPORTED_SHAPE : HYPERATTN_INVALID_ARGUMENT;
  if (p->out_dtype != p->dtype && p->out_dtype != HYPERATTN_FP32) return HYPERATTN_INVALID_ARGUMENT;
  if ((p->d != 64 && p->d != 128) || p->q_heads % p->kv_heads || p->q_heads / p->kv_heads > 128) return HYPERATTN_UNSUPPORTED_SHAPE;
  for (long long s : {p->q_row_stride, p->q_head_stride, p->k_row_stride, p->k_head_stride, p->v_row_stride, p->v_head_stride})
    if (bad_stride(s)) return HYPERATTN_UNSUPPORTED_SHAPE;
  if (p->requests == 0 || p->q_rows == 0) return HYPERATTN_OK;
  if (!p->q || (p->k_rows && (!p->k || !p->v)) || !p->out || !p->lse || !p->cu_q || !p->cu_k) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->q) || misaligned(p->k) || misaligned(p->v) || misaligned(p->out)) return HYPERATTN_MISALIGNED;
  if (p->out == p->q || p->out == p->k || p->out == p->v) return HYPERATTN_MISALIGNED;
  PromptArgs a;
  a.q = p->q; a.k = p->k; a.v = p->v;
  a.q_row = p->q_row_stride; a.q_head = p->q_head_stride; a.k_row = p->k_row_stride; a.k_head = p->k_head_stride; a.v_row = p->v_row_stride; a.v_head = p->v_head_stride;
  a.out = p->out; a.lse = p->lse; a.cu_q = p->cu_q; a.cu_k = p->cu_k;
  a.requests = p->requests; a.q_rows = p->q_rows; a.k_rows = p->k_rows; a.q_heads = p->q_heads; a.kv_heads = p->kv_heads;
  a.causal = p->causal != 0; a.out_kind = p->out_dtype;
  a.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.f / sqrtf((float)p->d)) * 1.4426950408889634f;
  const dim3 grid((unsigned)p->q_rows, (unsigned)((p->q_heads + 7) / 8));
  if (grid.y > 65535) return HYPERATTN_UNSUPPORTED_SHAPE;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  auto go = [&](auto kernel) {
    const cudaError_t e = launch(kernel, grid, dim3(256), 0, st, a);
    if (e == cudaSuccess) return (int)HYPERATTN_OK;
    std::fprintf(stderr, "hyperattn: prompt attention failed: %s\n", cudaGetErrorString(e));
    return (int)HYPERATTN_CUDA_ERROR;
  };
  const bool bf16 = p->dtype == HYPERATTN_BF16;
  if (p->d == 64) return bf16 ? go(prompt_rows_kernel<64, __nv_bfloat16>) : go(prompt_rows_kernel<64, __half>);
  return bf16 ? go(prompt_rows_kernel<128, __nv_bfloat16>) : go(prompt_rows_kernel<128, __half>);
}
