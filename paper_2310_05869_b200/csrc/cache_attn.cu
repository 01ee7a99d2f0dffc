// Attention of one query token a request over the paged 4-bit cache.
//
// A warp takes a block of 16 tokens of one key head and up to 16 query heads that read it, on the warp-level tensor cores
// (mma.sync m16n8k16, fp16 operands, fp32 sums):
//   S = Q K^T   the codes of K become 64 + c in fp16 by one logical operation for two of them; the sums start at -64 sum(q), so that
//               sum(q c) is left, and a group's scale and minimum enter in fp32:  s = sum_g scale_g sum(q c) + min_g sum_g(q)
//   p = exp2(s c - ref), the reference of a head moves when it is exceeded by more than 2^8
//   O^T += V^T P^T   V = min + scale * code in fp16 (exact codes, one rounding); its 32-bit words hold four tokens of two coordinates,
//               so that masking yields operands with pairs of tokens, and P^T is what the lanes have after S.
// fp16 and not bf16 for the weights and values: a product is then off by 2^-11 and not 2^-8, which is what the output's type can show; V fits by
// its format, a head's query after a power of two.
#include <cstdio>
#include "serving.cuh"

namespace hyperattn {
namespace {

constexpr float kMoveAt = 8.f;          // octaves the scores of a head may exceed its reference before that moves

struct CacheAttnArgs {
  CacheView cache;
  const void* q;
  long long q_row, q_head;
  void* out;
  float* lse;
  const int32_t *table, *lengths;
  int requests, width, q_heads, out_kind;      // out_kind: hyperattn_dtype
  float scale_log2;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// nibbles 1 and 5 of a word (bits 4..7 of either half) as 64 + code in fp16
__device__ __forceinline__ uint32_t codes_at_4(uint32_t w) { return (w & 0x00f000f0u) | 0x54005400u; }
__device__ __forceinline__ __half2 h2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
__device__ __forceinline__ uint32_t u32(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }

// What a warp keeps of the heads it works for: NT = 1: up to 8 of them (a lane's head: lane / 4), NT = 2: up to 16 (and lane / 4 + 8)
template <int D, int NT>
struct Heads {
  static constexpr int kGroups = D / kGroup;
  uint32_t q[NT][kGroups][4];           // fp16 pairs: coordinates 32 w + 8 c + 0..7
  float qsum[NT][kGroups];              // sums of the group's entries
  float scale[NT];                      // to the base-2 scores
  float ref[NT], sum[NT];               // sum: of this lane's tokens
  float o[NT][D / 16][4];               // O^T: coordinates lane / 4 (+ 8) of every 16, heads 2 c, 2 c + 1 (+ 8)
};

template <int D, int NT, class T>
__device__ __forceinline__ void load_heads(Heads<D, NT>& h, const CacheAttnArgs& a, int request, int first_head, int heads) {
  const int lane = threadIdx.x & 31, c = lane & 3;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int head = lane / 4 + 8 * t;
    float top = 0.f;
    uint4 raw[Heads<D, NT>::kGroups];
#pragma unroll
    for (int w = 0; w < Heads<D, NT>::kGroups; ++w) {
      raw[w] = make_uint4(0, 0, 0, 0);
      if (head < heads)
        raw[w] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.q) + request * a.q_row + (first_head + head) * a.q_head + 32 * w + 8 * c);
      const uint32_t v[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) { const float2 f = to_float2<T>(v[i]); top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y))); }
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 2^-e, e the exponent of the largest entry (0 and what is not finite: as it is)
    int e = (int)(__float_as_uint(top) >> 23) - 127;
    e = top == 0.f || !(top < INFINITY) ? 0 : min(max(e, -126), 126);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
    h.scale[t] = up * a.scale_log2;
#pragma unroll
    for (int w = 0; w < Heads<D, NT>::kGroups; ++w) {
      const uint32_t v[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = to_float2<T>(v[i]);
        h.q[t][w][i] = from_float2<__half>(f.x * down, f.y * down);
        const float2 r = to_float2<__half>(h.q[t][w][i]);
        sum += r.x + r.y;
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      h.qsum[t][w] = sum;
    }
    h.ref[t] = -INFINITY; h.sum[t] = 0.f;
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) h.o[t][m][i] = 0.f;
  }
}

// The references move to the scores' maximum where they are exceeded; sums and outputs follow.  top: the lane's largest score of its head.
template <int D, int NT>
__device__ __forceinline__ void move_reference(Heads<D, NT>& h, float (&top)[NT]) {
  const int lane = threadIdx.x & 31, c = lane & 3;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float m = top[t];
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
    float alpha = 1.f;
    if (m > h.ref[t] + kMoveAt) { alpha = ex2f(h.ref[t] - m); h.ref[t] = m; }      // (from -infinity: 0)
    h.sum[t] *= alpha;
    const float a0 = __shfl_sync(0xffffffffu, alpha, 8 * c), a1 = __shfl_sync(0xffffffffu, alpha, 8 * c + 4);
#pragma unroll
    for (int m16 = 0; m16 < D / 16; ++m16) {
      h.o[t][m16][0] *= a0; h.o[t][m16][1] *= a1;
      h.o[t][m16][2] *= a0; h.o[t][m16][3] *= a1;
    }
  }
}

// One block of 16 tokens at `block`, the first `valid` of which exist.
template <int D, int NT>
__device__ __forceinline__ void attend_block(Heads<D, NT>& h, const uint8_t* block, int valid) {
  constexpr int G = D / kGroup;
  const int lane = threadIdx.x & 31, c = lane & 3;
  // ---- scores ----
  float x[NT][4];                                        // tokens 2 c, 2 c + 1, 8 + 2 c, 9 + 2 c
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    uint32_t kw[G], sc[2 * G];
    if constexpr (D == 128) {
      const uint4 v = *reinterpret_cast<const uint4*>(block + half * 512 + lane * 16);
      kw[0] = v.x; kw[1] = v.y; kw[2] = v.z; kw[3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(block + lane * 16 + half * 8);
      kw[0] = v.x; kw[1] = v.y;
    }
#pragma unroll
    for (int i = 0; i < G / 2; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(block + Block<D>::kScaleK + (half * 4 + c) * G * 8 + i * 16);
      sc[4 * i] = v.x; sc[4 * i + 1] = v.y; sc[4 * i + 2] = v.z; sc[4 * i + 3] = v.w;
    }
    float s[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t][0] = s[t][1] = 0.f;
#pragma unroll
    for (int w = 0; w < G; ++w) {
      const uint32_t b0 = codes_at_4(kw[w] << 4), b1 = codes_at_4(kw[w]), b2 = codes_at_4(kw[w] >> 4), b3 = codes_at_4(kw[w] >> 8);
      float acc[4];
      acc[0] = acc[1] = -64.f * h.qsum[0][w];
      acc[2] = acc[3] = NT == 2 ? -64.f * h.qsum[NT - 1][w] : 0.f;
      mma_f16(acc, h.q[0][w][0], NT == 2 ? h.q[NT - 1][w][0] : 0u, h.q[0][w][1], NT == 2 ? h.q[NT - 1][w][1] : 0u, b0, b1);
      mma_f16(acc, h.q[0][w][2], NT == 2 ? h.q[NT - 1][w][2] : 0u, h.q[0][w][3], NT == 2 ? h.q[NT - 1][w][3] : 0u, b2, b3);
      const float2 fs = to_float2<__half>(sc[2 * w]), fm = to_float2<__half>(sc[2 * w + 1]);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        s[t][0] = fmaf(acc[2 * t], fs.x, fmaf(h.qsum[t][w], fm.x, s[t][0]));
        s[t][1] = fmaf(acc[2 * t + 1], fs.y, fmaf(h.qsum[t][w], fm.y, s[t][1]));
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      x[t][2 * half] = half * 8 + 2 * c < valid ? s[t][0] * h.scale[t] : -INFINITY;
      x[t][2 * half + 1] = half * 8 + 2 * c + 1 < valid ? s[t][1] * h.scale[t] : -INFINITY;
    }
  }
  // ---- weights ----
  float top[NT];
  bool move = false;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    top[t] = fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3]));
    move = move || top[t] > h.ref[t] + kMoveAt;
  }
  if (__any_sync(0xffffffffu, move)) move_reference<D, NT>(h, top);
  uint32_t p[NT][2];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const float ref = h.ref[t] == -INFINITY ? 0.f : h.ref[t];
    float e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = ex2f(x[t][i] - ref);
    h.sum[t] += (e[0] + e[1]) + (e[2] + e[3]);
    p[t][0] = from_float2<__half>(e[0], e[1]);
    p[t][1] = from_float2<__half>(e[2], e[3]);
  }
  // ---- values ----
  uint32_t sv[2][2 * G];                                 // (scale pair, minimum pair) of tokens (2 c, 2 c + 1), (8 + 2 c, 9 + 2 c)
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int i = 0; i < G / 2; ++i) {
      const uint4 v = *reinterpret_cast<const uint4*>(block + Block<D>::kScaleV + (half * 4 + c) * G * 8 + i * 16);
      sv[half][4 * i] = v.x; sv[half][4 * i + 1] = v.y; sv[half][4 * i + 2] = v.z; sv[half][4 * i + 3] = v.w;
    }
  if (valid < kBlockTokens) {                            // whatever the rest of the block holds: zeros
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t keep = (half * 8 + 2 * c < valid ? 0xffffu : 0u) | (half * 8 + 2 * c + 1 < valid ? 0xffff0000u : 0u);
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) sv[half][i] &= keep;
    }
  }
  const __half2 minus64 = __half2half2(__ushort_as_half(0xd400));
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const uint4 v = *reinterpret_cast<const uint4*>(block + Block<D>::kV + i * 512 + lane * 16);
    const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int u = 4 * i + j, w = u / 2;
      auto value = [&](uint32_t bits, int half) { return u32(__hfma2(__hadd2(h2(codes_at_4(bits)), minus64), h2(sv[half][2 * w]), h2(sv[half][2 * w + 1]))); };
      const uint32_t a0 = value(vw[j] << 4, 0), a1 = value(vw[j], 0), a2 = value(vw[j] >> 4, 1), a3 = value(vw[j] >> 8, 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) mma_f16(h.o[t][u], a0, a1, a2, a3, p[t][0], p[t][1]);
    }
  }
}

__device__ __forceinline__ void put(void* out, int kind, size_t at, float x) {
  if (kind == HYPERATTN_BF16) reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(x);
  else if (kind == HYPERATTN_FP16) reinterpret_cast<__half*>(out)[at] = __float2half_rn(x);
  else reinterpret_cast<float*>(out)[at] = x;
}

constexpr int kWarps = 4;

template <int D, int NT, class T>
__global__ void __launch_bounds__(32 * kWarps) cache_attn_kernel(CacheAttnArgs a, int chunks) {
  __shared__ float s_o[kWarps][8 * NT][D];
  __shared__ float s_ref[kWarps][8 * NT], s_sum[kWarps][8 * NT];
  wait_for_stream();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane & 3;
  const int r = blockIdx.x, kv = blockIdx.y / chunks, chunk = blockIdx.y % chunks;
  const int per_kv = a.q_heads / a.cache.heads, first = kv * per_kv + chunk * 8 * NT, heads = min(per_kv - chunk * 8 * NT, 8 * NT);
  Heads<D, NT> h;
  load_heads<D, NT, T>(h, a, r, first, heads);
  const int len = min(max(a.lengths[r], 0), a.width * a.cache.page), subs = a.cache.page / kBlockTokens;
  for (int b = warp; b * kBlockTokens < len; b += kWarps) {
    const int page = a.table[(size_t)r * a.width + b / subs];
    if (page < 0 || page >= a.cache.num_pages) continue;
    attend_block<D, NT>(h, block_at<D>(a.cache, page, kv, b % subs), min(len - b * kBlockTokens, kBlockTokens));
  }
  // ---- the warps' parts together ----
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float sum = h.sum[t];
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if (c == 0) { s_ref[warp][lane / 4 + 8 * t] = h.ref[t]; s_sum[warp][lane / 4 + 8 * t] = sum; }
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_o[warp][8 * t + 2 * c + (i & 1)][16 * m + lane / 4 + 8 * (i >> 1)] = h.o[t][m][i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < heads * D; i += 32 * kWarps) {
    const int head = i / D, x = i - head * D;
    float ref = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) ref = fmaxf(ref, s_ref[w][head]);
    float sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = s_ref[w][head] == -INFINITY ? (s_sum[w][head] == 0.f ? 0.f : 1.f) : ex2f(s_ref[w][head] - ref);   // (a sum without a reference: NaN)
      sum += f * s_sum[w][head];
      o += f * s_o[w][head][x];
    }
    const size_t row = (size_t)r * a.q_heads + first + head;
    put(a.out, a.out_kind, row * D + x, sum == 0.f ? 0.f : o / sum);
    if (x == 0) a.lse[row] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
  }
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_cache_attention_workspace_bytes(const hyperattn_cache_attention_params* p, size_t* bytes) {
  if (!p || !bytes) return HYPERATTN_INVALID_ARGUMENT;
  *bytes = 0;
  return HYPERATTN_OK;
}

extern "C" int hyperattn_cache_attention(const hyperattn_cache_attention_params* p) {
  int rc;
  if (!p || p->requests < 0 || p->table_width <= 0 || p->q_heads <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_cache(p->cache, &rc)) return rc;
  if (p->dtype != HYPERATTN_BF16 && p->dtype != HYPERATTN_FP16) return p->dtype == HYPERATTN_FP32 ? HYPERATTN_UNSUPPORTED_SHAPE : HYPERATTN_INVALID_ARGUMENT;
  if (p->out_dtype != p->dtype && p->out_dtype != HYPERATTN_FP32) return HYPERATTN_INVALID_ARGUMENT;
  if (p->q_heads % p->cache.kv_heads || bad_stride(p->q_row_stride) || bad_stride(p->q_head_stride)) return HYPERATTN_UNSUPPORTED_SHAPE;
  if ((long long)p->table_width * p->cache.page_tokens > 0x7fffffffLL) return HYPERATTN_UNSUPPORTED_SHAPE;
  if (p->requests == 0) return HYPERATTN_OK;
  if (!p->q || !p->out || !p->lse || !p->table || !p->lengths) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->q) || misaligned(p->out)) return HYPERATTN_MISALIGNED;
  CacheAttnArgs a;
  a.cache = {reinterpret_cast<uint8_t*>(p->cache.pages), p->cache.num_pages, p->cache.page_tokens, p->cache.kv_heads};
  a.q = p->q; a.q_row = p->q_row_stride; a.q_head = p->q_head_stride;
  a.out = p->out; a.lse = p->lse; a.table = p->table; a.lengths = p->lengths;
  a.requests = p->requests; a.width = p->table_width; a.q_heads = p->q_heads; a.out_kind = p->out_dtype;
  const int d = p->cache.d, per_kv = p->q_heads / p->cache.kv_heads;
  a.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.f / sqrtf((float)d)) * 1.4426950408889634f;
  const bool two = per_kv > 8;
  const int chunks = (per_kv + (two ? 15 : 7)) / (two ? 16 : 8);
  const dim3 grid((unsigned)p->requests, (unsigned)(p->cache.kv_heads * chunks));
  if (grid.y > 65535) return HYPERATTN_UNSUPPORTED_SHAPE;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  auto go = [&](auto kernel) {
    const cudaError_t e = launch(kernel, grid, dim3(32 * kWarps), 0, st, a, chunks);
    if (e == cudaSuccess) return (int)HYPERATTN_OK;
    std::fprintf(stderr, "hyperattn: cache attention failed: %s\n", cudaGetErrorString(e));
    return (int)HYPERATTN_CUDA_ERROR;
  };
  const bool bf16 = p->dtype == HYPERATTN_BF16;
  if (d == 64) {
    if (two) return bf16 ? go(cache_attn_kernel<64, 2, __nv_bfloat16>) : go(cache_attn_kernel<64, 2, __half>);
    return bf16 ? go(cache_attn_kernel<64, 1, __nv_bfloat16>) : go(cache_attn_kernel<64, 1, __half>);
  }
  if (two) return bf16 ? go(cache_attn_kernel<128, 2, __nv_bfloat16>) : go(cache_attn_kernel<128, 2, __half>);
  return bf16 ? go(cache_attn_kernel<128, 1, __nv_bfloat16>) : go(cache_attn_kernel<128, 1, __half>);
}
