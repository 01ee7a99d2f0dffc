// Attention of one query token a request over the paged 4-bit cache.
//
// A warp takes a block of 16 tokens of one key head and up to 16 query heads that read it, on the warp-level tensor cores
// (mma.sync m16n8k16, fp16 operands, fp32 sums):
//   S^T = K Q^T with the codes of K as fp16 numbers (see codes_of), exact sums of a group, s = sum_g scale_g sum(q c) + min_g sum_g(q) in fp32
//   p = exp2(s c - ref), the reference of a head moves when it is exceeded by more than 2^8
//   O^T += V^T P^T   V = min + scale * code in fp16 (exact codes, one rounding); its 32-bit words hold four tokens of two coordinates,
//               so that masking yields operands with pairs of tokens; P^T is turned once (movmatrix).
// fp16 and not bf16 for the weights and values: a product is then off by 2^-11 and not 2^-8, which is what the output's type can show; V fits by
// its format, a head's query after a power of two.  For fp16 results, which show 2^-11, the weights' rounding errors go through the products too.
//
// The blocks of all (request, key head, up to 16 heads) segments are one sequence, cut into equal parts, one for every warp that the
// GPU holds, whatever the lengths are.  A warp streams its blocks through a ring of its own in shared memory (bulk copies, no other
// warp to wait for).  A segment that lies in one part is finished there; pieces of others go to the workspace - one piece for a
// CTA that is inside a segment as a whole - and a second launch puts them together, in order, so that results do not depend on timing.
#include <cstdio>
#include <type_traits>
#include "serving.cuh"
#include "tc_util.cuh"

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
  int chunks;                                  // of query heads of a key head
  float scale_log2;
  int* starts;                                 // [requests + 1] units before each request; [requests + 1]: units of a warp's part
  float* part;                                 // pieces: [slots][heads of a chunk][d + 2] (outputs, reference, sum)
  int part_heads;                              // heads of a chunk
};

// c += A B, or d = A B (no registers to be cleared)
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ __half2 h2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
__device__ __forceinline__ uint32_t u32(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
// The codes of a word (8 of them, k at bit 4 k) as fp16 pairs (k, k + 4), k = 0..3: even ones as they are, odd ones 64 too large.  A code with the exponent
// of 2^6 above its bits 4..7 is 64 + c; both codes of a byte with that of 2^10 are 1024 + low + 16 high, from which 16 (64 + high) is taken.  (Two logical
// operations and half a shift for two pairs: those run at half the rate of the fused multiply-adds and are what a block has most of.)
struct Constants { uint32_t e6, e10, minus16, minus64; };       // fp16 pairs: 2^6, 2^10, -16, -64
__device__ __forceinline__ Constants constants() {                // (opaque, so that they stay in registers instead of being made again at every use)
  Constants k;
  asm volatile("mov.b32 %0, 0x54005400;\n\tmov.b32 %1, 0x64006400;\n\tmov.b32 %2, 0xcc00cc00;\n\tmov.b32 %3, 0xd400d400;" : "=r"(k.e6), "=r"(k.e10), "=r"(k.minus16), "=r"(k.minus64));
  return k;
}
template <uint32_t MASK> __device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t bits) {   // (one operation; written with & and | it became two)
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(w), "n"(MASK), "r"(bits));
  return r;
}
__device__ __forceinline__ void codes_of(uint32_t w, const Constants& n, uint32_t (&k)[4]) {
  const uint32_t up = w >> 8;
  k[1] = and_or<0x00f000f0u>(w, n.e6);
  k[3] = and_or<0x00f000f0u>(up, n.e6);
  k[0] = u32(__hfma2(h2(k[1]), h2(n.minus16), h2(and_or<0x00ff00ffu>(w, n.e10))));
  k[2] = u32(__hfma2(h2(k[3]), h2(n.minus16), h2(and_or<0x00ff00ffu>(up, n.e10))));
}

// What a warp keeps of the heads it works for: NT tiles of up to 8 of them.  As an operand a lane has head lane / 4, in results heads 2 c, 2 c + 1.
constexpr float kNoReference = 3.0e38f;
template <int D, int NT>
struct Heads {
  static constexpr int kGroups = D / kGroup;
  uint32_t q[NT][kGroups][4];           // fp16 pairs: coordinates 32 w + 8 c + 0..7
  uint32_t fix[NT][2];                  // operands of the product that adds what belongs to minima and to codes that are 64 too large, see load_heads
  float scale[NT][2];                   // to the base-2 scores
  float minus[NT][2], sum[NT][2];       // minus the reference (kNoReference: none yet); sum of this lane's tokens
  float o[NT][D / 16][4];               // O^T: coordinates lane / 4 (+ 8) of every 16
};

template <int D, int NT, class T>
__device__ __forceinline__ void load_heads(Heads<D, NT>& h, const CacheAttnArgs& a, int request, int first_head, int heads) {
  constexpr int G = Heads<D, NT>::kGroups;
  const int lane = threadIdx.x & 31, c = lane & 3;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int head = lane / 4 + 8 * t;
    float top = 0.f;
    uint4 raw[G];
#pragma unroll
    for (int w = 0; w < G; ++w) {
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
    const float down = __uint_as_float((uint32_t)(127 - e) << 23), scale = __uint_as_float((uint32_t)(127 + e) << 23) * a.scale_log2;
    // Scores want sum_g min_g sum(q) - 64 scale_g sum(q at odd codes).  That is one product more over 16 "coordinates" of a token: the minima of the groups,
    // again, their scales, again, with the sums (as two fp16 numbers, high and low part) as the query's entries.  A lane has groups 2 (c % 2), + 1 (d = 64:
    // 0, 1), the high parts for c < 2 (d = 64: c = 0), the low ones otherwise (c = 1; none).
    float all[G], odd[G];
#pragma unroll
    for (int w = 0; w < G; ++w) {
      const uint32_t v[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
      all[w] = odd[w] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = to_float2<T>(v[i]);
        h.q[t][w][i] = from_float2<__half>(f.x * down, f.y * down);
        const float2 r = to_float2<__half>(h.q[t][w][i]);
        all[w] += r.x + r.y;
        if (i & 1) odd[w] += r.x + r.y;
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        all[w] += __shfl_xor_sync(0xffffffffu, all[w], o);
        odd[w] += __shfl_xor_sync(0xffffffffu, odd[w], o);
      }
      odd[w] *= -64.f;
    }
    const bool second = G == 4 && (c & 1), low = G == 4 ? c >= 2 : c == 1, none = G == 2 && c >= 2;
    auto operand = [&](const float (&x)[G]) {
      const float x0 = second ? x[G - 2] : x[0], x1 = second ? x[G - 1] : x[1];
      const uint32_t high = from_float2<__half>(x0, x1);
      const float2 f = to_float2<__half>(high);
      return none ? 0u : low ? from_float2<__half>(x0 - f.x, x1 - f.y) : high;
    };
    h.fix[t][0] = operand(all);
    h.fix[t][1] = operand(odd);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      h.scale[t][i] = __shfl_sync(0xffffffffu, scale, 8 * c + 4 * i);
      h.minus[t][i] = kNoReference;
      h.sum[t][i] = 0.f;
    }
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) h.o[t][m][i] = 0.f;
  }
}

// One block of 16 tokens at `block`, the first `valid` of which exist.  FINE: what rounding the weights to fp16 has lost is added.
template <int D, int NT, bool FINE>
__device__ __forceinline__ void attend_block(Heads<D, NT>& h, const Constants& num, const uint8_t* block, int valid) {
  constexpr int G = D / kGroup;
  const int lane = threadIdx.x & 31, c = lane & 3;
  // ---- scores: S^T of tokens lane / 4 (+ 8) and heads 2 c, 2 c + 1 ----
  uint32_t kw[2][G], sc[2][G / 2], mn[2];                // codes, scales of group pairs, minima of the lane's pair (see load_heads)
  if constexpr (D == 128) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint4 v = *reinterpret_cast<const uint4*>(block + half * 512 + lane * 16);
      kw[half][0] = v.x; kw[half][1] = v.y; kw[half][2] = v.z; kw[half][3] = v.w;
    }
  } else {
    const uint4 v = *reinterpret_cast<const uint4*>(block + lane * 16);
    kw[0][0] = v.x; kw[0][1] = v.y; kw[1][0] = v.z; kw[1][1] = v.w;
  }
  const uint32_t pick = lane & 4 ? 0x7632u : 0x5410u;    // of two halves with tokens (2 i, 2 i + 1): the lane's token
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint8_t* at = block + Block<D>::kScaleK + (half * 4 + lane / 8) * G * 8;
    const uint4 v = *reinterpret_cast<const uint4*>(at);
    sc[half][0] = __byte_perm(v.x, v.z, pick);
    if constexpr (G == 2) mn[half] = __byte_perm(v.y, v.w, pick);
    else {
      const uint4 u = *reinterpret_cast<const uint4*>(at + 16);
      sc[half][G / 2 - 1] = __byte_perm(u.x, u.z, pick);
      mn[half] = __byte_perm(c & 1 ? u.y : v.y, c & 1 ? u.w : v.w, pick);
    }
  }
  float s[NT][4];
#pragma unroll
  for (int t = 0; t < NT; ++t)
    mma_f16_first(s[t], mn[0], mn[1], G == 4 && (c & 1) ? sc[0][G / 2 - 1] : sc[0][0], G == 4 && (c & 1) ? sc[1][G / 2 - 1] : sc[1][0], h.fix[t][0], h.fix[t][1]);
#pragma unroll
  for (int w = 0; w < G; ++w) {
    uint32_t k0[4], k1[4];
    codes_of(kw[0][w], num, k0);
    codes_of(kw[1][w], num, k1);
    const float2 f0 = to_float2<__half>(sc[0][w / 2]), f1 = to_float2<__half>(sc[1][w / 2]);
    const float a0 = w & 1 ? f0.y : f0.x, a1 = w & 1 ? f1.y : f1.x;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float acc[4];
      mma_f16_first(acc, k0[0], k1[0], k0[1], k1[1], h.q[t][w][0], h.q[t][w][1]);
      mma_f16(acc, k0[2], k1[2], k0[3], k1[3], h.q[t][w][2], h.q[t][w][3]);
      s[t][0] = fmaf(acc[0], a0, s[t][0]); s[t][1] = fmaf(acc[1], a0, s[t][1]);
      s[t][2] = fmaf(acc[2], a1, s[t][2]); s[t][3] = fmaf(acc[3], a1, s[t][3]);
    }
  }
  if (valid < kBlockTokens) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane / 4 + 8 * (i >> 1) >= valid) s[t][i] = -INFINITY;
  }
  // ---- weights ----
  float y[NT][4], most = -INFINITY;
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[t][i] = fmaf(s[t][i], h.scale[t][i & 1], h.minus[t][i & 1]);
      most = fmaxf(most, y[t][i]);
    }
  if (__any_sync(0xffffffffu, most > kMoveAt)) {
    // the references move to the scores' maximum where they are exceeded; sums and outputs follow
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float m = fmaxf(s[t][i], s[t][i + 2]) * h.scale[t][i];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (m + h.minus[t][i] > kMoveAt) {
          const float alpha = h.minus[t][i] == kNoReference ? 0.f : ex2(-h.minus[t][i] - m);
          h.minus[t][i] = -m;
          h.sum[t][i] *= alpha;
#pragma unroll
          for (int u = 0; u < D / 16; ++u) { h.o[t][u][i] *= alpha; h.o[t][u][i + 2] *= alpha; }
        }
        y[t][i] = fmaf(s[t][i], h.scale[t][i], h.minus[t][i]);
        y[t][i + 2] = fmaf(s[t][i + 2], h.scale[t][i], h.minus[t][i]);
      }
  }
  uint32_t p[NT][2], rest[NT][2];                        // P^T as an operand: head lane / 4, tokens 2 c, 2 c + 1 and 8 + 2 c, 9 + 2 c
  auto turn = [](uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
  };
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = ex2(y[t][i]);
    h.sum[t][0] += e[0] + e[2];
    h.sum[t][1] += e[1] + e[3];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t both = from_float2<__half>(e[2 * i], e[2 * i + 1]);
      p[t][i] = turn(both);
      if constexpr (FINE) {
        const float2 f = to_float2<__half>(both);
        rest[t][i] = turn(from_float2<__half>(e[2 * i] - f.x, e[2 * i + 1] - f.y));
      }
    }
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
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const uint4 v = *reinterpret_cast<const uint4*>(block + Block<D>::kV + i * 512 + lane * 16);
    const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int u = 4 * i + j, w = u / 2;
      uint32_t k[4];
      codes_of(vw[j], num, k);
      auto value = [&](__half2 code, int half) { return u32(__hfma2(code, h2(sv[half][2 * w]), h2(sv[half][2 * w + 1]))); };
      const uint32_t a0 = value(h2(k[0]), 0), a1 = value(__hadd2(h2(k[1]), h2(num.minus64)), 0), a2 = value(h2(k[2]), 1), a3 = value(__hadd2(h2(k[3]), h2(num.minus64)), 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        mma_f16(h.o[t][u], a0, a1, a2, a3, p[t][0], p[t][1]);
        if constexpr (FINE) mma_f16(h.o[t][u], a0, a1, a2, a3, rest[t][0], rest[t][1]);
      }
    }
  }
}

__device__ __forceinline__ void put(void* out, int kind, size_t at, float x) {
  if (kind == HYPERATTN_BF16) reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(x);
  else if (kind == HYPERATTN_FP16) reinterpret_cast<__half*>(out)[at] = __float2half_rn(x);
  else reinterpret_cast<float*>(out)[at] = x;
}

constexpr int kWarps = 4;
constexpr int kMaxRequests = 4096;      // running sums in shared memory

// A unit of work and of the ring: 32 (d = 128) or 64 tokens of a segment, 5 KB.
template <int D>
struct Ring {
  static constexpr int kUnit = D == 128 ? 2 : 4;                         // blocks
  static constexpr int kUnitBytes = kUnit * Block<D>::kBytes, kUnitTokens = kUnit * kBlockTokens;
  static constexpr int kStages = 2;                                      // units on their way, a warp
  static constexpr int kWarpBytes = kStages * kUnitBytes;                // (>= 16 x D floats: a warp's outputs, when the parts are put together)
  static constexpr int kOffBar = kWarps * kWarpBytes, kOffMisc = kOffBar + kWarps * kStages * 8, kOffStarts = kOffMisc + 768;
  static constexpr int bytes(int requests) { return kOffStarts + (requests + 1) * 4; }
};
// CTAs that an SM holds: by registers (two tiles of heads need 168 a thread), and by shared memory
template <int D, int NT> constexpr int ctas_by_registers() { return NT == 1 ? 4 : 3; }
template <int D> int ctas_by_memory(int requests) { return 227 * 1024 / (Ring<D>::bytes(requests) + 1024); }

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <int D> __device__ __forceinline__ int units_of(const CacheAttnArgs& a, int r) {
  return (min(max(a.lengths[r], 0), a.width * a.cache.page) + Ring<D>::kUnitTokens - 1) / Ring<D>::kUnitTokens;
}
// where the pieces of a segment lie: see combine
__device__ __forceinline__ float* piece_at(const CacheAttnArgs& a, long long slot, int head, int d) { return a.part + (slot * a.part_heads + head) * (d + 2); }

template <int D, int NT, class T>
__global__ void __launch_bounds__(32 * kWarps, (ctas_by_registers<D, NT>())) cache_attn_kernel(const __grid_constant__ CacheAttnArgs a, int* status) {
  using R = Ring<D>;
  constexpr bool FINE = std::is_same<T, __half>::value;
  extern __shared__ __align__(128) uint8_t smem[];
  int* s_starts = reinterpret_cast<int*>(smem + R::kOffStarts);          // [requests + 1] units (of one segment each) before a request
  int* s_sums = reinterpret_cast<int*>(smem + R::kOffMisc);              // [kWarps]
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + R::kOffMisc + 64);
  float* s_stat = reinterpret_cast<float*>(smem + R::kOffMisc + 128);    // [kWarps][16][2] references, sums
  const int tid = threadIdx.x, lane = tid & 31, c = lane & 3;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t ring = smem_u32(smem) + warp * R::kWarpBytes, bars = smem_u32(smem) + R::kOffBar + warp * R::kStages * 8;
  if (tid == 0) *s_abort = 0;
  if (lane == 0) {
    for (int st = 0; st < R::kStages; ++st) mbar_init(bars + 8 * st, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_stream();
  // ---- running sum of the requests' units ----
  const int per = (a.requests + 32 * kWarps - 1) / (32 * kWarps), r0 = min(a.requests, tid * per), r1 = min(a.requests, r0 + per);
  int mine = 0;
  for (int r = r0; r < r1; ++r) mine += units_of<D>(a, r);
  int run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += y; }
  if (lane == 31) s_sums[warp] = run;
  __syncthreads();
  run -= mine;
  for (int w = 0; w < warp; ++w) run += s_sums[w];
  for (int r = r0; r < r1; ++r) { s_starts[r] = run; run += units_of<D>(a, r); }
  if (tid == 32 * kWarps - 1) s_starts[a.requests] = run;
  __syncthreads();
  const int segs = a.cache.heads * a.chunks;                             // of a request
  const int total = s_starts[a.requests] * segs, warps = gridDim.x * kWarps, part = max(1, (total + warps - 1) / warps);
  if (blockIdx.x == 0) {
    for (int r = tid; r <= a.requests; r += 32 * kWarps) a.starts[r] = s_starts[r];
    if (tid == 0) a.starts[a.requests + 1] = part;
  }
  const int cta_first = (int)min((long long)blockIdx.x * kWarps * part, (long long)total), cta_end = (int)min((long long)cta_first + kWarps * part, (long long)total);
  const int first = (int)min((long long)cta_first + warp * part, (long long)total), end = min(first + min(part, total - first), total);
  const int count = end - first;                                  // units of this warp
  const int subs = a.cache.page / kBlockTokens, per_kv = a.q_heads / a.cache.heads;

  // A lane knows one block of the next 32 / kUnit units: its segment (of all requests'), how many tokens there are from its unit on, and which block of
  // the cache it is (-1: none).
  constexpr int U = R::kUnit, kBatch = 32 / U;
  struct Known { int seg, left, at; };
  auto know = [&](int unit) {                                            // units unit .. unit + kBatch - 1
    Known k = {0, 0, -1};
    const int i = unit + lane / U;
    if (i >= count) return k;
    const int n = first + i;
    int lo = 0, hi = a.requests;                                         // the last request whose units start there or before
    const int t = n / segs;
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (s_starts[mid] <= t) lo = mid; else hi = mid; }
    const int units = s_starts[lo + 1] - s_starts[lo];
    const int rest = n - s_starts[lo] * segs;
    const int seg = rest / units, b = (rest - seg * units) * U + lane % U;
    k.seg = lo * segs + seg;
    k.left = min(a.lengths[lo], a.width * a.cache.page) - (b - lane % U) * kBlockTokens;
    if ((lane % U) * kBlockTokens < k.left) {
      const int page = a.table[(size_t)lo * a.width + b / subs];
      if (page >= 0 && page < a.cache.num_pages) k.at = (page * a.cache.heads + seg / a.chunks) * subs + b % subs;
    }
    return k;
  };
  int asked = 0;                                                         // units whose copies have been asked for
  auto ask = [&](const Known& k, int from) {                              // the next one, known by lanes U from, ...
    const int st = asked % R::kStages;
    const uint32_t dst = ring + st * R::kUnitBytes, bar = bars + 8 * st;
    if (subs % U == 0) {                                                 // a unit never leaves its page: one copy
      const int at = __shfl_sync(0xffffffffu, k.at, U * from), left = __shfl_sync(0xffffffffu, k.left, U * from);
      if (lane == 0) {
        const uint32_t bytes = at < 0 ? 0 : (min(left, R::kUnitTokens) + kBlockTokens - 1) / kBlockTokens * Block<D>::kBytes;
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
        if (bytes) bulk_copy(dst, a.cache.pages + (size_t)at * Block<D>::kBytes, bytes, bar);
      }
    } else {
      const bool mine = lane / U == from && k.at >= 0;
      const unsigned all = __ballot_sync(0xffffffffu, mine);
      if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(__popc(all) * Block<D>::kBytes) : "memory");
      if (mine) bulk_copy(dst + (lane % U) * Block<D>::kBytes, a.cache.pages + (size_t)k.at * Block<D>::kBytes, Block<D>::kBytes, bar);
    }
    ++asked;
  };
  Known now = know(0), next = now;
  while (asked < R::kStages && asked < count) ask(now, asked);
  bool ok = true;
  const Constants num = constants();
  Heads<D, NT> h;
  int segment = -1, request = 0, seg = 0;                                // segment = request * segs + seg
  // the segment's results, or a piece of them
  auto flush = [&](float* to) {                                            // to: null for final results
    const int chunk = seg % a.chunks, kv = seg / a.chunks, first_head = kv * per_kv + chunk * 8 * NT, heads = min(per_kv - chunk * 8 * NT, 8 * NT);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum = h.sum[t][i];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float ref = h.minus[t][i] == kNoReference ? -INFINITY : -h.minus[t][i];
        const int head = 8 * t + 2 * c + i;
        if (head < heads) {
          const size_t row = (size_t)request * a.q_heads + first_head + head;
          if (lane < 4) {
            if (to) { to[head * (D + 2) + D] = ref; to[head * (D + 2) + D + 1] = sum; }
            else a.lse[row] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
          }
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
          for (int m = 0; m < D / 16; ++m)
#pragma unroll
            for (int up = 0; up < 2; ++up) {
              const int x = 16 * m + lane / 4 + 8 * up;
              const float v = h.o[t][m][i + 2 * up];
              if (to) to[head * (D + 2) + x] = v;
              else put(a.out, a.out_kind, row * D + x, v * inv);
            }
        }
      }
  };
  bool together = false;                                                 // the whole CTA works for one segment
  for (int n = 0; n < count; ++n) {
    const int at = n % kBatch;
    if (at == 0) {
      if (n > 0) now = next;
      next = know(n + kBatch);
    }
    const int sg = __shfl_sync(0xffffffffu, now.seg, at * U), left = __shfl_sync(0xffffffffu, now.left, at * U);
    const unsigned there = __ballot_sync(0xffffffffu, now.at >= 0) >> (at * U);
    if (sg != segment) {
      segment = sg;
      request = segment / segs; seg = segment - request * segs;
      const int kv = seg / a.chunks, chunk = seg - kv * a.chunks;
      load_heads<D, NT, T>(h, a, request, kv * per_kv + chunk * 8 * NT, min(per_kv - chunk * 8 * NT, 8 * NT));
    }
    const int st = n % R::kStages;
    ok = warp_wait<12>(bars + 8 * st, (uint32_t)(n / R::kStages) & 1, s_abort, status);
    if (!ok) break;
#pragma unroll 1
    for (int b = 0; b < U; ++b)
      if ((there >> b) & 1) attend_block<D, NT, FINE>(h, num, smem + warp * R::kWarpBytes + st * R::kUnitBytes + b * Block<D>::kBytes, left - b * kBlockTokens);
    __syncwarp();
    if (asked < count) { if (at + R::kStages < kBatch) ask(now, at + R::kStages); else ask(next, at + R::kStages - kBatch); }
    if (left <= R::kUnitTokens || n + 1 == count) {                        // the segment's last unit, or the part's
      const int units = s_starts[request + 1] - s_starts[request], seg_first = s_starts[request] * segs + seg * units, seg_end = seg_first + units;
      if (seg_first >= first && seg_end <= end) flush(nullptr);
      else {
        together = seg_first <= cta_first && seg_end >= cta_end;
        if (!together) flush(piece_at(a, 2 * ((long long)blockIdx.x * kWarps + warp) + (seg_first < first ? 0 : 1), 0, D));
      }
    }
  }
  if (!ok)                                                               // nothing may be on its way into shared memory when the CTA ends
    for (int st = 0; st < R::kStages && st < asked; ++st) mbar_drain(bars + 8 * st, (uint32_t)((asked - 1 - st) / R::kStages) & 1);
  // ---- a CTA inside one segment: one piece ----
  if (__syncthreads_or(together)) {
    float* s_o = reinterpret_cast<float*>(smem + warp * R::kWarpBytes);  // [8 NT][D] of this warp
    if (together) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int head = 8 * t + 2 * c + i;
          float sum = h.sum[t][i];
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          if (lane < 4) { s_stat[(warp * 16 + head) * 2] = h.minus[t][i] == kNoReference ? -INFINITY : -h.minus[t][i]; s_stat[(warp * 16 + head) * 2 + 1] = sum; }
#pragma unroll
          for (int m = 0; m < D / 16; ++m)
#pragma unroll
            for (int up = 0; up < 2; ++up) s_o[head * D + 16 * m + lane / 4 + 8 * up] = h.o[t][m][i + 2 * up];
        }
    }
    __syncthreads();
    const int used = (int)((cta_end - cta_first + part - 1) / part);     // warps that have a part
    const int heads = min(per_kv - (seg % a.chunks) * 8 * NT, 8 * NT);
    if (warp < used) {
      for (int i = warp * 32 + lane; i < heads * D; i += used * 32) {
        const int head = i / D, x = i - head * D;
        float ref = -INFINITY;
        for (int w = 0; w < used; ++w) ref = fmaxf(ref, s_stat[(w * 16 + head) * 2]);
        float sum = 0.f, o = 0.f;
        for (int w = 0; w < used; ++w) {
          const float rw = s_stat[(w * 16 + head) * 2], sw = s_stat[(w * 16 + head) * 2 + 1];
          const float f = rw == -INFINITY ? (sw == 0.f ? 0.f : 1.f) : ex2(rw - ref);          // (a sum without a reference: NaN)
          sum += f * sw;
          o += f * reinterpret_cast<const float*>(smem + w * R::kWarpBytes)[i];
        }
        float* to = piece_at(a, 2 * (long long)blockIdx.x * kWarps, head, D);
        to[x] = o;
        if (x == 0) { to[D] = ref; to[D + 1] = sum; }
      }
    }
  }
}

// Puts the pieces of segments together that lie in several parts; requests without tokens get their zeros.
constexpr int kJoinThreads = 128;

template <int D>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ CacheAttnArgs a, int heads_per_cta) {
  constexpr int LANES = D / 4, ROWS = kJoinThreads / LANES;               // a thread: four coordinates of every ROWS-th piece
  __shared__ float4 s_o[ROWS][LANES];
  __shared__ float s_ref[ROWS], s_sum[ROWS];
  wait_for_stream();
  const int segs = a.cache.heads * a.chunks, per_kv = a.q_heads / a.cache.heads;
  const int r = blockIdx.x / segs, seg = blockIdx.x - r * segs, kv = seg / a.chunks, chunk = seg - kv * a.chunks;
  const int first_head = kv * per_kv + chunk * a.part_heads, heads = min(per_kv - chunk * a.part_heads, a.part_heads);
  const long long part = a.starts[a.requests + 1], units = a.starts[r + 1] - a.starts[r];
  const long long begin = (long long)a.starts[r] * segs + seg * units, end = begin + units, cta_part = part * kWarps, total = (long long)a.starts[a.requests] * segs;
  const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
  const int h0 = blockIdx.y * heads_per_cta, h1 = min(h0 + heads_per_cta, heads);
  if (units == 0) {
    for (int i = threadIdx.x; i < (h1 - h0) * D; i += kJoinThreads) put(a.out, a.out_kind, ((size_t)r * a.q_heads + first_head + h0) * D + i, 0.f);
    for (int i = h0 + threadIdx.x; i < h1; i += kJoinThreads) a.lse[(size_t)r * a.q_heads + first_head + i] = -INFINITY;
    return;
  }
  const long long w0 = begin / part, w1 = (end - 1) / part;               // warps that have a part of it
  if (w0 == w1) return;                                                   // finished there
  // Its pieces in order: those of the first CTA's warps (or its one), one of every CTA inside, those of the last CTA's warps (or its one)
  const long long c0 = w0 / kWarps, c1 = w1 / kWarps;
  auto whole = [&](long long cta) { return cta * cta_part >= begin && min((cta + 1) * cta_part, total) <= end; };
  const int n0 = whole(c0) ? 1 : (int)(min(w1, c0 * kWarps + kWarps - 1) - w0 + 1);
  const int n1 = c1 == c0 ? 0 : whole(c1) ? 1 : (int)(w1 - c1 * kWarps + 1);
  const int inside = c1 > c0 ? (int)(c1 - c0 - 1) : 0, count = n0 + inside + n1;
  auto slot_of = [&](int i) {
    long long w;
    if (i < n0) { if (whole(c0)) return 2 * c0 * kWarps; w = w0 + i; }
    else if (i < n0 + inside) return 2 * (c0 + 1 + i - n0) * kWarps;
    else { if (whole(c1)) return 2 * c1 * kWarps; w = c1 * kWarps + (i - n0 - inside); }
    return 2 * w + (begin < w * part ? 0 : 1);
  };
  for (int head = h0; head < h1; ++head) {
    float ref = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = row; i < count; i += ROWS) {
      const float* from = piece_at(a, slot_of(i), head, D);
      const float rw = from[D], sw = from[D + 1];
      const float2 lo = *reinterpret_cast<const float2*>(from + 4 * lane), hi = *reinterpret_cast<const float2*>(from + 4 * lane + 2);
      const float m = fmaxf(ref, rw);
      const float f = rw == -INFINITY ? (sw == 0.f ? 0.f : 1.f) : ex2(rw - m), g = ref == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : ex2(ref - m);
      ref = m;
      sum = sum * g + sw * f;
      o = make_float4(o.x * g + lo.x * f, o.y * g + lo.y * f, o.z * g + hi.x * f, o.w * g + hi.y * f);
    }
    s_o[row][lane] = o;
    if (lane == 0) { s_ref[row] = ref; s_sum[row] = sum; }
    __syncthreads();
    if (row == 0) {
      float m = ref;
#pragma unroll
      for (int i = 1; i < ROWS; ++i) m = fmaxf(m, s_ref[i]);
      sum = 0.f;
      o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const float f = s_ref[i] == -INFINITY ? (s_sum[i] == 0.f ? 0.f : 1.f) : ex2(s_ref[i] - m);
        sum += f * s_sum[i];
        o = make_float4(o.x + f * s_o[i][lane].x, o.y + f * s_o[i][lane].y, o.z + f * s_o[i][lane].z, o.w + f * s_o[i][lane].w);
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const size_t at = (size_t)r * a.q_heads + first_head + head;
      const float v[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
#pragma unroll
      for (int i = 0; i < 4; ++i) put(a.out, a.out_kind, at * D + 4 * lane + i, v[i]);
      if (lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
    }
    __syncthreads();
  }
}

// What a call's launches look like: heads of a chunk, CTAs, bytes of the workspace (which follow from the call's arguments alone)
struct Shape { bool two; int chunks, part_heads, ctas; size_t starts, bytes; };
Shape shape_of(const hyperattn_cache_attention_params& p) {
  Shape s;
  const int per_kv = p.q_heads / p.cache.kv_heads;
  s.two = per_kv > 8;
  s.chunks = (per_kv + (s.two ? 15 : 7)) / (s.two ? 16 : 8);
  s.part_heads = s.two ? 16 : 8;
  if (s.part_heads > per_kv) s.part_heads = per_kv;
  const int unit = p.cache.d == 64 ? Ring<64>::kUnitTokens : Ring<128>::kUnitTokens;
  const long long units = (long long)p.requests * p.cache.kv_heads * s.chunks * (((long long)p.table_width * p.cache.page_tokens + unit - 1) / unit);
  const long long ctas = (units + kWarps - 1) / kWarps;
  const int memory = p.cache.d == 64 ? ctas_by_memory<64>(p.requests) : ctas_by_memory<128>(p.requests), registers = s.two ? ctas_by_registers<128, 2>() : ctas_by_registers<128, 1>();
  const int most = kSms * (memory < registers ? memory : registers);
  s.ctas = (int)(ctas < most ? ctas : most);
  s.starts = ((size_t)(p.requests + 2) * 4 + 255) / 256 * 256;
  s.bytes = s.starts + (size_t)s.ctas * kWarps * 2 * s.part_heads * (p.cache.d + 2) * 4;
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
  CacheAttnArgs a;
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
    cudaError_t e = launch(kernel, dim3((unsigned)s.ctas), dim3(32 * kWarps), Ring<D>::bytes(p->requests), st, a, status);
    // few segments: a CTA for a head or some
    int split = (4 * kSms + segments - 1) / segments;
    if (split > s.part_heads) split = s.part_heads;
    const int heads = (s.part_heads + split - 1) / split;
    if (e == cudaSuccess) e = launch(join_kernel<D>, dim3((unsigned)segments, (unsigned)((s.part_heads + heads - 1) / heads)), dim3(kJoinThreads), 0, st, a, heads);
    if (e == cudaSuccess) return (int)HYPERATTN_OK;
    std::fprintf(stderr, "hyperattn: cache attention failed: %s\n", cudaGetErrorString(e));
    return (int)HYPERATTN_CUDA_ERROR;
  };
  auto build = [&](auto dim, auto tiles, auto type) {
    constexpr int D = decltype(dim)::value, NT = decltype(tiles)::value;
    using T = decltype(type);
    if (allow_smem<cache_attn_kernel<D, NT, T>>(Ring<D>::bytes(kMaxRequests)) != cudaSuccess) return (int)HYPERATTN_CUDA_ERROR;
    return go(dim, cache_attn_kernel<D, NT, T>);
  };
  auto of_type = [&](auto dim, auto tiles) { return p->dtype == HYPERATTN_BF16 ? build(dim, tiles, __nv_bfloat16()) : build(dim, tiles, __half()); };
  auto of_tiles = [&](auto dim) { return s.two ? of_type(dim, std::integral_constant<int, 2>{}) : of_type(dim, std::integral_constant<int, 1>{}); };
  return d == 64 ? of_tiles(std::integral_constant<int, 64>{}) : of_tiles(std::integral_constant<int, 128>{});
}
