// Attention of one query token a request, or of a few, over the paged 4-bit cache, and the weight that cached tokens get from such queries: the kernels, which
// cache_attn.cu and cache_rows.cu build and launch.
//
// A warp takes a block of 16 tokens of one key head and up to 16 query heads that read it, on the warp-level tensor cores
// (mma.sync m16n8k16, fp16 operands, fp32 sums):
//   S^T = K Q^T with the codes of K as fp16 numbers (see codes_of), exact sums of a group:  s = sum_g scale_g sum(q c) + min_g sum_g(q)  in fp32
//   p = exp2(s c - ref), the reference of a head is set 2^12 below its largest score and moves when that exceeds it by 2^14; P^T is turned once (movmatrix)
//   O^T += V^T P^T  likewise: V = min + scale * code, so the codes meet the weights times the group's scales, the minima the weights.  V's 32-bit words
//               hold four tokens of two coordinates, so that masking yields operands with pairs of tokens.
// fp16 and not bf16 for the weights: they are then off by 2^-11 and not 2^-8, which bf16 results do not show; for fp16 results what the rounding has lost goes
// through the products too.  What rounding a weight times a scale has lost always does: scale * code and minimum are both larger than the value they add up to.
//
// A segment is a request, a key head and up to 8 or 16 of its query heads.  The tokens of all segments are one sequence of units of 5 KB, cut into equal
// parts, one for every warp that the GPU holds, whatever the lengths are.  A warp streams its units through a ring of its own in shared memory (bulk
// copies, no other warp to wait for).  A segment that lies in one part is finished there; pieces of others go to the workspace - one piece for
// a CTA that is inside a segment as a whole - and a second launch puts them together, in order, so that results do not depend on timing.
//
// What bounds it: no unit is full (issue 58 to 63 % of the cycles, the pipe of logical operations 54 to 59 %, DRAM half); four warps a scheduler, which their 128 registers
// leave room for, do not cover the fixed latencies of their chains of about 190 (d = 64) or 330 (d = 128) operations a block.  2 requests of up to 131072
// tokens, 32 heads of 64: 149 us, 658 MB at 4.4 TB/s (68 % of copy bandwidth; the copies without the arithmetic 103 us).  64 requests of up to 8192,
// 32 / 8 heads of 128: 67 us, 4.1 TB/s, of which the running sums, the first loads and the join take 14.  4 requests of up to 600: 10.5 us, two launches of
// dependent loads.  16 requests of up to 32768, 32 / 2 heads of 128 (two tiles of heads): 55 us for a floor of 13.
#pragma once
#include <cstdio>
#include <type_traits>
#include "serving.cuh"
#include "tc_util.cuh"

namespace hyperattn {
namespace {

constexpr float kBelow = 12.f, kMoveAt = 14.f;      // octaves that a head's reference is set below its largest score, and that scores may exceed it by before it moves: weights
                                                    // of up to 2^14 use fp16's range, and times a scale below 2 they are still numbers

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
  // several queries a request: its rows are its tokens times the query heads of a key head, a chunk some of them
  const int32_t* cu_q;
  int rows, causal, most;                      // most: requests with more rows than this are not for this launch
  const float *lse_in, *before;                // weights: log-sum-exps of the rows, what tokens had
  float* weights;
  float decay;
};

// K's codes, scales and minima of `run` blocks that follow each other, as boxes of the cache
struct alignas(64) KeyMaps {
  CUtensorMap codes, scales;
};

// What a build is for: one query a request; some rows a request; the weight that tokens get from some rows
enum Mode { kOneQuery, kSomeRows, kWeights };

template <Mode MODE> struct KernelArgs : CacheAttnArgs {};
template <> struct KernelArgs<kWeights> : CacheAttnArgs {
  KeyMaps maps;
  int run;                                     // blocks of a copy: the largest power of two, up to a unit, that divides a page's
};

__device__ __forceinline__ int group_of(const CacheAttnArgs& a) { return a.q_heads / a.cache.heads; }
// a request's tokens of queries (first row, how many; -1: it has more rows than this launch is for)
__device__ __forceinline__ int2 queries_of(const CacheAttnArgs& a, int r) {
  if (!a.cu_q) return make_int2(r, group_of(a) > a.most ? -1 : 1);
  const int first = min(max(a.cu_q[r], 0), a.rows), n = min(max(a.cu_q[r + 1], first), a.rows) - first;
  return make_int2(first, n * group_of(a) > a.most ? -1 : n);
}
// the chunks of a request come after those of the ones before it, wherever those end
__host__ __device__ __forceinline__ long long chunk_slots(long long rows_before, int requests_before, int group, int per_chunk) { return rows_before * group / per_chunk + requests_before; }
constexpr int kNeverSeen = 1 << 30;

// c += A B, or d = A B (no registers to be cleared), the latter over 8 too
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
__device__ __forceinline__ void mma_f16_first8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%7,%7,%7,%7};\n"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(b0), "f"(0.f));
}
__device__ __forceinline__ __half2 h2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
__device__ __forceinline__ uint32_t u32(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
// The codes of a word (8 of them, k at bit 4 k) as fp16 pairs (k, k + 4), k = 0..3.  A code in the lowest bits of an fp16 number is that number:
// c 2^-24 at bits 0..3 and c 2^-20 at bits 4..7, subnormal and exact, and products take them as any others.  So five logical operations are all that
// eight codes cost; the powers of two are made up for in the queries (even k) and in results.
constexpr float kTwo20 = 1048576.f, kTwo24 = 16777216.f;
__device__ __forceinline__ void codes_of(uint32_t w, uint32_t (&k)[4]) {
  const uint32_t up = w >> 8;
  k[0] = w & 0x000f000fu;
  k[1] = w & 0x00f000f0u;
  k[2] = up & 0x000f000fu;
  k[3] = up & 0x00f000f0u;
}

// What a warp keeps of the heads it works for: NT tiles of up to 8 of them.  As an operand a lane has head lane / 4, in results heads 2 c, 2 c + 1.
constexpr float kNoReference = 3.0e38f;
template <int D, int NT>
struct Heads {
  static constexpr int kGroups = D / kGroup;
  uint32_t q[NT][kGroups][4];           // fp16 pairs: coordinates 32 w + 8 c + 0..7, 0, 1, 4, 5 of them times 16
  uint32_t sums[NT];                    // operand of the product with the minima, see load_heads
  float scale[NT][2];                   // to the base-2 scores
  float minus[NT][2], sum[NT][2];       // minus the reference (kNoReference: none yet); sum of this lane's tokens
  float o[NT][D / 16][4];               // O^T without the minima: coordinates lane / 4 (times 2^-24) and lane / 4 + 8 (times 2^-20) of every 16
  float om[NT][2];                      // sum of weights times minima of group lane / 4
  int back[NT][2], most_back;           // some rows: the last token that a row sees, from the end of the request's (1: the last one); the most of the chunk's
};

// Heads first_head, ... of a request, `heads` of them; with several queries a request, rows first_head, ... of key head kv.
template <int D, int NT, bool PAIR, class T, Mode MODE>
__device__ __forceinline__ void load_heads(Heads<D, NT>& h, const CacheAttnArgs& a, int request, int first_head, int heads, int kv, int2 queries) {
  constexpr int G = Heads<D, NT>::kGroups;
  const int lane = threadIdx.x & 31, c = lane & 3;
  float lse[NT][2];                                      // weights: of the rows of the lane's results (asked for beside the queries)
  if constexpr (MODE == kWeights) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int g = group_of(a), mine = 8 * t + 2 * c + i, row = first_head + mine, token = row / g;
        lse[t][i] = mine < heads ? a.lse_in[(size_t)(queries.x + token) * a.q_heads + kv * g + row - token * g] : -INFINITY;
      }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int head = PAIR ? lane / 4 % 4 : lane / 4 + 8 * t;
    float top = 0.f;
    uint4 raw[G];
#pragma unroll
    for (int w = 0; w < G; ++w) {
      raw[w] = make_uint4(0, 0, 0, 0);
      if constexpr (MODE != kOneQuery) {
        if (head < heads) {
          const int g = group_of(a), row = first_head + head, token = row / g;
          raw[w] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.q) + (long long)(queries.x + token) * a.q_row + (long long)(kv * g + row - token * g) * a.q_head + 32 * w + 8 * c);
        }
      } else if (head < heads)
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
    // Scores want sum_g min_g sum(q): one product more, over 8 "coordinates" of a token, the minima of the groups and again, with the sums (as two fp16
    // numbers, high and low part) as the query's entries.  A lane has groups 2 (c % 2), + 1 (d = 64: 0, 1), the high parts for c < 2 (d = 64: c = 0), the
    // low ones otherwise (c = 1; none).
    float all[G];
#pragma unroll
    for (int w = 0; w < G; ++w) {
      const uint32_t v[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
      all[w] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = to_float2<T>(v[i]);
        const uint32_t entry = from_float2<__half>(f.x * down, f.y * down);
        const float2 r = to_float2<__half>(entry);
        all[w] += r.x + r.y;
        h.q[t][w][i] = i & 1 ? entry : from_float2<__half>(r.x * 16.f, r.y * 16.f);
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) all[w] += __shfl_xor_sync(0xffffffffu, all[w], o);
    }
    const bool second = G == 4 && (c & 1), low = G == 4 ? c >= 2 : c == 1, none = G == 2 && c >= 2;
    const float x0 = second ? all[G - 2] : all[0], x1 = second ? all[G - 1] : all[1];
    const uint32_t high = from_float2<__half>(x0, x1);
    const float2 hf = to_float2<__half>(high);
    h.sums[t] = none ? 0u : low ? from_float2<__half>(x0 - hf.x, x1 - hf.y) : high;
#pragma unroll
    for (int i = 0; i < 2; ++i) h.om[t][i] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      h.scale[t][i] = __shfl_sync(0xffffffffu, scale, 8 * c + 4 * i);
      h.minus[t][i] = kNoReference;
      h.sum[t][i] = 0.f;
      if constexpr (MODE != kOneQuery) {
        const int g = group_of(a), mine = PAIR ? (2 * c + i) % 4 : 8 * t + 2 * c + i, row = first_head + mine, token = row / g;
        h.back[t][i] = mine >= heads ? kNeverSeen : a.causal ? queries.y - token : 1;
        if constexpr (MODE == kWeights) h.minus[t][i] = lse[t][i] == -INFINITY ? -INFINITY : -lse[t][i] * 1.4426950408889634f;           // (a row that saw nothing gives nothing)
      }
    }
#pragma unroll
    for (int m = 0; m < D / 16; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) h.o[t][m][i] = 0.f;
  }
  if constexpr (MODE != kOneQuery) h.most_back = a.causal ? queries.y - first_head / group_of(a) : 1;
}

// Scores of one block of 16 tokens at `block`, the first `valid` of which exist: S^T of tokens lane / 4 (+ 8) and heads 2 c, 2 c + 1.  scales: K's.
template <int D, int NT, Mode MODE>
__device__ __forceinline__ void scores_of(const Heads<D, NT>& h, const uint8_t* block, const uint8_t* scales, int valid, float (&s)[NT][4]) {
  constexpr int G = D / kGroup;
  const int lane = threadIdx.x & 31, c = lane & 3;
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
    const uint8_t* at = scales + (half * 4 + lane / 8) * G * 8;
    const uint4 v = *reinterpret_cast<const uint4*>(at);
    sc[half][0] = __byte_perm(v.x, v.z, pick);
    if constexpr (G == 2) mn[half] = __byte_perm(v.y, v.w, pick);
    else {
      const uint4 u = *reinterpret_cast<const uint4*>(at + 16);
      sc[half][G / 2 - 1] = __byte_perm(u.x, u.z, pick);
      mn[half] = __byte_perm(c & 1 ? u.y : v.y, c & 1 ? u.w : v.w, pick);
    }
  }
#pragma unroll
  for (int w = 0; w < G; ++w) {
    uint32_t k0[4], k1[4];
    codes_of(kw[0][w], k0);
    codes_of(kw[1][w], k1);
    const float2 f0 = to_float2<__half>(sc[0][w / 2]), f1 = to_float2<__half>(sc[1][w / 2]);
    const float a0 = w & 1 ? f0.y : f0.x, a1 = w & 1 ? f1.y : f1.x;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float acc[4];
      mma_f16_first(acc, k0[0], k1[0], k0[1], k1[1], h.q[t][w][0], h.q[t][w][1]);
      mma_f16(acc, k0[2], k1[2], k0[3], k1[3], h.q[t][w][2], h.q[t][w][3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = w ? fmaf(acc[i], i < 2 ? a0 : a1, s[t][i]) : acc[i] * (i < 2 ? a0 : a1);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float m[4];
    mma_f16_first8(m, mn[0], mn[1], h.sums[t]);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[t][i] = fmaf(s[t][i], kTwo20, m[i]);
  }
  if constexpr (MODE != kOneQuery) {
    if (valid < kBlockTokens - 1 + h.most_back) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (lane / 4 + 8 * (i >> 1) > valid - h.back[t][i & 1]) s[t][i] = -INFINITY;
    }
  } else if (valid < kBlockTokens) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane / 4 + 8 * (i >> 1) >= valid) s[t][i] = -INFINITY;
  }
}

// O^T += V^T P^T of NB blocks, P^T (and what rounding it to fp16 has lost) as operands: the codes with the weights times the scales, the minima with the weights.
// The products of the blocks are summed from zero and then added to O: the tensor cores' sums are cut, not rounded, and both parts of O are many times
// as large as what they add up to in a long context (131072 tokens in one chain of products a warp: results off by 0.7 %; like this 0.024 %).
// PAIR: up to four heads, twice.  Columns 4 .. 7 of the operand P^T have what the rounding of columns 0 .. 3 has lost, in the same product; the two are added at the
// segment's end.  (2 x 131072 tokens, 32 / 32 heads of 64: 156 -> 150 us; 64 requests, 32 / 8 of 128: 71 -> 67.)
template <int D, int NT, bool PAIR, int NB, bool FINE, Mode MODE>
__device__ __forceinline__ void add_values(Heads<D, NT>& h, const uint8_t* block, const int (&valid)[NB], uint32_t (&p)[NB][NT][2], uint32_t (&rest)[NB][NT][2]) {
  constexpr int G = D / kGroup;
  const int lane = threadIdx.x & 31, c = lane & 3;
  const bool upper = lane >= 16;                         // (the lane's column of P^T is one of 4 .. 7)
  uint32_t sv[NB][2][G], mv[NB][2];                      // scales of tokens (2 c, 2 c + 1), (8 + 2 c, 9 + 2 c); minima of those of group lane / 4
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const uint8_t* scales = block + b * Block<D>::kBytes + Block<D>::kScaleV;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int i = 0; i < G / 2; ++i) {
        const uint4 v = *reinterpret_cast<const uint4*>(scales + (half * 4 + c) * G * 8 + i * 16);
        sv[b][half][2 * i] = v.x; sv[b][half][2 * i + 1] = v.z;
      }
      mv[b][half] = *reinterpret_cast<const uint32_t*>(scales + ((half * 4 + c) * G + lane / 4 % G) * 8 + 4);
    }
    if (valid[b] < kBlockTokens) {                       // whatever the rest of the block holds: zeros
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t keep = (half * 8 + 2 * c < valid[b] ? 0xffffu : 0u) | (half * 8 + 2 * c + 1 < valid[b] ? 0xffff0000u : 0u);
#pragma unroll
        for (int i = 0; i < G; ++i) sv[b][half][i] &= keep;
        mv[b][half] &= keep;
      }
    }
    // Some rows: a NaN in the values of tokens that not all rows see would reach the others as 0 * NaN; it becomes zero, and NaN the sums of the rows that do see it.
    if constexpr (MODE == kSomeRows) {
      if (valid[b] < kBlockTokens - 1 + h.most_back) {
        uint32_t flags = 0;                              // of the lane's four tokens: bit 4 (2 half + second) + group
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          auto look = [&](uint32_t& x, int g) {
            const uint32_t bad = ((x & 0x7fff7fffu) + 0x04000400u) & 0x80008000u;
            x &= ~((bad >> 15) * 0xffffu);
            flags |= (bad >> 15 & 1u) << (8 * half + g) | (bad >> 31) << (8 * half + 4 + g);
          };
#pragma unroll
          for (int i = 0; i < G; ++i) look(sv[b][half][i], i);
          look(mv[b][half], lane / 4 % G);
        }
        if (__any_sync(0xffffffffu, flags)) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) flags |= __shfl_xor_sync(0xffffffffu, flags, o);
          // (a scale that is no number while the minimum is one, or the other way round: both go)
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t gone = e ? 0xffff0000u : 0xffffu;
#pragma unroll
              for (int i = 0; i < G; ++i)
                if (flags >> (8 * half + 4 * e + i) & 1) sv[b][half][i] &= ~gone;
              if (flags >> (8 * half + 4 * e + lane / 4 % G) & 1) mv[b][half] &= ~gone;
            }
#pragma unroll
          for (int cc = 0; cc < 4; ++cc) {
            const uint32_t f = __shfl_sync(0xffffffffu, flags, cc);
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (f >> (4 * k + lane / 4 % G) & 1) {
                const int token = k / 2 * 8 + 2 * cc + k % 2;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                  for (int i = 0; i < 2; ++i)
                    if (token <= valid[b] - h.back[t][i]) h.om[t][i] = NAN;
              }
          }
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float m[4];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if constexpr (PAIR) {
        const uint32_t w0 = upper ? (FINE ? rest[b][t][0] : 0u) : p[b][t][0], w1 = upper ? (FINE ? rest[b][t][1] : 0u) : p[b][t][1];
        if (b == 0) mma_f16_first(m, mv[b][0], 0u, mv[b][1], 0u, w0, w1);
        else mma_f16(m, mv[b][0], 0u, mv[b][1], 0u, w0, w1);
        continue;
      }
      if (b == 0) mma_f16_first(m, mv[b][0], 0u, mv[b][1], 0u, p[b][t][0], p[b][t][1]);
      else mma_f16(m, mv[b][0], 0u, mv[b][1], 0u, p[b][t][0], p[b][t][1]);
      if constexpr (FINE) mma_f16(m, mv[b][0], 0u, mv[b][1], 0u, rest[b][t][0], rest[b][t][1]);
    }
    unpack_f2(fadd2(pack_f2(h.om[t][0], h.om[t][1]), pack_f2(m[0], m[1])), h.om[t][0], h.om[t][1]);
  }
  // Scales of 2 and more (values that differ by 30 in a group): the weights get so much smaller that the products stay numbers, the sums larger.  What a weight then
  // loses below fp16's 2^-24 is lost: 2^-25 beside a largest one of 2^(12 - k).
  uint32_t any = 0;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < G; ++i) any |= sv[b][half][i];
  float up = 1.f;
  if (__any_sync(0xffffffffu, any & 0x40004000u)) {
    __half2 most = __half2half2(__ushort_as_half(0));    // the largest scales (of a number and NaN the number: a NaN's group is NaN whatever the others are multiplied with)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < G; ++i) most = __hmax2(most, h2(sv[b][half][i]));
    const uint32_t top = __reduce_max_sync(0xffffffffu, max(u32(most) & 0xffffu, u32(most) >> 16));
    const int k = max((int)(top >> 10) - 15, 0);         // all scales are below 2^(k + 1)
    const __half2 down = __half2half2(__float2half_rn(__uint_as_float((uint32_t)(127 - k) << 23)));
    up = __uint_as_float((uint32_t)(127 + k) << 23);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          p[b][t][half] = u32(__hmul2(h2(p[b][t][half]), down));
          if constexpr (FINE) rest[b][t][half] = u32(__hmul2(h2(rest[b][t][half]), down));
        }
  }
  uint32_t minus[NB][NT][2];                             // PAIR: minus the weights in columns 4 .. 7, so that p s + (minus s) is the product there rounded off, elsewhere the product
  if constexpr (PAIR) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          minus[b][t][half] = upper ? p[b][t][half] ^ 0x80008000u : 0u;
          if constexpr (FINE) rest[b][t][half] = upper ? rest[b][t][half] : 0u;
        }
  }
  const uint64_t up2 = pack_f2(up, up);
  auto add = [&](float (&to)[4], const float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) unpack_f2(ffma2(pack_f2(x[i], x[i + 1]), up2, pack_f2(to[i], to[i + 1])), to[i], to[i + 1]);
  };
  uint32_t ps[NB][NT][2], pr[NB][NT][2];                 // weights times scales of a group, and what rounding them has lost
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    uint32_t vw[NB][4];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const uint4 v = *reinterpret_cast<const uint4*>(block + b * Block<D>::kBytes + Block<D>::kV + i * 512 + lane * 16);
      vw[b][0] = v.x; vw[b][1] = v.y; vw[b][2] = v.z; vw[b][3] = v.w;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int u = 4 * i + j, w = u / 2;
      float x[NT][4];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        uint32_t k[4];
        codes_of(vw[b][j], k);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (j % 2 == 0) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const __half2 sc = h2(sv[b][half][w]), prod = PAIR ? __hneg2(__hmul2(h2(minus[b][t][half]), sc)) : __hmul2(h2(p[b][t][half]), sc);
              ps[b][t][half] = u32(prod);
              const __half2 lost = __hfma2(h2(p[b][t][half]), sc, __hneg2(prod));
              pr[b][t][half] = u32(FINE ? __hfma2(h2(rest[b][t][half]), sc, lost) : lost);
            }
          }
          if constexpr (!PAIR) {
            if (b == 0) mma_f16_first(x[t], k[0], k[1], k[2], k[3], ps[b][t][0], ps[b][t][1]);
            else mma_f16(x[t], k[0], k[1], k[2], k[3], ps[b][t][0], ps[b][t][1]);
          }
          if (PAIR && b == 0) mma_f16_first(x[t], k[0], k[1], k[2], k[3], pr[b][t][0], pr[b][t][1]);
          else mma_f16(x[t], k[0], k[1], k[2], k[3], pr[b][t][0], pr[b][t][1]);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) add(h.o[t][u], x[t]);
    }
  }
}

// NB blocks that follow each other, `valid[b]` tokens of each (0: nothing there).  FINE: what rounding the weights to fp16 has lost is added.
// (Several at a time: a block is a chain of products, exponentials and products again that four warps a scheduler do not hide.)
template <int D, int NT, bool PAIR, int NB, bool FINE, Mode MODE>
__device__ __forceinline__ void attend_blocks(Heads<D, NT>& h, const uint8_t* block, const int (&valid)[NB]) {
  float s[NB][NT][4], y[NB][NT][4], most = -INFINITY;
#pragma unroll
  for (int b = 0; b < NB; ++b) scores_of<D, NT, MODE>(h, block + b * Block<D>::kBytes, block + b * Block<D>::kBytes + Block<D>::kScaleK, valid[b], s[b]);
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[b][t][i] = fmaf(s[b][t][i], h.scale[t][i & 1], h.minus[t][i & 1]);
        most = fmaxf(most, y[b][t][i]);
      }
  if (__any_sync(0xffffffffu, most > kMoveAt)) {
    // the references move to the scores' maximum where they are exceeded; sums and outputs follow
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float m = -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b) m = fmaxf(m, fmaxf(s[b][t][i], s[b][t][i + 2]));
        m *= h.scale[t][i];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (m + h.minus[t][i] > kMoveAt) {
          const float alpha = h.minus[t][i] == kNoReference ? 0.f : ex2(kBelow - m - h.minus[t][i]);
          h.minus[t][i] = kBelow - m;
          h.sum[t][i] *= alpha;
#pragma unroll
          for (int u = 0; u < D / 16; ++u) { h.o[t][u][i] *= alpha; h.o[t][u][i + 2] *= alpha; }
          h.om[t][i] *= alpha;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          y[b][t][i] = fmaf(s[b][t][i], h.scale[t][i], h.minus[t][i]);
          y[b][t][i + 2] = fmaf(s[b][t][i + 2], h.scale[t][i], h.minus[t][i]);
        }
      }
  }
  uint32_t p[NB][NT][2], rest[NB][NT][2];                // P^T as an operand: head lane / 4, tokens 2 c, 2 c + 1 and 8 + 2 c, 9 + 2 c
  auto turn = [](uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
  };
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = ex2(y[b][t][i]);
      h.sum[t][0] += e[0] + e[2];
      h.sum[t][1] += e[1] + e[3];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t both = from_float2<__half>(e[2 * i], e[2 * i + 1]);
        p[b][t][i] = turn(both);
        if constexpr (FINE) {
          const float2 f = to_float2<__half>(both);
          rest[b][t][i] = turn(from_float2<__half>(e[2 * i] - f.x, e[2 * i + 1] - f.y));
        }
      }
    }
  add_values<D, NT, PAIR, NB, FINE, MODE>(h, block, valid, p, rest);
}

__device__ __forceinline__ void put(void* out, int kind, size_t at, float x) {
  if (kind == HYPERATTN_BF16) reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(x);
  else if (kind == HYPERATTN_FP16) reinterpret_cast<__half*>(out)[at] = __float2half_rn(x);
  else reinterpret_cast<float*>(out)[at] = x;
}

// warps of a CTA, and CTAs that an SM holds by registers (two tiles of heads need 168 a thread)
constexpr int kWarps = 4;
constexpr int ctas_by_registers(int tiles) { return tiles == 1 ? 4 : 3; }
constexpr int kMaxRequests = 4096;      // running sums in shared memory

// A unit of work and of the ring: 32 (d = 128) or 64 tokens of a segment, 5 KB.
template <int D, Mode MODE>
struct Ring {
  static constexpr int kUnit = (D == 128 ? 2 : 4) * (MODE == kWeights ? 2 : 1);                // blocks (weights: K's half of them)
  static constexpr int kBlockBytes = MODE == kWeights ? 10 * D : Block<D>::kBytes;
  static constexpr int kUnitBytes = kUnit * kBlockBytes, kUnitTokens = kUnit * kBlockTokens;
  static constexpr int kStages = 2;                                      // units on their way, a warp
  static constexpr int kWarpBytes = kStages * kUnitBytes;                // (>= 16 x D floats: a warp's outputs, when the parts are put together)
  static constexpr int kKnown = MODE == kOneQuery ? 1280 : 1536;         // what a warp knows of its next units
  static constexpr int bytes(int requests) { return kWarps * (kWarpBytes + kKnown + kStages * 8 + 4 + 16 * 12) + 16 + (requests + 1) * 4 + (MODE == kOneQuery ? 0 : (requests + 1) * 8); }
};
template <int D, Mode MODE> int ctas_by_memory(int requests) { return 227 * 1024 / (Ring<D, MODE>::bytes(requests) + 1024); }

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Weights: empty units at a segment's end, for what its beginning costs (queries and log-sum-exps, 2.5 to 4 us beside 1 us a unit; without them a warp that had
// requests of a token each was what 64 requests waited for: 64 us).
constexpr int kBegin = 2;
template <int D, Mode MODE> __device__ __forceinline__ int units_of(const CacheAttnArgs& a, int r) {
  const int tokens = min(max(a.lengths[r], 0), a.width * a.cache.page);        // (up to 2^31 - 1)
  const int units = tokens / Ring<D, MODE>::kUnitTokens + (tokens % Ring<D, MODE>::kUnitTokens != 0);
  return MODE == kWeights && units ? units + kBegin : units;
}
// A unit's tokens: what they had, times the decay, and what the request's rows of key head kv give them (in chunks; nearly always one).  A lane ends up with the two tokens
// lane / 4 (+ 8) of blocks c, c + 4, ...; wait(): until the unit's keys are there.
template <int D, int NT, class T, class W>
__device__ __forceinline__ void weigh_unit(Heads<D, NT>& h, const CacheAttnArgs& a, const uint8_t* unit, int request, int kv, int chunks, int first, int left, int there, int2 queries, bool fresh, W wait) {
  constexpr int U = Ring<D, kWeights>::kUnit, MINE = U / 4;
  const int lane = threadIdx.x & 31, c = lane & 3, cap = a.width * a.cache.page;
  const int len = first + left, old = len - queries.y;                   // tokens from `old` on are the rows' own
  const size_t at = ((size_t)request * a.cache.heads + kv) * cap;
  float had[MINE][2], got[MINE][2];
#pragma unroll
  for (int k = 0; k < MINE; ++k)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int token = first + (4 * k + c) * kBlockTokens + lane / 4 + 8 * e;
      had[k][e] = a.before && token < old ? a.before[at + token] : 0.f;
      got[k][e] = 0.f;
    }
  // (a segment's first unit: its queries, beside what the tokens had)
  if (fresh) load_heads<D, NT, false, T, kWeights>(h, a, request, 0, min(queries.y * group_of(a), 8 * NT), kv, queries);
  if (!wait()) return;
  for (int chunk = 0; chunk < chunks; ++chunk) {
    if (chunks > 1 && !(chunk == 0 && fresh)) load_heads<D, NT, false, T, kWeights>(h, a, request, chunk * 8 * NT, min(queries.y * group_of(a) - chunk * 8 * NT, 8 * NT), kv, queries);
#pragma unroll
    for (int b4 = 0; b4 < U; b4 += 4) {
      // four blocks; two at a time where they are there, so that one's products cover the other's latencies
      float sum[4][2];
      auto block = [&](int i) {
        float s[NT][4];
        scores_of<D, NT, kWeights>(h, unit + (b4 + i) * 8 * D, unit + U * 8 * D + (b4 + i) * 2 * D, left - (b4 + i) * kBlockTokens, s);
        sum[i][0] = sum[i][1] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < 4; ++k) sum[i][k >> 1] += ex2(fmaf(s[t][k], h.scale[t][k & 1], h.minus[t][k & 1]));
      };
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const int two = there >> (b4 + i) & 3;
        if (two == 3) { block(i); block(i + 1); }
        else {
#pragma unroll
          for (int k = i; k < i + 2; ++k) {
            if (there >> (b4 + k) & 1) block(k);
            else sum[k][0] = sum[k][1] = 0.f;
          }
        }
      }
      // over the four lanes of a token: each ends up with one block's
      const bool b0 = c & 1, b1 = c & 2;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float x = (b0 ? sum[1][e] : sum[0][e]) + __shfl_xor_sync(0xffffffffu, b0 ? sum[0][e] : sum[1][e], 1);
        const float y = (b0 ? sum[3][e] : sum[2][e]) + __shfl_xor_sync(0xffffffffu, b0 ? sum[2][e] : sum[3][e], 1);
        got[b4 / 4][e] += (b1 ? y : x) + __shfl_xor_sync(0xffffffffu, b1 ? x : y, 2);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < MINE; ++k)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int token = first + (4 * k + c) * kBlockTokens + lane / 4 + 8 * e;
      if (token < cap) a.weights[at + token] = token < len ? (token < old ? a.decay * had[k][e] : 0.f) + got[k][e] : 0.f;
    }
}
// where the pieces of a segment lie: see combine
__device__ __forceinline__ float* piece_at(const CacheAttnArgs& a, long long slot, int head, int d) { return a.part + (slot * a.part_heads + head) * (d + 2); }

// FINE: what rounding the weights to fp16 has lost enters too (fp16 queries; some rows: also fp32 results, which would show it)
template <int D, int NT, bool PAIR, class T, Mode MODE, bool FINE = std::is_same<T, __half>::value>
__global__ void __launch_bounds__(32 * kWarps, ctas_by_registers(NT)) cache_attn_kernel(const __grid_constant__ KernelArgs<MODE> a, int* status) {
  using R = Ring<D, MODE>;
  constexpr int kPerChunk = PAIR ? 4 : 8 * NT;                           // rows (heads) of a chunk
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* misc = smem + kWarps * (R::kWarpBytes + R::kKnown + R::kStages * 8);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc);
  int* s_sums = reinterpret_cast<int*>(misc + 16);                       // [kWarps]
  float* s_stat = reinterpret_cast<float*>(s_sums + kWarps);             // [kWarps][16][2] references, sums
  float* s_factor = s_stat + kWarps * 32;                                // [kWarps][16]
  int* s_starts = reinterpret_cast<int*>(s_factor + kWarps * 16);        // [requests + 1] units (of one segment each; some rows: of one key head) before a request
  int2* s_queries = reinterpret_cast<int2*>(s_starts + (a.requests + 2) / 2 * 2);               // some rows, weights: [requests] a request's queries: first row, how many
  auto chunks_of = [&](int r) { return (s_queries[r].y * group_of(a) + kPerChunk - 1) / kPerChunk; };
  const int tid = threadIdx.x, lane = tid & 31, c = lane & 3;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t ring = smem_u32(smem) + warp * R::kWarpBytes, bars = smem_u32(smem) + kWarps * (R::kWarpBytes + R::kKnown) + warp * R::kStages * 8;
  if (tid == 0) *s_abort = 0;
  if (lane == 0) {
    for (int st = 0; st < R::kStages; ++st) mbar_init(bars + 8 * st, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  wait_for_stream();
  // ---- running sum of the requests' units ----
  const int per = (a.requests + 32 * kWarps - 1) / (32 * kWarps), r0 = min(a.requests, tid * per), r1 = min(a.requests, r0 + per);
  int mine = 0;
  for (int r = r0; r < r1; ++r) {
    s_starts[r] = mine;
    int units = units_of<D, MODE>(a, r);
    if constexpr (MODE != kOneQuery) {
      s_queries[r] = queries_of(a, r);
      if (s_queries[r].y < 0) { s_queries[r].y = 0; units = 0; }
      if (MODE == kSomeRows) units *= chunks_of(r);
    }
    if constexpr (MODE == kSomeRows) mine = plus(mine, units);
    else mine += units;
  }
  int run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run = MODE == kSomeRows ? plus(run, y) : run + y; }
  if (lane == 31) s_sums[warp] = run;
  __syncthreads();
  run -= mine;
  for (int w = 0; w < warp; ++w) run = MODE == kSomeRows ? plus(run, s_sums[w]) : run + s_sums[w];
  for (int r = r0; r < r1; ++r) s_starts[r] = MODE == kSomeRows ? plus(s_starts[r], run) : s_starts[r] + run;
  if (tid == 32 * kWarps - 1) s_starts[a.requests] = MODE == kSomeRows ? plus(run, mine) : run + mine;
  __syncthreads();
  if constexpr (MODE == kWeights) blank(a.weights, a.lengths, a.requests, a.cache.heads, a.width * a.cache.page, R::kUnitTokens, blockIdx.x, gridDim.x);
  const int segs = a.cache.heads * (MODE == kOneQuery ? a.chunks : 1);   // of a request (some rows: key heads, of which each has the request's chunks)
  if constexpr (MODE == kSomeRows) {                                     // (offsets that do not ascend may ask for more units than a number holds: none then)
    const bool many = s_starts[a.requests] > 0x7fffffff / segs;
    __syncthreads();
    if (many)
      for (int r = tid; r <= a.requests; r += 32 * kWarps) s_starts[r] = 0;
    __syncthreads();
  }
  const int total = s_starts[a.requests] * segs, warps = gridDim.x * kWarps, part = max(1, total / warps + (total % warps != 0));
  if (MODE != kWeights && blockIdx.x == 0) {
    for (int r = tid; r <= a.requests; r += 32 * kWarps) a.starts[r] = s_starts[r];
    if (tid == 0) a.starts[a.requests + 1] = part;
  }
  const int cta_first = (int)min((long long)blockIdx.x * kWarps * part, (long long)total), cta_end = (int)min((long long)cta_first + kWarps * part, (long long)total);
  const int first = (int)min((long long)cta_first + warp * part, (long long)total), end = (int)min((long long)first + part, (long long)total);
  const int count = end - first;                                         // units of this warp
  const int subs = a.cache.page / kBlockTokens, per_kv = a.q_heads / a.cache.heads;

  // What is known of the blocks of the next 32 / kUnit units, a lane a block, in shared memory (a batch while another is used): first, by look(), where to
  // look - {segment of all requests', block in it, page, length} and the block's place in its page, page and length on their way - and then, by know(),
  // what is there: {segment, tokens from the unit on, block of the cache, bytes of the copy to ask for | blocks of the unit that exist << 16}.  A unit that
  // cannot leave its page is one copy, its first block's.
  // NB blocks at a time.  One tile of heads, fp16: four at d = 64 (2 x 131072 tokens, 32 / 32 heads: 150 us; two 153, one 160), two at d = 128 (16 x 32768, 8 / 8: 75; one 77).
  // bf16, whose blocks are less work: half of that (64, 32 / 8: 39, with four, which spill, 41; 128, 64 requests: 66, two 68).  Two tiles: two (36 / 4 heads of 64: 33.9,
  // four, which spill, 35.6; 32 / 2 of 128: 34.7, one 35.8).
  constexpr int U = R::kUnit, kBatch = 32 / U, NB = NT == 2 ? 2 : (D == 64 ? 2 : 1) * (FINE ? 2 : 1);
  const bool whole = subs % U == 0;
  const int shift = subs & (subs - 1) ? -1 : 31 - __clz(subs);           // blocks of a page: a power of two?
  int4* s_known = reinterpret_cast<int4*>(smem + kWarps * R::kWarpBytes) + warp * 64;                       // [2][32]
  int* s_place = reinterpret_cast<int*>(smem + kWarps * (R::kWarpBytes + 1024)) + warp * 64;                // [2][32]
  int* s_request = reinterpret_cast<int*>(smem + kWarps * (R::kWarpBytes + 1280)) + warp * 64;              // some rows, weights: [2][32], the segment is then that of the request
  auto look = [&](int unit) {                                            // units unit .. unit + kBatch - 1
    const int slot = (unit / kBatch & 1) * 32 + lane, i = min(unit + lane / U, count - 1);
    const int n = first + i;
    int lo = 0, hi = a.requests;                                         // the last request whose units start there or before
    const int t = n / segs;
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (s_starts[mid] <= t) lo = mid; else hi = mid; }
    int units = s_starts[lo + 1] - s_starts[lo];
    const int chunks = MODE == kOneQuery ? a.chunks : MODE == kSomeRows ? chunks_of(lo) : 1;
    if constexpr (MODE == kSomeRows) units /= chunks;
    const int rest = n - s_starts[lo] * segs, seg = rest / units, b = (rest - seg * units) * U + lane % U;
    const int column = shift >= 0 ? b >> shift : b / subs;
    *reinterpret_cast<int2*>(&s_known[slot]) = make_int2(MODE == kOneQuery ? lo * segs + seg : seg, b);
    if constexpr (MODE != kOneQuery) s_request[slot] = lo;
    s_place[slot] = (chunks == 1 ? seg : seg / chunks) * subs + b - column * subs;
    const uint32_t to = smem_u32(&s_known[slot]);
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n\tcp.async.ca.shared.global [%2], [%3], 4;" ::"r"(to + 8), "l"(a.table + (size_t)lo * a.width + min(column, a.width - 1)), "r"(to + 12),
                 "l"(a.lengths + lo) : "memory");
  };
  auto know = [&](int unit) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    const int slot = (unit / kBatch & 1) * 32 + lane, in_unit = lane % U;
    const int4 k = s_known[slot];
    const int left = min(k.w, a.width * a.cache.page) - (k.y - in_unit) * kBlockTokens;
    const bool there = in_unit * kBlockTokens < left && k.z >= 0 && k.z < a.cache.num_pages;
    const unsigned all = __ballot_sync(0xffffffffu, there) >> (lane - in_unit) & ((1u << U) - 1);
    const int bytes = whole ? (in_unit == 0 ? __popc(all) : 0) : there;
    s_known[slot] = make_int4(k.x, left, k.z * a.cache.heads * subs + s_place[slot], bytes * Block<D>::kBytes | all << 16);
    if constexpr (MODE == kWeights) s_place[slot] = k.y * kBlockTokens;   // (weights: from here on the block's first token)
    __syncwarp();
  };
  int asked = 0;                                                         // units whose copies have been asked for
  auto ask = [&] {
    if constexpr (MODE == kWeights) {                                    // the unit's codes, then its scales; a run of blocks is in one page and comes as a whole
      if (lane < U) {
        const int st = asked % R::kStages;
        const uint32_t bar = bars + 8 * st;
        const int4 k = s_known[asked % (2 * kBatch) * U + lane];
        const uint32_t leaders = a.run == 1 ? 0xffu : a.run == 2 ? 0x55u : a.run == 4 ? 0x11u : 0x01u;
        if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(__popc(k.w >> 16 & leaders) * a.run * R::kBlockBytes) : "memory");
        if ((leaders >> lane & 1) && (k.w >> 16 >> lane & 1)) {
          const uint32_t to = ring + st * R::kUnitBytes;
          tma_tile(to + lane * 8 * D, &a.maps.codes, 0, k.z, bar);
          tma_tile(to + U * 8 * D + lane * 2 * D, &a.maps.scales, 4 * D, k.z, bar);
        }
      }
    } else if (lane < U) {
      const int st = asked % R::kStages;
      const uint32_t bar = bars + 8 * st;
      const int4 k = s_known[asked % (2 * kBatch) * U + lane];
      if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(__popc(k.w >> 16) * Block<D>::kBytes) : "memory");
      if (k.w & 0xffff) bulk_copy(ring + st * R::kUnitBytes + lane * Block<D>::kBytes, a.cache.pages + (size_t)k.z * Block<D>::kBytes, k.w & 0xffff, bar);
    }
    ++asked;
  };
  bool ok = true;
  Heads<D, NT> h;
  int segment = -1, request = -1, seg = 0, chunks = a.chunks;            // segment = request * segs + seg; some rows, weights: the request's
  int2 queries = make_int2(0, 0);
  auto take_segment = [&](int sg, int rq) {
    segment = sg;
    if constexpr (MODE == kOneQuery) {
      request = segment / segs; seg = segment - request * segs;
      const int kv = seg / a.chunks, chunk = seg - kv * a.chunks;
      load_heads<D, NT, PAIR, T, MODE>(h, a, request, kv * per_kv + chunk * 8 * NT, min(per_kv - chunk * 8 * NT, 8 * NT), kv, queries);
    } else {
      request = rq; seg = sg;
      queries = s_queries[request];
      chunks = MODE == kSomeRows ? chunks_of(request) : 1;
      const int kv = seg / chunks, chunk = seg - kv * chunks;
      load_heads<D, NT, PAIR, T, MODE>(h, a, request, chunk * kPerChunk, min(queries.y * per_kv - chunk * kPerChunk, kPerChunk), kv, queries);
    }
  };
  if (count > 0) {
    look(0);
    __syncwarp();
    take_segment(s_known[0].x, MODE == kOneQuery ? 0 : s_request[0]);     // (beside the table's and the lengths' loads)
    know(0);
  }
  while (asked < R::kStages && asked < count) ask();
  // the segment's results, or a piece of them
  auto flush = [&](float* to) {                                            // to: null for final results
    const int chunk = seg % chunks, kv = seg / chunks, first_head = MODE == kOneQuery ? kv * per_kv + chunk * 8 * NT : chunk * kPerChunk;
    const int heads = MODE == kOneQuery ? min(per_kv - chunk * 8 * NT, 8 * NT) : min(queries.y * per_kv - first_head, kPerChunk);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float sum = h.sum[t][i];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float ref = h.minus[t][i] == kNoReference ? -INFINITY : -h.minus[t][i];
        float om[D / kGroup];
#pragma unroll
        for (int w = 0; w < D / kGroup; ++w) om[w] = __shfl_sync(0xffffffffu, h.om[t][i], 4 * w + c);
        const int head = 8 * t + 2 * c + i;
        if (head < heads) {
          size_t row = (size_t)request * a.q_heads + first_head + head;
          if constexpr (MODE != kOneQuery) {
            const int token = (first_head + head) / per_kv;
            row = (size_t)(queries.x + token) * a.q_heads + kv * per_kv + first_head + head - token * per_kv;
          }
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
              const float v = fmaf(h.o[t][m][i + 2 * up], up ? kTwo20 : kTwo24, om[m / 2]);
              if (to) to[head * (D + 2) + x] = v;
              else put(a.out, a.out_kind, row * D + x, v * inv);
            }
        }
      }
  };
  bool together = false;                                                 // the whole CTA works for one segment
  for (int n = 0; n < count; ++n) {
    if (n % kBatch == 0 && n + kBatch < count) look(n + kBatch);
    if (n % kBatch == kBatch / 2 && n + kBatch / 2 < count) know(n + kBatch / 2);
    const int4 unit = s_known[n % (2 * kBatch) * U];
    const int sg = unit.x, left = unit.y, there = unit.w >> 16;
    const int rq = MODE == kOneQuery ? 0 : s_request[n % (2 * kBatch) * U];
    if (MODE == kWeights && left <= 0) {                                  // (an empty unit: no copy was asked for)
      if (asked < count) ask();
      continue;
    }
    const bool fresh = sg != segment || (MODE != kOneQuery && rq != request);
    if (MODE != kWeights && fresh) take_segment(sg, rq);
    const int st = n % R::kStages;
    if constexpr (MODE == kWeights) {
      segment = seg = sg;
      request = rq;
      queries = s_queries[rq];
      weigh_unit<D, NT, T>(h, a, smem + warp * R::kWarpBytes + st * R::kUnitBytes, request, seg, chunks_of(request), s_place[n % (2 * kBatch) * U], left, there, queries, fresh, [&] {
        ok = warp_wait<12>(bars + 8 * st, (uint32_t)(n / R::kStages) & 1, s_abort, status);
        return ok;
      });
      if (!ok) break;
      __syncwarp();
      if (asked < count) ask();
      continue;
    }
    ok = warp_wait<12>(bars + 8 * st, (uint32_t)(n / R::kStages) & 1, s_abort, status);
    if (!ok) break;
#pragma unroll 1
    for (int b = 0; b < U; b += NB) {
      // (a block that is not there: whatever its place holds, no token of it)
      int valid[NB];
#pragma unroll
      for (int i = 0; i < NB; ++i) valid[i] = (there >> (b + i)) & 1 ? left - (b + i) * kBlockTokens : 0;
      if ((there >> b) & ((1 << NB) - 1)) attend_blocks<D, NT, PAIR, NB, FINE, MODE>(h, smem + warp * R::kWarpBytes + st * R::kUnitBytes + b * Block<D>::kBytes, valid);
    }
    __syncwarp();
    if (asked < count) ask();
    if (left <= R::kUnitTokens || n + 1 == count) {                        // the segment's last unit, or the part's
      if constexpr (PAIR) {                                                // what columns 4 .. 7 have belongs to heads 0 .. 3
#pragma unroll
        for (int u = 0; u < D / 16; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) h.o[0][u][i] += __shfl_xor_sync(0xffffffffu, h.o[0][u][i], 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) h.om[0][i] += __shfl_xor_sync(0xffffffffu, h.om[0][i], 2);
      }
      int units = s_starts[request + 1] - s_starts[request];
      if constexpr (MODE == kSomeRows) units /= chunks;
      const int seg_first = s_starts[request] * segs + seg * units, seg_end = seg_first + units;
      if (seg_first >= first && seg_end <= end) flush(nullptr);
      else {
        together = seg_first <= cta_first && seg_end >= cta_end;
        if (!together) flush(piece_at(a, 2 * ((long long)blockIdx.x * kWarps + warp) + (seg_first < first ? 0 : 1), 0, D));
      }
    }
  }
  if (!ok)                                                               // nothing may be on its way into shared memory when the CTA ends
    for (int st = 0; st < R::kStages && st < asked; ++st) mbar_drain(bars + 8 * st, (uint32_t)((asked - 1 - st) / R::kStages) & 1);
  if constexpr (MODE == kWeights) return;
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
            for (int up = 0; up < 2; ++up) s_o[head * D + 16 * m + lane / 4 + 8 * up] = fmaf(h.o[t][m][i + 2 * up], up ? kTwo20 : kTwo24, __shfl_sync(0xffffffffu, h.om[t][i], 4 * (m / 2) + c));
        }
    }
    __syncthreads();
    const int used = (cta_end - cta_first + part - 1) / part;            // warps that have a part: all of them are together
    float* piece = piece_at(a, 2ll * blockIdx.x * kWarps, 0, D);
    if (tid < 8 * NT) {
      float ref = -INFINITY, sum = 0.f;
      for (int w = 0; w < used; ++w) ref = fmaxf(ref, s_stat[(w * 16 + tid) * 2]);
      for (int w = 0; w < used; ++w) {
        const float rw = s_stat[(w * 16 + tid) * 2], sw = s_stat[(w * 16 + tid) * 2 + 1];
        const float f = rw == -INFINITY ? (sw == 0.f ? 0.f : 1.f) : ex2(rw - ref);            // (a sum without a reference: NaN)
        s_factor[w * 16 + tid] = f;
        sum += f * sw;
      }
      if (tid < a.part_heads) { piece[tid * (D + 2) + D] = ref; piece[tid * (D + 2) + D + 1] = sum; }
    }
    __syncthreads();
    for (int i = tid; i < a.part_heads * (D / 4); i += 32 * kWarps) {    // (of a chunk with fewer heads the others are not read)
      const int head = i / (D / 4), x = i - head * (D / 4);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < used; ++w) {
        const float f = s_factor[w * 16 + head];
        const float4 v = reinterpret_cast<const float4*>(smem + w * R::kWarpBytes)[i];
        o = make_float4(o.x + f * v.x, o.y + f * v.y, o.z + f * v.z, o.w + f * v.w);
      }
      float2* to = reinterpret_cast<float2*>(piece + head * (D + 2) + 4 * x);
      to[0] = make_float2(o.x, o.y); to[1] = make_float2(o.z, o.w);
    }
  }
}

// Puts the pieces of segments together that lie in several parts; requests without tokens get their zeros.
constexpr int kJoinThreads = 128;

template <int D, Mode MODE>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ CacheAttnArgs a, int heads_per_cta) {
  constexpr int LANES = D / 4, ROWS = kJoinThreads / LANES;               // a thread: four coordinates of every ROWS-th piece
  __shared__ float4 s_o[ROWS][LANES];
  __shared__ float s_ref[ROWS], s_sum[ROWS];
  wait_for_stream();
  const int per_kv = a.q_heads / a.cache.heads;
  int segs, r, seg, kv, first_head, heads, first_query = 0, chunks = 1;
  if constexpr (MODE == kOneQuery) {
    segs = a.cache.heads * a.chunks;
    r = blockIdx.x / segs; seg = blockIdx.x - r * segs; kv = seg / a.chunks;
    const int chunk = seg - kv * a.chunks;
    first_head = kv * per_kv + chunk * a.part_heads; heads = min(per_kv - chunk * a.part_heads, a.part_heads);
  } else {
    // which request has the chunk (of all) that this CTA is for
    __shared__ int s_found;
    segs = a.cache.heads;
    const int slot = blockIdx.x / segs;
    kv = blockIdx.x - slot * segs;
    if (threadIdx.x == 0) s_found = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < a.requests; i += kJoinThreads) {
      const int2 q = queries_of(a, i);
      const long long first = chunk_slots(q.x, i, per_kv, a.part_heads);
      const int n = (max(q.y, 0) * per_kv + a.part_heads - 1) / a.part_heads;
      if (slot >= first && slot < first + n) atomicMax(&s_found, i);      // (one of them, if offsets that do not ascend give a chunk to several)
    }
    __syncthreads();
    r = s_found;
    if (r < 0) return;
    const int2 q = queries_of(a, r);
    const int chunk = (int)(slot - chunk_slots(q.x, r, per_kv, a.part_heads));
    first_query = q.x;
    first_head = chunk * a.part_heads;
    heads = min(q.y * per_kv - first_head, a.part_heads);
    chunks = (q.y * per_kv + a.part_heads - 1) / a.part_heads;
    seg = kv * chunks + chunk;
  }
  auto row_of = [&](int head) {
    if constexpr (MODE == kOneQuery) return (size_t)r * a.q_heads + first_head + head;
    const int token = (first_head + head) / per_kv;
    return (size_t)(first_query + token) * a.q_heads + kv * per_kv + first_head + head - token * per_kv;
  };
  const int part = a.starts[a.requests + 1], before = a.starts[r], units = (a.starts[r + 1] - before) / chunks, total = a.starts[a.requests] * segs;
  const int begin = before * segs + seg * units, end = begin + units;
  const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES;
  const int h0 = blockIdx.y * heads_per_cta, h1 = min(h0 + heads_per_cta, heads);
  if (units == 0) {
    for (int i = threadIdx.x; i < (h1 - h0) * D; i += kJoinThreads) put(a.out, a.out_kind, row_of(h0 + i / D) * D + i % D, 0.f);
    for (int i = h0 + threadIdx.x; i < h1; i += kJoinThreads) a.lse[row_of(i)] = -INFINITY;
    return;
  }
  const int w0 = begin / part, w1 = (end - 1) / part;                     // warps that have a part of it
  if (w0 == w1) return;                                                   // finished there
  // Its pieces in order: those of the first CTA's warps (or its one), one of every CTA inside, those of the last CTA's warps (or its one)
  const int c0 = w0 / kWarps, c1 = w1 / kWarps;
  auto whole = [&](int cta) { return (long long)cta * kWarps * part >= begin && min((long long)(cta + 1) * kWarps * part, (long long)total) <= end; };
  const bool whole0 = whole(c0), whole1 = whole(c1);
  const int n0 = whole0 ? 1 : min(w1, c0 * kWarps + kWarps - 1) - w0 + 1;
  const int n1 = c1 == c0 ? 0 : whole1 ? 1 : w1 - c1 * kWarps + 1;
  const int inside = c1 > c0 ? c1 - c0 - 1 : 0, count = n0 + inside + n1;
  auto slot_of = [&](int i) {
    int w;
    if (i < n0) { if (whole0) return 2ll * c0 * kWarps; w = w0 + i; }
    else if (i < n0 + inside) return 2ll * (c0 + 1 + i - n0) * kWarps;
    else { if (whole1) return 2ll * c1 * kWarps; w = c1 * kWarps + (i - n0 - inside); }
    return 2ll * w + (begin < (long long)w * part ? 0 : 1);
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
      const size_t at = row_of(head);
      const float v[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
#pragma unroll
      for (int i = 0; i < 4; ++i) put(a.out, a.out_kind, at * D + 4 * lane + i, v[i]);
      if (lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
    }
    __syncthreads();
  }
}

}  // namespace
}  // namespace hyperattn
