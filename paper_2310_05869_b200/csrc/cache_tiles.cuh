// What the tcgen05 kernels over the paged 4-bit cache have in common: requests' rows and tokens, queries as operands, keys as operands, parts of the work.
//
// Scores are exact products: a key is minimum + scale * code, and
//   <q, k> = sum_g ( sum_x q_x (scale_g code_x) + minimum_g sum_x q_x ),
// where scale * code has 15 bits, which two fp16 numbers hold (the product rounded, and what the rounding has lost), the minimum is an fp16 number, and the sum of a group's
// queries is three.  Queries are fp16 numbers after a power of two for their row, scales and minima after one for their token (or tile), so the fp32 sums of the tensor cores are all
// that is rounded.  (Keys rounded to 16 bits would be half the products, and scores off by 2e-4: weights and log-sum-exps are fp32 results, which show it.)
#pragma once
#include <climits>
#include "serving.cuh"
#include "tc_util.cuh"

namespace hyperattn {
namespace {

struct ChunkArgs {
  CacheView cache;
  const void* q;
  long long q_row, q_head;
  const int32_t *table, *lengths, *cu_q;
  int requests, rows, width, q_heads, causal, least;      // least: requests of so few rows are not for this launch (-1: all are)
  float scale_log2;
  uint8_t* images;                       // queries as operands, see Image
};
struct Span {                            // a request's query rows and tokens
  int first, rows, len;
};
__device__ __forceinline__ Span span_of(const ChunkArgs& a, int r) {
  Span s;
  s.first = a.cu_q ? min(max(a.cu_q[r], 0), a.rows) : r;
  s.rows = a.cu_q ? min(max(a.cu_q[r + 1], s.first), a.rows) - s.first : 1;
  s.len = min(max(a.lengths[r], 0), a.width * a.cache.page);
  return s;
}

__device__ __forceinline__ bool is_for(const ChunkArgs& a, const Span& s) { return s.rows * (a.q_heads / a.cache.heads) > a.least; }

// ---- queries ---------------------------------------------------------------------------------------------------------------
// A request's rows of a key head are its tokens times the head's query heads.  NR of them, as shared memory holds them: fp16 [NR x d] with the 128-byte swizzle in slabs of 64
// columns; sums of the groups [2][NR][8] (high parts, what those lack, what is still missing, zeros); minus the rows' log-sum-exps (to base 2); their factors to base-2 scores;
// and the factor of all rows, if they have one (0: they do not).  Rows that do not exist are zeros (minus infinity).
template <int D, int NR>
struct Image {
  static constexpr uint32_t kSlab = NR * 128, kSums = NR * 2 * D, kMinus = kSums + NR * 32, kFactors = kMinus + NR * 4, kFactor = kFactors + NR * 4, kBytes = (kFactor + 4 + 1023) / 1024 * 1024;
};
constexpr int kSpread = 12;              // octaves that a row may be smaller than the image's largest and have its factor: 2^-21 of its largest entry are still whole steps
// The images of a request come after those of the ones before it, wherever those end: one for each request before is room for what its last one does not fill.  Requests of up to `least` rows have
// none; so no more than a request for every least + 1 rows needs that room (1024 places of a server with a part of a prompt or two: some tens of megabytes instead of 745).
__host__ __device__ __forceinline__ long long image_slots(long long rows_before, int requests_before, int group, int nr, int least) {
  const long long rows = rows_before * group, most = least < 0 ? requests_before : rows / (least + 1);
  return rows / nr + (most < requests_before ? most : requests_before);
}

template <int D, int NR, class T>
__global__ void __launch_bounds__(128) image_kernel(const __grid_constant__ ChunkArgs a, const float* lse, int images, float* out, int unit) {
  constexpr int LANES = D / 8, AT_ONCE = 128 / LANES, G = D / kGroup;
  using I = Image<D, NR>;
  wait_for_stream();
  if ((int)blockIdx.x >= images) {                     // the others: zeros beyond the requests' tokens
    blank(out, a.lengths, a.requests, a.cache.heads, a.width * a.cache.page, unit, blockIdx.x - images, gridDim.x - images);
    return;
  }
  const int kv = blockIdx.x % a.cache.heads, group = a.q_heads / a.cache.heads;
  const long long slot = blockIdx.x / a.cache.heads;
  int lo = 0, hi = a.requests;                         // the last request whose images start there or before
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (image_slots(span_of(a, mid).first, mid, group, NR, a.least) <= slot) lo = mid; else hi = mid;
  }
  const Span s = span_of(a, lo);
  const long long row0 = (slot - image_slots(s.first, lo, group, NR, a.least)) * NR, rows = (long long)s.rows * group;
  if (row0 < 0 || row0 >= rows || !is_for(a, s)) return;
  uint8_t* to = a.images + (size_t)blockIdx.x * I::kBytes;
  __shared__ int s_exp[NR], s_most, s_apart;
  if (threadIdx.x == 0) { s_most = INT_MIN; s_apart = 0; }
  const int c = threadIdx.x % LANES;
  auto query = [&](int i) {
    if (row0 + i >= rows) return make_uint4(0, 0, 0, 0);
    const int row = s.first + (int)((row0 + i) / group), head = kv * group + (int)((row0 + i) % group);
    return *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(a.q) + (long long)row * a.q_row + (long long)head * a.q_head + 8 * c);
  };
  // The rows' exponents.  A row is multiplied by 2^(9 - e), e the exponent of its largest entry (then a group's sum is an fp16 number, and entries 2^-33 of the largest are whole
  // steps) - or of the image's largest, if it is not much smaller, so that all have one factor.
  __syncthreads();
#pragma unroll 4
  for (int i = threadIdx.x / LANES; i < NR; i += AT_ONCE) {
    const uint4 raw = query(i);
    const uint32_t v[4] = {raw.x, raw.y, raw.z, raw.w};
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) { const float2 f = to_float2<T>(v[k]); top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y))); }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int e = top == 0.f || !(top < INFINITY) ? INT_MIN : min(max((int)(__float_as_uint(top) >> 23) - 127 - 9, -126), 126);      // (0, and what is not finite: any will do)
    if (c == 0) {
      s_exp[i] = e;
      if (e != INT_MIN) atomicMax(&s_most, e);
    }
  }
  __syncthreads();
  const int most = s_most == INT_MIN ? 0 : s_most;
#pragma unroll 2
  for (int i = threadIdx.x / LANES; i < NR; i += AT_ONCE) {
    const bool there = row0 + i < rows;
    const int row = s.first + (int)((row0 + i) / group), head = kv * group + (int)((row0 + i) % group);
    const uint4 raw = query(i);
    const uint32_t v[4] = {raw.x, raw.y, raw.z, raw.w};
    const int own = s_exp[i], e = own == INT_MIN || most - own <= kSpread ? most : own;
    if (c == 0 && e != most) s_apart = 1;
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[4];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 f = to_float2<T>(v[k]);
      w[k] = from_float2<__half>(f.x * down, f.y * down);
      const float2 r = to_float2<__half>(w[k]);
      sum += r.x + r.y;
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    *reinterpret_cast<uint4*>(to + (c >> 3) * I::kSlab + i * 128 + (((c & 7) ^ (i & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    // lane 4 g of the row has group g's sum
    float part[3];
    part[0] = __half2float(__float2half_rn(sum));
    part[1] = __half2float(__float2half_rn(sum - part[0]));
    part[2] = sum - part[0] - part[1];
    float all[3][G];
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int g = 0; g < G; ++g) all[p][g] = __shfl_sync(0xffffffffu, part[p], 4 * g, LANES);
    uint32_t sums[8] = {};
#pragma unroll
    for (int p = 0; p < 3; ++p)
#pragma unroll
      for (int g = 0; g < G; g += 2) sums[(p * G + g) / 2] = from_float2<__half>(all[p][g], all[p][g + 1]);
    if (c == 0) {
      *reinterpret_cast<uint4*>(to + I::kSums + i * 16) = make_uint4(sums[0], sums[1], sums[2], sums[3]);
      *reinterpret_cast<uint4*>(to + I::kSums + (NR + i) * 16) = make_uint4(sums[4], sums[5], sums[6], sums[7]);
      const float l = there ? lse[(size_t)row * a.q_heads + head] : -INFINITY;
      reinterpret_cast<float*>(to + I::kMinus)[i] = l == -INFINITY ? l : -l * 1.4426950408889634f;           // (a row that saw nothing gives nothing)
      reinterpret_cast<float*>(to + I::kFactors)[i] = __uint_as_float((uint32_t)(127 + e) << 23) * a.scale_log2;
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) *reinterpret_cast<float*>(to + I::kFactor) = s_apart ? 0.f : __uint_as_float((uint32_t)(127 + most) << 23) * a.scale_log2;
}

// ---- keys ------------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ __half2 as_half2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }
__device__ __forceinline__ uint32_t as_u32(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
// The codes of a word (8 of them, k at bit 4 k) as fp16 pairs (k, k + 4): 1024 + c, or 1024 + 16 c, is c in the lowest bits of 1024
__device__ __forceinline__ void half_codes(uint32_t w, uint32_t (&k)[4]) {
  const uint32_t up = w >> 8, magic = 0x64006400u;
  const __half2 minus = as_half2(0xe400e400u), minus64 = as_half2(0xd400d400u), sixteenth = as_half2(0x2c002c00u);      // -1024, -64, 1 / 16
  k[0] = as_u32(__hadd2(as_half2((w & 0x000f000fu) | magic), minus));
  k[1] = as_u32(__hfma2(as_half2((w & 0x00f000f0u) | magic), sixteenth, minus64));
  k[2] = as_u32(__hadd2(as_half2((up & 0x000f000fu) | magic), minus));
  k[3] = as_u32(__hfma2(as_half2((up & 0x00f000f0u) | magic), sixteenth, minus64));
}
// Of scales and minima (pairs of fp16 numbers) the exponent t so that all numbers they stand for are below 2^(t - 14): the bits' largest exponents, a scale's + 4; what is
// not finite does not count.
__device__ __forceinline__ int exponent_of(uint32_t scales, uint32_t minima) {
  auto of = [](uint32_t h) { const int e = (int)(h >> 10 & 31u); return e == 31 ? 0 : e; };
  return max(max(of(scales), of(scales >> 16)) + 4, max(of(minima), of(minima >> 16)));
}
// The power of two (its exponent) that brings such numbers below 2^15, 2^15 at most
__device__ __forceinline__ int lift_of(int exponent) { return min(29 - exponent, 15); }
__device__ __forceinline__ __half2 lift2(int lift) { return __half2half2(__ushort_as_half((unsigned short)((lift + 15) << 10))); }

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// K of the lane's token as an A operand in TMEM, a lane a token: scale * code [d / 2 columns], what its rounding has lost [d / 2], minima [8].  codes, scales: of the token's block (in
// shared memory).  Returns the factor that the scores are to be multiplied with.
template <int D>
struct KeyCols { static constexpr uint32_t kRest = D / 2, kMinima = D, kAll = D + 8; };
template <int D>
__device__ __forceinline__ float keys_to_tmem(uint32_t col, const uint8_t* codes, const uint8_t* scales, int t, bool there) {
  constexpr int G = D / kGroup;
  uint32_t cw[4][G];                                   // [octet][group]
#pragma unroll
  for (int o = 0; o < 4; ++o) {
    if constexpr (D == 128) {
      const uint4 v = *reinterpret_cast<const uint4*>(codes + t / 8 * 512 + (t % 8 * 4 + o) * 16);
      cw[o][0] = v.x; cw[o][1] = v.y; cw[o][2] = v.z; cw[o][3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(codes + (t % 8 * 4 + o) * 16 + t / 8 * 8);
      cw[o][0] = v.x; cw[o][1] = v.y;
    }
  }
  const uint32_t same = t & 1 ? 0x3232u : 0x1010u;
  uint32_t s[G], m[G];                                 // twice each
#pragma unroll
  for (int g = 0; g < G; g += 2) {
    const uint4 v = *reinterpret_cast<const uint4*>(scales + t / 2 * G * 8 + g * 8);
    s[g] = there ? __byte_perm(v.x, 0, same) : 0u; m[g] = there ? __byte_perm(v.y, 0, same) : 0u;
    s[g + 1] = there ? __byte_perm(v.z, 0, same) : 0u; m[g + 1] = there ? __byte_perm(v.w, 0, same) : 0u;
  }
  int exponent = 0;
#pragma unroll
  for (int g = 0; g < G; ++g) exponent = max(exponent, exponent_of(s[g], m[g]));
  const int lift = lift_of(exponent);
  const __half2 up = lift2(lift);
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const __half2 sc = __hmul2(as_half2(s[g]), up);
    m[g] = as_u32(__hmul2(as_half2(m[g]), up));
    uint32_t p[16], rest[16];
#pragma unroll
    for (int o = 0; o < 4; ++o) {
      uint32_t k[4];
      half_codes(cw[o][g], k);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __half2 x = __hmul2(as_half2(k[i]), sc);
        p[4 * o + i] = as_u32(x);
        rest[4 * o + i] = as_u32(__hfma2(as_half2(k[i]), sc, __hneg2(x)));
      }
    }
    tmem_st16(col + 16 * g, p);
    tmem_st16(col + KeyCols<D>::kRest + 16 * g, rest);
  }
  uint32_t minima[8] = {};
#pragma unroll
  for (int p = 0; p < 3; ++p)
#pragma unroll
    for (int g = 0; g < G; g += 2) minima[(p * G + g) / 2] = __byte_perm(m[g], m[g + 1], 0x5410);
  tmem_st8(col + KeyCols<D>::kMinima, minima);
  return __uint_as_float((uint32_t)(127 - lift) << 23);
}
// descriptors' high words: 128-byte swizzle; none, 8 rows of 16 bytes next to each other
constexpr uint32_t kDescSwizzled = (1024u >> 4) | (1u << 14) | (2u << 29), kDescPlain = (128u >> 4) | (1u << 14);
// S^T = K Q^T of 128 tokens (in TMEM, see above) and the NR rows of an image at `image` in shared memory; by one thread
template <int D, int NR>
__device__ __forceinline__ void scores_of_keys(uint32_t to, uint32_t keys, uint32_t image) {
  using I = Image<D, NR>;
  constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NR >> 3) << 17) | ((128u >> 4) << 24);
  const uint32_t q_lo = (image >> 4) | (1u << 16);
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      mma_ts2(to, keys + part * KeyCols<D>::kRest + 8 * ks, q_lo + (((ks >> 2) * I::kSlab + (ks & 3) * 32) >> 4), kDescSwizzled, idesc, part + ks > 0);
  mma_ts2(to, keys + KeyCols<D>::kMinima, ((image + I::kSums) >> 4) | (((NR * 16u) >> 4) << 16), kDescPlain, idesc, 1);
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// ---- parts of the work -----------------------------------------------------------------------------------------------------
// All requests' tiles are one sequence; a request has `tiles` of equal cost.  Position x of `parts` cuts it at equal costs: the first tile that starts at or behind it, as (request, tile).
// All threads together; s_sums [THREADS / 32].  (A request's cost and tiles: what(r), which may be asked twice.)
struct Place { int request, tile; };
template <int THREADS, class F>
__device__ __forceinline__ void places_of(int requests, int part, int parts, F what, long long* s_sums, Place* s_place) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (requests + THREADS - 1) / THREADS, r0 = min(requests, tid * per), r1 = min(requests, r0 + per);
  long long mine = 0;
  for (int r = r0; r < r1; ++r) { const int2 w = what(r); mine += (long long)w.x * w.y; }
  long long run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += y; }
  if (lane == 31) s_sums[warp] = run;
  if (tid < 2) s_place[tid] = {requests, 0};
  __syncthreads();
  long long total = 0, before = run - mine;
  for (int w = 0; w < THREADS / 32; ++w) { if (w < warp) before += s_sums[w]; total += s_sums[w]; }
  const long long share = total / parts, extra = total % parts;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const long long x = share * (part + e) + min((long long)(part + e), extra);
    if (x < total && x >= before && x < before + mine) {
      long long at = before;
      for (int r = r0; r < r1; ++r) {
        const int2 w = what(r);
        const long long cost = (long long)w.x * w.y;
        if (x < at + cost) { s_place[e] = {r, (int)((x - at + w.y - 1) / w.y)}; break; }
        at += cost;
      }
    }
  }
  __syncthreads();
}

// Places of a table row: so far below 2^31 that what a loop over them, or a last unit of tokens, adds does not pass it
constexpr long long kMostPlaces = 0x7fffffffLL - (1 << 16);

template <class P>
int check_chunk(const P* p) {
  int rc;
  if (!p || p->requests < 0 || p->rows < 0 || p->table_width <= 0 || p->q_heads <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_cache(p->cache, &rc)) return rc;
  if (p->dtype != HYPERATTN_BF16 && p->dtype != HYPERATTN_FP16) return p->dtype == HYPERATTN_FP32 ? HYPERATTN_UNSUPPORTED_SHAPE : HYPERATTN_INVALID_ARGUMENT;
  if (p->q_heads % p->cache.kv_heads || bad_stride(p->q_row_stride) || bad_stride(p->q_head_stride) || p->requests > HYPERATTN_PLAN_MAX_REQUESTS) return HYPERATTN_UNSUPPORTED_SHAPE;
  if ((long long)p->table_width * p->cache.page_tokens > kMostPlaces || (long long)p->rows * p->q_heads > 0x7fffffffLL ||
      (long long)p->cache.num_pages * (p->cache.page_tokens / kBlockTokens) * p->cache.kv_heads > 0x7fffffffLL ||
      ((long long)p->table_width * p->cache.page_tokens / 64 + 1) * p->cache.kv_heads > 0x7fffffffLL)
    return HYPERATTN_UNSUPPORTED_SHAPE;
  return HYPERATTN_OK;
}
template <class P>
ChunkArgs chunk_args(const P& p) {
  ChunkArgs a = {};
  a.cache = view_of(p.cache);
  a.q = p.q; a.q_row = p.q_row_stride; a.q_head = p.q_head_stride;
  a.table = p.table; a.lengths = p.lengths; a.cu_q = p.cu_q;
  a.requests = p.requests; a.rows = p.rows; a.width = p.table_width; a.q_heads = p.q_heads; a.causal = p.causal != 0;
  a.scale_log2 = (p.softmax_scale > 0.f ? p.softmax_scale : 1.f / sqrtf((float)p.cache.d)) * 1.4426950408889634f;
  a.least = -1;
  a.images = reinterpret_cast<uint8_t*>(p.workspace);
  return a;
}

}  // namespace
}  // namespace hyperattn
