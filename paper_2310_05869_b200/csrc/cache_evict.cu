// Requests that have grown too long: new pages for what stays (plan), which tokens stay, and moving them.
#include "serving.cuh"
#include "tc_util.cuh"

namespace hyperattn {
namespace {

// ---- plan ------------------------------------------------------------------------------------------------------------------
// As the cache's plan (cache.cu): every CTA makes the running sums for itself, then some write the tables, some the stack, one the requests' lengths.  256 requests 6.5 us, 1024 x 2048 pages 16.6.
constexpr int kColumns = 512;            // table entries of a warp at a time
struct EvictParts { int tables, stack; };
constexpr int kBeyond = 1 << 20;        // what the step of a loop may add to the last index that there is

__global__ void __launch_bounds__(kPlanThreads) evict_plan_kernel(const __grid_constant__ hyperattn_evict_plan p, EvictParts parts) {
  extern __shared__ int smem[];
  __shared__ int s_warp[1][kPlanWarps], s_given;
  wait_for_stream();
  const int R = p.requests, W = p.table_width, P = p.page_tokens, F = p.num_free;
  // running sums (inclusive) of the pages that are asked for and of those that come back; pages that a request has, 1 << 30: it is cut
  int *s_need = smem, *s_rel = smem + R, *s_have = smem + 2 * R;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n_free = min(max(p.n_free[0], 0), F);
  if (tid == 0) s_given = 0;
  auto pages_of = [&](int tokens) { return (int)(((long long)tokens + P - 1) / P); };
  const int per = (R + kPlanThreads - 1) / kPlanThreads, r0 = min(R, tid * per), r1 = min(R, r0 + per);
  int sum[1] = {0};
  for (int r = r0; r < r1; ++r) {
    const int len = max(p.lengths[r], 0), keep = p.keep[r];
    const bool wants = keep >= 0 && keep < len && pages_of(keep) <= W;
    sum[0] += wants ? pages_of(keep) : 0;
    s_need[r] = sum[0];
    s_have[r] = min(pages_of(len), W) | (wants ? 1 << 30 : 0);
  }
  sums_before(sum, s_warp);
  int back[1] = {0}, given = 0;
  for (int r = r0; r < r1; ++r) {
    s_need[r] += sum[0];
    const int need = s_need[r] - (r > r0 ? s_need[r - 1] : sum[0]);
    if ((s_have[r] >> 30) && need > 0 && s_need[r] > n_free) s_have[r] &= ~(1 << 30);
    if ((s_have[r] >> 30) && need > 0) given = s_need[r];
    back[0] += s_have[r] >> 30 ? s_have[r] & 0x3fffffff : 0;
    s_rel[r] = back[0];
  }
  __syncthreads();                                     // (s_warp is used again)
  if (given) atomicMax(&s_given, given);
  sums_before(back, s_warp);
  for (int r = r0; r < r1; ++r) s_rel[r] += back[0];
  __syncthreads();
  const int left = n_free - s_given, total = min(left + s_rel[R - 1], F);
  auto before = [](const int* a, int r) { return r ? a[r - 1] : 0; };
  auto cut = [&](int r) { return (s_have[r] >> 30 & 1) != 0; };

  int cta = blockIdx.x;
  if (cta < parts.tables) {
    const int pieces = (W + kColumns - 1) / kColumns;
    for (int u = cta * kPlanWarps + warp; u < R * pieces; u += parts.tables * kPlanWarps) {
      const int r = u / pieces, c0 = (u - r * pieces) * kColumns;
      const bool moved = cut(r);
      const int first = before(s_need, r), end = moved ? s_need[r] - first : s_have[r] & 0x3fffffff;
      const int32_t* from = p.table + (size_t)r * W;
      int v[kColumns / 32];
#pragma unroll
      for (int i = 0; i < kColumns / 32; ++i) {
        const int c = c0 + 32 * i + lane;
        v[i] = c >= end ? -1 : moved ? p.free_pages[n_free - 1 - first - c] : from[c];
      }
#pragma unroll
      for (int i = 0; i < kColumns / 32; ++i) {
        const int c = c0 + 32 * i + lane;
        if (c < W) p.table_out[(size_t)r * W + c] = v[i];
      }
    }
    return;
  }
  cta -= parts.tables;
  if (cta < parts.stack) {
    auto stack = [&](int i) {
      if (i >= total) return -1;
      if (i < left) return p.free_pages[i];
      const int r = upper_bound(s_rel, R, i - left);
      return r < R ? p.table[(size_t)r * W + (i - left - before(s_rel, r))] : -1;
    };
    const bool quads = ((reinterpret_cast<uintptr_t>(p.free_pages) | reinterpret_cast<uintptr_t>(p.free_out)) & 15) == 0;
    for (int i = 4 * (cta * kPlanThreads + tid); i < F; i += 4 * parts.stack * kPlanThreads) {
      if (quads && i + 4 <= F && (i >= total || i + 4 <= left))
        *reinterpret_cast<int4*>(p.free_out + i) = i >= total ? make_int4(-1, -1, -1, -1) : *reinterpret_cast<const int4*>(p.free_pages + i);
      else
        for (int k = i; k < min(i + 4, F); ++k) p.free_out[k] = stack(k);
    }
    return;
  }
  for (int r = tid; r < R; r += kPlanThreads) p.lengths_out[r] = cut(r) ? p.keep[r] : max(p.lengths[r], 0);
  if (tid == 0) p.n_free_out[0] = total;
}

// ---- which tokens stay -------------------------------------------------------------------------------------------------------
struct EvictArgs {
  CacheView cache;
  const float* weights;
  float* weights_out;
  int32_t* kept;
  const int32_t *table, *lengths, *to_table, *to_lengths;
  int requests, width, recent, first;
};
struct Cut {                             // of a request
  int len, n;                            // tokens before and after
  __device__ __forceinline__ bool moved() const { return n < len; }
};
__device__ __forceinline__ Cut cut_of(const EvictArgs& a, int r) {
  Cut c;
  c.len = min(max(a.lengths[r], 0), a.width * a.cache.page);
  c.n = min(max(a.to_lengths[r], 0), c.len);
  return c;
}
// the order of weights as that of whole numbers: those that are negative or no numbers count as 0
__device__ __forceinline__ uint32_t order_of(float w) { return w > 0.f ? __float_as_uint(w) : 0u; }

// A cluster of CTAs takes a request and key head, each a slice of its tokens, whose weights (in order) it holds in shared memory if they fit.  The smallest weight that stays is
// found by three digits of 10, 11 and 10 bits, from the top: a histogram in each CTA, which all add up for themselves.  Then every warp counts a part of the slice, and numbers it.
// 131072 tokens to 8192 beside a request of 7148 that stays, 32 heads: 57 us (115 with four digits of 8 bits), of 13 for its bytes: two waves of clusters, instructions and latencies between the digits.  32 requests up to 8192
// tokens, 8 heads: 19 us.
constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32, kBins = 2048, kMostHeld = 40960;

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// a word of another CTA's shared memory, at the place where this one has `addr`
__device__ __forceinline__ int peer_word(uint32_t addr, uint32_t rank) {
  uint32_t at;
  int v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

__global__ void __launch_bounds__(kSelectThreads) select_kernel(const __grid_constant__ EvictArgs a, int ctas, int held) {
  extern __shared__ __align__(16) int s_mem[];
  int* s_hist = s_mem;                                 // [3][kBins]
  uint32_t* s_key = reinterpret_cast<uint32_t*>(s_mem + 3 * kBins);            // [held]
  __shared__ int s_digit, s_above, s_count[2];
  __shared__ uint32_t s_warp[kSelectWarps];
  wait_for_stream();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int pair = blockIdx.x / ctas, rank = ctas > 1 ? (int)cluster_rank() : 0, r = pair / a.cache.heads, cap = a.width * a.cache.page;
  const Cut c = cut_of(a, r);
  const float* w = a.weights + (size_t)pair * cap;
  float* out = a.weights_out + (size_t)pair * cap;
  int32_t* kept = a.kept + (size_t)pair * cap;
  const int4 none = make_int4(-1, -1, -1, -1);
  if (!c.moved()) {                                    // (all CTAs of the cluster)
    for (int t = 4 * (rank * kSelectThreads + tid); t < cap; t += 4 * ctas * kSelectThreads) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (t < c.len) {
        x = *reinterpret_cast<const float4*>(w + t);
        if (t + 1 >= c.len) x.y = 0.f;
        if (t + 2 >= c.len) x.z = 0.f;
        if (t + 3 >= c.len) x.w = 0.f;
      }
      *reinterpret_cast<float4*>(out + t) = x;
      *reinterpret_cast<int4*>(kept + t) = none;
    }
    return;
  }
  const int recent = min(a.recent, c.n), first = min(a.first, c.n - recent), begin = first, end = c.len - recent;
  int want = c.n - recent - first;                     // tokens of [begin, end) that stay
  // (a multiple of 4 tokens each; no sum that wraps)
  const int slice = ((c.len - 1) / ctas / 4 + 1) * 4, t0 = (int)min((long long)rank * slice, (long long)c.len), t1 = (int)min((long long)t0 + slice, (long long)c.len);
  const bool hold = slice <= held;
  for (int i = tid; i < 3 * kBins; i += kSelectThreads) s_hist[i] = 0;
  __syncthreads();
  auto key_of = [&](int t) { return hold ? s_key[t - t0] : order_of(w[t]); };
  auto inside = [&](int t) { return t >= begin && t < end; };
  uint32_t top = 0;                                    // digits of the smallest weight that stays, so far
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 1 ? 2048 : 1024;
    int* hist = s_hist + pass * kBins;
    if (pass == 0) {
      for (int t = t0 + 4 * tid; t < t1; t += 4 * kSelectThreads) {
        const float4 x = *reinterpret_cast<const float4*>(w + t);                // (a row is whole quads)
        const uint4 k = make_uint4(order_of(x.x), order_of(x.y), order_of(x.z), order_of(x.w));
        if (hold) *reinterpret_cast<uint4*>(s_key + t - t0) = k;
        if (inside(t)) atomicAdd(&hist[k.x >> 21], 1);
        if (inside(t + 1) && t + 1 < t1) atomicAdd(&hist[k.y >> 21], 1);
        if (inside(t + 2) && t + 2 < t1) atomicAdd(&hist[k.z >> 21], 1);
        if (inside(t + 3) && t + 3 < t1) atomicAdd(&hist[k.w >> 21], 1);
      }
    } else {
      const int done = pass == 1 ? 21 : 10;
      for (int t = max(begin, t0) + tid; t < min(end, t1); t += kSelectThreads) {
        const uint32_t x = key_of(t);
        if (x >> done == top >> done) atomicAdd(&hist[x >> shift & (bins - 1)], 1);
      }
    }
    if (ctas > 1) cluster_sync(); else __syncthreads();
    // a thread has one digit or two, from the largest downwards
    const int each = bins / kSelectThreads;
    int mine[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < each; ++e) {
      const int digit = bins - 1 - each * tid - e;
      if (ctas > 1) {
#pragma unroll 8
        for (int k = 0; k < ctas; ++k) mine[e] += peer_word(smem_u32(hist + digit), k);
      } else mine[e] = hist[digit];
    }
    int sum = mine[0] + mine[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += y; }
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    const int before = lane < warp ? (int)s_warp[lane] : 0;
    int above = __reduce_add_sync(0xffffffffu, before) + sum - mine[0] - mine[1];
#pragma unroll
    for (int e = 0; e < each; ++e) {
      if (above < want && above + mine[e] >= want) { s_digit = bins - 1 - each * tid - e; s_above = above; }
      above += mine[e];
    }
    __syncthreads();
    if (want > 0) {                                    // (0: none of these stays)
      top |= (uint32_t)s_digit << shift;
      want -= s_above;
    }
  }
  if (want == 0) top = 0xffffffffu;
  // `want` of those that weigh `top` stay, the first ones; and all that weigh more.  A warp has consecutive tokens
  const int part = ((t1 - t0 + kSelectWarps - 1) / kSelectWarps + 31) / 32 * 32, p0 = min(t0 + warp * part, t1), p1 = min(p0 + part, t1);
  int sure = 0, same = 0;                              // tokens that stay for sure, and equal ones: of the warp, then before it
  for (int t = p0 + lane; t < p1 + lane; t += 32) {
    const uint32_t x = t < p1 ? key_of(t) : 0u;
    sure += __popc(__ballot_sync(0xffffffffu, t < p1 && (!inside(t) || x > top)));
    same += __popc(__ballot_sync(0xffffffffu, t < p1 && inside(t) && x == top));
  }
  uint2* s_part = reinterpret_cast<uint2*>(s_hist);    // [kSelectWarps] (the first digit's histogram has been read by all: two rounds ago)
  if (lane == 0) s_part[warp] = make_uint2(sure, same);
  __syncthreads();
  uint2 counts = s_part[lane];
  int ahead_sure = __reduce_add_sync(0xffffffffu, lane < warp ? counts.x : 0u), ahead_same = __reduce_add_sync(0xffffffffu, lane < warp ? counts.y : 0u);
  if (ctas > 1) {
    const int all_sure = __reduce_add_sync(0xffffffffu, counts.x), all_same = __reduce_add_sync(0xffffffffu, counts.y);
    if (tid == 0) { s_count[0] = all_sure; s_count[1] = all_same; }
    cluster_sync();
    for (int k = 0; k < rank; ++k) { ahead_sure += peer_word(smem_u32(&s_count[0]), k); ahead_same += peer_word(smem_u32(&s_count[1]), k); }
  }
  for (int t = p0 + lane; t < p1 + lane; t += 32) {
    const uint32_t x = t < p1 ? key_of(t) : 0u;
    const bool s = t < p1 && (!inside(t) || x > top), e = t < p1 && inside(t) && x == top;
    const unsigned ms = __ballot_sync(0xffffffffu, s), me = __ballot_sync(0xffffffffu, e), below = (1u << lane) - 1;
    const int eq = ahead_same + __popc(me & below);
    if (s || (e && eq < want)) {
      const int at = ahead_sure + __popc(ms & below) + min(eq, want);
      kept[at] = t;
      out[at] = w[t];
    }
    ahead_sure += __popc(ms);
    ahead_same += __popc(me);
  }
  const int whole = min((c.n + 3) / 4 * 4, cap);
  if (rank == 0 && tid < whole - c.n) { out[c.n + tid] = 0.f; kept[c.n + tid] = -1; }
  for (int t = whole + 4 * (rank * kSelectThreads + tid); t < cap; t += 4 * ctas * kSelectThreads) {
    *reinterpret_cast<float4*>(out + t) = make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<int4*>(kept + t) = none;
  }
  if (ctas > 1) cluster_sync();                        // (nobody's shared memory goes while another may read it)
}
static_assert(kSelectWarps == 32, "a lane for every warp");

// ---- moving them -------------------------------------------------------------------------------------------------------------
// A warp makes a block of 16 tokens of the new pages at a time, from the blocks that its tokens are in: K by pieces of a token (16 bytes, d = 64: 8), V by 16-byte loads that
// hold a token's byte of four words, scales and minima one by one.  The blocks of all requests that are cut are one sequence, in equal parts for the warps.
// 32 requests to 2048 tokens, 8 heads of 128: 41 us (115 MB read where tokens that stay have about 40: sectors are used in part; stalls are those of gathers).
// With 12 CTAs an SM, of which 9 are there at a time, 127.8 for all of the eviction and its reading back, with 18 or 36 123.5 (131072 tokens to 8192, 32 heads of 64: 131.1, 128.6).
constexpr int kMoveWarps = 4, kMostRequests = HYPERATTN_PLAN_MAX_REQUESTS;

template <int D>
__global__ void __launch_bounds__(32 * kMoveWarps) move_kernel(const __grid_constant__ EvictArgs a) {
  using B = Block<D>;
  constexpr int G = B::kGroups;
  extern __shared__ int s_starts[];                    // [requests + 1] blocks of one head before a request
  __shared__ int s_sums[kMoveWarps];
  wait_for_stream();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.requests + 32 * kMoveWarps - 1) / (32 * kMoveWarps), r0 = min(a.requests, tid * per), r1 = min(a.requests, r0 + per);
  int mine = 0;
  for (int r = r0; r < r1; ++r) {
    const Cut c = cut_of(a, r);
    s_starts[r] = mine;
    mine += c.moved() ? (c.n + kBlockTokens - 1) / kBlockTokens : 0;
  }
  int run = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += y; }
  if (lane == 31) s_sums[warp] = run;
  __syncthreads();
  run -= mine;
  for (int w = 0; w < warp; ++w) run += s_sums[w];
  for (int r = r0; r < r1; ++r) s_starts[r] += run;
  if (tid == 32 * kMoveWarps - 1) s_starts[a.requests] = run + mine;
  __syncthreads();
  const int H = a.cache.heads, subs = a.cache.page / kBlockTokens, cap = a.width * a.cache.page;
  const long long total = (long long)s_starts[a.requests] * H, warps = (long long)gridDim.x * kMoveWarps;
  const uint8_t* pages = a.cache.pages;
  // A block's place, and for lane t < 16 where its token t comes from: asked for two blocks (which tokens) and one block (which pages) before it is made.
  struct Job { int r, head, b, src, page, to_page; };
  auto find = [&](long long u, Job& j, int from) {     // which tokens
    j.r = -1;
    j.src = -1;
    if (u >= total) return;
    int r = from;                                      // (blocks come in order: the request is this one or a later one)
    while ((long long)s_starts[r + 1] * H <= u) ++r;
    const int blocks = s_starts[r + 1] - s_starts[r], rest = (int)(u - (long long)s_starts[r] * H);
    j.r = r;
    j.head = rest / blocks;
    j.b = rest - j.head * blocks;
    const int at = j.b * kBlockTokens + lane;
    if (lane < kBlockTokens && at < cap) j.src = a.kept[((size_t)r * H + j.head) * cap + at];
  };
  auto pages_of = [&](Job& j) {
    j.page = j.to_page = -1;
    if (j.r < 0) return;
    if (j.b / subs < a.width) j.to_page = a.to_table[(size_t)j.r * a.width + j.b / subs];
    if (j.src >= 0 && j.src < cap) j.page = a.table[(size_t)j.r * a.width + j.src / a.cache.page];
  };
  long long u = blockIdx.x * kMoveWarps + warp;
  Job now, next, then;
  find(u, now, 0);
  find(u + warps, next, max(now.r, 0));
  pages_of(now);
  for (; now.r >= 0; u += warps, now = next, next = then) {
    pages_of(next);
    find(u + 2 * warps, then, max(next.r, 0));
    const int head = now.head, b = now.b;
    if (now.to_page < 0 || now.to_page >= a.cache.num_pages) continue;
    uint8_t* to = block_at<D>(a.cache, now.to_page, head, b % subs);
    // (block -1: nowhere, zeros)
    const int block = now.page >= 0 && now.page < a.cache.num_pages ? (now.page * H + head) * subs + now.src % a.cache.page / kBlockTokens : -1;
    int src = now.src;
    src &= kBlockTokens - 1;
    auto block_of = [&](int t) { return __shfl_sync(0xffffffffu, block, t); };
    auto token_of = [&](int t) { return __shfl_sync(0xffffffffu, src, t); };
    auto bytes_at = [&](int blk, int at) { return pages + (size_t)blk * B::kBytes + at; };
    // K
    uint4 k[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int blk = block_of(half * 8 + lane / 4), t = token_of(half * 8 + lane / 4), ln = t % 8 * 4 + lane % 4;
      if constexpr (D == 128) k[half] = blk < 0 ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(bytes_at(blk, t / 8 * 512 + ln * 16));
      else {
        const uint2 x = blk < 0 ? make_uint2(0, 0) : *reinterpret_cast<const uint2*>(bytes_at(blk, ln * 16 + t / 8 * 8));
        if (half) { k[0].z = x.x; k[0].w = x.y; } else { k[0].x = x.x; k[0].y = x.y; }
      }
    }
    // V: bytes of a word: tokens 2 c, 8 + 2 c, 2 c + 1, 9 + 2 c
    uint4 v[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) v[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int mine_t = 2 * (lane % 4) + p / 2 + (p & 1) * 8, blk = block_of(mine_t), t = token_of(mine_t), byte = t % 2 * 2 + t / 8;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint4 x = blk < 0 ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(bytes_at(blk, B::kV + i * 512 + (lane / 4 * 4 + t % 8 / 2) * 16));
        const uint32_t pick = 0x3210u & ~(0xfu << (4 * p)) | (uint32_t)(4 + byte) << (4 * p);              // byte p from the source
        v[i].x = __byte_perm(v[i].x, x.x, pick); v[i].y = __byte_perm(v[i].y, x.y, pick);
        v[i].z = __byte_perm(v[i].z, x.z, pick); v[i].w = __byte_perm(v[i].w, x.w, pick);
      }
    }
    // scales and minima: words of tokens 2 i, 2 i + 1
    uint32_t sc[2 * D / 64];
#pragma unroll
    for (int j = 0; j < 2 * D / 64; ++j) {
      const int word = j * 32 + lane, tp = word / (2 * G) % 8, at = B::kScaleK + (word / (16 * G)) * 2 * D;         // K's, then V's
      uint32_t both = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int blk = block_of(2 * tp + e), t = token_of(2 * tp + e);
        const uint32_t x = blk < 0 ? 0u : *reinterpret_cast<const uint16_t*>(bytes_at(blk, at + (t / 2 * 2 * G + word % (2 * G)) * 4 + t % 2 * 2));
        both |= x << (16 * e);
      }
      sc[j] = both;
    }
    *reinterpret_cast<uint4*>(to + lane * 16) = k[0];
    if constexpr (D == 128) *reinterpret_cast<uint4*>(to + 512 + lane * 16) = k[1];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) *reinterpret_cast<uint4*>(to + B::kV + i * 512 + lane * 16) = v[i];
#pragma unroll
    for (int j = 0; j < 2 * D / 64; ++j) *reinterpret_cast<uint32_t*>(to + B::kScaleK + (j * 32 + lane) * 4) = sc[j];
  }
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_cache_evict_plan(const hyperattn_evict_plan* p) {
  if (!p || p->requests < 0 || p->table_width <= 0 || p->num_free < 0 || p->page_tokens <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (p->requests > HYPERATTN_PLAN_MAX_REQUESTS || (long long)p->table_width * p->page_tokens > 0x7fffffffLL || p->table_width >= 1 << 28 ||
      (long long)p->requests * p->table_width + p->num_free > 0x7fffffffLL - kBeyond)
    return HYPERATTN_UNSUPPORTED_SHAPE;
  if (p->requests == 0) return HYPERATTN_OK;
  if (!p->lengths || !p->keep || !p->table || (p->num_free && (!p->free_pages || !p->free_out)) || !p->n_free || !p->lengths_out || !p->table_out || !p->n_free_out)
    return HYPERATTN_INVALID_ARGUMENT;
  if (p->lengths_out == p->lengths || p->lengths_out == p->keep || p->table_out == p->table || (p->num_free && p->free_out == p->free_pages) || p->n_free_out == p->n_free)
    return HYPERATTN_MISALIGNED;
  const int smem = 3 * p->requests * (int)sizeof(int);
  if (smem > 40 * 1024)
    if (int rc = status_of(allow_smem<evict_plan_kernel>(3 * HYPERATTN_PLAN_MAX_REQUESTS * (int)sizeof(int)), "evict plan: shared memory")) return rc;
  auto ctas = [](long long work, int per, int most) { return (int)(work <= 0 ? 0 : (work + per - 1) / per < most ? (work + per - 1) / per : most); };
  const EvictParts parts = {ctas((long long)p->requests * ((p->table_width + kColumns - 1) / kColumns), kPlanWarps, 2 * kSms), ctas(p->num_free, 8 * kPlanThreads, kSms)};
  return status_of(launch(evict_plan_kernel, dim3((unsigned)(parts.tables + parts.stack + 1)), dim3(kPlanThreads), smem, reinterpret_cast<cudaStream_t>(p->stream), *p, parts), "evict plan");
}

extern "C" int hyperattn_cache_evict(const hyperattn_evict_params* p) {
  int rc;
  if (!p || p->requests < 0 || p->table_width <= 0 || p->recent < 0 || p->first < 0) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_cache(p->cache, &rc)) return rc;
  if (p->requests > kMostRequests || (long long)p->table_width * p->cache.page_tokens > 0x7fffffffLL - kBeyond || (long long)p->requests * p->cache.kv_heads > 0x7fffffffLL / 8 ||
      (long long)p->requests * p->table_width * (p->cache.page_tokens / kBlockTokens) > 0x7fffffffLL ||
      (long long)p->cache.num_pages * (p->cache.page_tokens / kBlockTokens) * p->cache.kv_heads > 0x7fffffffLL)
    return HYPERATTN_UNSUPPORTED_SHAPE;
  if (p->requests == 0) return HYPERATTN_OK;
  if (!p->weights || !p->weights_out || !p->kept || !p->table || !p->lengths || !p->to_table || !p->to_lengths) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->weights) || misaligned(p->weights_out) || misaligned(p->kept) || p->weights == p->weights_out) return HYPERATTN_MISALIGNED;
  const EvictArgs a = {view_of(p->cache), p->weights, p->weights_out, p->kept, p->table, p->lengths, p->to_table, p->to_lengths, p->requests, p->table_width, p->recent, p->first};
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  // CTAs of a cluster: so that each has some 8192 tokens at most, up to eight
  const int cap = p->table_width * p->cache.page_tokens;
  int ctas = 1;
  while (ctas < 8 && cap > 8192 * ctas) ctas *= 2;
  int held = (cap / ctas + 7) / 4 * 4;
  if (held > kMostHeld) held = 0;
  const int smem = (3 * kBins + held) * 4;
  cudaError_t e = allow_smem<select_kernel>((3 * kBins + kMostHeld) * 4);
  if (e == cudaSuccess) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)ctas, 1, 1};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p->requests * p->cache.kv_heads * ctas)); cfg.blockDim = dim3(kSelectThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, select_kernel, a, ctas, held);
  }
  if (e == cudaSuccess) {
    const long long blocks = (long long)p->requests * p->cache.kv_heads * ((long long)p->table_width * p->cache.page_tokens / kBlockTokens);
    const long long want = (blocks + kMoveWarps - 1) / kMoveWarps;
    const dim3 grid((unsigned)(want < 18 * kSms ? want : 18 * kSms));
    const int smem = (p->requests + 1) * (int)sizeof(int);
    e = p->cache.d == 64 ? launch(move_kernel<64>, grid, dim3(32 * kMoveWarps), smem, st, a) : launch(move_kernel<128>, grid, dim3(32 * kMoveWarps), smem, st, a);
  }
  return status_of(e, "evict");
}
