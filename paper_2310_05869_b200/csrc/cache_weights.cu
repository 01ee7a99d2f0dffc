// The attention weight that cached tokens get from some rows, on the 5th-generation tensor cores.
//
// A tile is 128 tokens of a key head.  Its keys become an operand in TMEM, a lane a token (cache_tiles.cuh), and meet the request's rows NR at a time:
//     S^T = K Q^T                                  tcgen05.mma, queries from shared memory (images that a first launch makes, one bulk copy each)
//     w_t += sum_i exp2(s_ti c_i - lse_i)          a thread a token, so that sums over rows stay in it
// Every token's sum is one thread's (two: a tile's first, third ... images and its second, fourth ...), so nothing is atomic and results do not depend on timing.
//
// What bounds it: exponentials, 16 a clock and SM (60 % of the cycles), and what stands around them: 2 requests, 1025 rows over up to 32000 tokens, 32 heads of 64: 299 us (251 without the
// exponentials, 273 without the products, 167 without the sums, 293 without the keys' conversion); bytes alone 50.  16 warps for the sums instead of 8: 310; one pair of exponentials in eight by
// arithmetic: 347; the next scores on their way while 16 are used: 355.
//
// Warp roles: 0-7 sums (two groups of four, for every other image), 8-15 keys (two groups, for every other tile), 16 products (and TMEM), 17 copies of keys, 18 of images.
// Every wait is bounded: a CTA that gives up raises the device status word, drains its copies, frees its TMEM and returns.
#include <climits>
#include <type_traits>
#include "cache_rows.cuh"
#include "cache_tiles.cuh"

namespace hyperattn {
namespace {

struct alignas(64) KeyMaps {
  CUtensorMap codes, scales;             // K's codes, scales and minima of `run` blocks that follow each other
};

struct WeightArgs {
  ChunkArgs c;
  const float* before;
  float* out;
  float decay;
  int run;                               // blocks of a copy: the largest power of two (up to 8) that divides a page's
};

constexpr int kTileTokens = 128, kWThreads = 608;
// cost of a tile's keys in images
constexpr int kKeyCost = 2;

template <int D, int NR>
struct WCfg {
  using I = Image<D, NR>;
  static constexpr uint32_t kRawBlock = 10 * D, kRaw = 8 * kRawBlock, kScales = 64 * D;           // K's half of 8 blocks: their codes, then their scales
  static constexpr int kRawStages = D == 128 ? 6 : 8, kQStages = 4;
  static constexpr uint32_t kOffQ = 0, kOffRaw = kQStages * I::kBytes, kOffMisc = kOffRaw + kRawStages * kRaw;
  static constexpr uint32_t kOffNext = kOffMisc + 4096, kMostRequests = HYPERATTN_PLAN_MAX_REQUESTS;
  static constexpr uint32_t kSmem = kOffNext + kMostRequests * 2 + 1024;         // (the images begin at multiples of 1024)
  // TMEM columns: keys of two tiles, scores of several images
  static constexpr uint32_t kColS = 2 * KeyCols<D>::kAll;
  static constexpr int kStages = (512 - kColS) / NR < 4 ? (512 - kColS) / NR : 4;
};

// a CTA's tiles in order
struct Walk {
  int request, tile, tiles, head, j;     // tile: of the request's tiles of all heads; tiles, j: of the head's
  Span s;
  int images, first;                     // of the request; first one with a row that sees one of the tile's tokens
  bool end;
};
// The request that tile `tile` of w.request is in, if any.  next: of each request, the next one with tiles (most of a server's places may be without a request; asked one after the other, 1023 of them
// took 230 us).
template <int NR>
__device__ __forceinline__ void walk_request(const ChunkArgs& a, Walk& w, const Place& end, const uint16_t* next) {
  for (;; w.request = next[w.request], w.tile = 0) {
    w.end = w.request > end.request || (w.request == end.request && w.tile >= end.tile) || w.request >= a.requests;
    if (w.end) return;
    w.s = span_of(a, w.request);
    w.tiles = is_for(a, w.s) ? (w.s.len + kTileTokens - 1) / kTileTokens : 0;
    if (w.tile < w.tiles * a.cache.heads) break;
  }
  w.images = (int)(((long long)w.s.rows * (a.q_heads / a.cache.heads) + NR - 1) / NR);
  w.head = w.tile / w.tiles;
  w.j = w.tile - w.head * w.tiles;
}
template <int NR>
__device__ __forceinline__ void walk_first(const ChunkArgs& a, Walk& w) {
  const int from = w.j * kTileTokens - (w.s.len - w.s.rows);               // first row (token) that sees the tile's first token
  w.first = a.causal && from > 0 ? (int)min((long long)from * (a.q_heads / a.cache.heads) / NR, (long long)w.images) : 0;
}
// (out of line: as a part of each role it made all of them slower, 2 requests of 1025 rows 298 -> 340 us)
template <int NR>
__device__ __noinline__ Walk walk_from(const ChunkArgs& a, const Place& begin, const Place& end, const uint16_t* next) {
  Walk w = {};
  w.request = begin.request;
  w.tile = begin.tile;
  walk_request<NR>(a, w, end, next);
  walk_first<NR>(a, w);
  return w;
}
template <int NR>
__device__ __forceinline__ void walk_on(const ChunkArgs& a, Walk& w, const Place& end, const uint16_t* next) {
  ++w.tile;
  if (++w.j == w.tiles) { w.j = 0; ++w.head; }
  if (w.head == a.cache.heads) { w.request = next[w.request]; w.tile = 0; walk_request<NR>(a, w, end, next); }
  else w.end = w.request == end.request && w.tile >= end.tile;
  walk_first<NR>(a, w);
}

template <int D, int NR>
__global__ void __launch_bounds__(kWThreads, 1) weights_kernel(const __grid_constant__ WeightArgs p, const __grid_constant__ KeyMaps maps, int* status) {
  using C = WCfg<D, NR>;
  using I = Image<D, NR>;
  constexpr int NS = C::kStages, NQ = C::kQStages, NRAW = C::kRawStages;
  const ChunkArgs& a = p.c;
  extern __shared__ uint8_t smem_[];
  uint8_t* smem = smem_ + (1024 - (smem_u32(smem_) & 1023)) % 1024;
  const uint32_t ubase = smem_u32(smem);
  uint8_t* misc = smem + C::kOffMisc;
  float* s_factor = reinterpret_cast<float*>(misc);                            // [2][128] of the tiles' tokens; negative: no such token
  float* s_part = s_factor + 256;                                              // [2][128] sums of odd images
  long long* s_sums = reinterpret_cast<long long*>(misc + 2048);               // [18]
  Place* s_place = reinterpret_cast<Place*>(misc + 2048 + 160);                // [2]
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc + 2048 + 176);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc + 2048 + 180);
  uint32_t* s_there = reinterpret_cast<uint32_t*>(misc + 2048 + 184);          // [kRawStages] which of a tile's blocks are in the cache
  uint32_t* s_with = reinterpret_cast<uint32_t*>(misc + 3 * 1024);                 // [kMostRequests / 32] a bit a request: it has tiles
  uint16_t* s_next = reinterpret_cast<uint16_t*>(smem + C::kOffNext);          // [kMostRequests] the next request that has
  const uint32_t bar0 = ubase + C::kOffMisc + 2048 + 232;
  static_assert(232 + 64 + 8 * (2 * NS + 2 * NQ + 2 * NRAW) <= 1024 && C::kMostRequests / 8 <= 1024, "room for barriers and bits");
  auto bar_key = [&](int b) { return bar0 + 8 * b; };                          // keys of a tile are in TMEM
  auto bar_keyfree = [&](int b) { return bar0 + 16 + 8 * b; };                 // multiplied, factors read
  auto bar_s = [&](int s) { return bar0 + 32 + 8 * s; };                       // scores of an image
  auto bar_sfree = [&](int s) { return bar0 + 32 + 8 * (NS + s); };
  auto bar_q = [&](int s) { return bar0 + 32 + 8 * (2 * NS + s); };            // an image has landed
  auto bar_qfree = [&](int s) { return bar0 + 32 + 8 * (2 * NS + NQ + s); };
  auto bar_raw = [&](int s) { return bar0 + 32 + 8 * (2 * NS + 2 * NQ + s); }; // K's bytes of a tile have landed
  auto bar_rawfree = [&](int s) { return bar0 + 32 + 8 * (2 * NS + 2 * NQ + NRAW + s); };
  auto bar_part = [&](int b) { return bar0 + 32 + 8 * (2 * NS + 2 * NQ + 2 * NRAW + b); };          // sums of odd images
  auto bar_partfree = [&](int b) { return bar0 + 48 + 8 * (2 * NS + 2 * NQ + 2 * NRAW + b); };
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) *s_abort = *reinterpret_cast<volatile int*>(status);
  __syncthreads();
  if (*s_abort) return;
  __syncthreads();
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) { mbar_init(bar_key(i), 128); mbar_init(bar_keyfree(i), 1 + 4); mbar_init(bar_part(i), 128); mbar_init(bar_partfree(i), 128); }
    for (int i = 0; i < NS; ++i) { mbar_init(bar_s(i), 1); mbar_init(bar_sfree(i), 128); }
    for (int i = 0; i < NQ; ++i) { mbar_init(bar_q(i), 1); mbar_init(bar_qfree(i), 1 + 4); }
    for (int i = 0; i < NRAW; ++i) { mbar_init(bar_raw(i), 1); mbar_init(bar_rawfree(i), 4); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = tid; i < (int)C::kMostRequests / 32; i += kWThreads) s_with[i] = 0;
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *s_tmem, 0);
  wait_for_stream();
  const int group = a.q_heads / a.cache.heads, cap = a.width * a.cache.page, subs = a.cache.page / kBlockTokens;
  places_of<kWThreads>(a.requests, blockIdx.x, gridDim.x, [&](int r) {
    const Span s = span_of(a, r);
    const int tiles = is_for(a, s) ? (s.len + kTileTokens - 1) / kTileTokens : 0;
    if (tiles > 0) atomicOr(&s_with[r >> 5], 1u << (r & 31));
    return make_int2(tiles * a.cache.heads, kKeyCost + (int)(((long long)s.rows * group + NR - 1) / NR));
  }, s_sums, s_place);
  const Place begin = s_place[0], end = s_place[1];
  for (int r = tid; r < a.requests; r += kWThreads) {
    int word = (r + 1) >> 5;
    uint32_t bits = r + 1 < a.requests ? s_with[word] >> ((r + 1) & 31) << ((r + 1) & 31) : 0u;
    while (!bits && ++word * 32 < a.requests) bits = s_with[word];
    s_next[r] = (uint16_t)(bits ? word * 32 + __ffs(bits) - 1 : a.requests);
  }
  __syncthreads();
  auto image_at = [&](const Walk& w, int i) { return a.images + ((size_t)(image_slots(w.s.first, w.request, group, NR, a.least) + i) * a.cache.heads + w.head) * I::kBytes; };
  bool ok = true;

  if (warp < 8) {
    // ================= sums: a thread a token ==============================================================
    const int g = warp >> 2, t = tid & 127;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    auto sum_of = [](const uint64_t (&x)[2]) {
      float s0, s1;
      unpack_f2(fadd2(x[0], x[1]), s0, s1);
      return s0 + s1;
    };
    int images = 0, keyed = 0, plain = 0, shared = 0;      // images, tiles with rows, without, and with several images so far
    auto had = [&](const Walk& w, bool mine) {             // what the token had, asked for ahead
      const int token = w.j * kTileTokens + t;
      return mine && p.before && token < w.s.len - w.s.rows ? p.before[((size_t)w.request * a.cache.heads + w.head) * cap + token] : 0.f;
    };
    for (Walk w = walk_from<NR>(a, begin, end, s_next); !w.end && ok; walk_on<NR>(a, w, end, s_next)) {
      const int token = w.j * kTileTokens + t, count = w.images - w.first;
      const size_t at = ((size_t)w.request * a.cache.heads + w.head) * cap + token;
      // the group that has the tile's first image puts its results together; the other one has nothing to do with a tile of one image
      const int lead = (count ? images : plain++) & 1;
      const bool mine = lead == g;
      if (!mine && count < 2) { images += count; keyed += count; continue; }
      const float old = had(w, mine);
      uint64_t sum2[2] = {0, 0};
      bool there = token < w.s.len;
      if (count) {
        const int b = keyed & 1;
        ok = warp_wait<20>(bar_key(b), (keyed >> 1) & 1, s_abort, status);
        if (!ok) break;
        const float f = s_factor[b * 128 + t];
        __syncwarp();
        if (count == 1 && lane == 0) mbar_arrive(bar_keyfree(b));
        ++keyed;
        there = there && f > 0.f;
        // columns of all images that see the token: from `sees` on, up to the rows that there are
        const long long sees = a.causal ? (long long)(token - (w.s.len - w.s.rows)) * group : 0, rows = (long long)w.s.rows * group;
        const long long partly = a.causal ? (long long)(w.j * kTileTokens + kTileTokens - 1 - (w.s.len - w.s.rows)) * group : 0;       // (of the tile's last token)
        for (int i = w.first; i < w.images; ++i, ++images) {
          if ((images & 1) != g) continue;
          const int st = images % NS, qs = images % NQ;
          ok = warp_wait<21>(bar_s(st), (images / NS) & 1, s_abort, status);
          if (ok) ok = warp_wait<22>(bar_q(qs), (images / NQ) & 1, s_abort, status);                    // (it has landed: the factors beside it are visible to this thread too)
          if (!ok) break;
          tc_fence_after();
          const uint8_t* image = smem + C::kOffQ + qs * I::kBytes;
          const long long c0 = (long long)i * NR;
          const float factor = *reinterpret_cast<const float*>(image + I::kFactor);
          // Rows that all tokens of the tile see, in steps of 32; masks, and rows with factors of their own, are a path apart; what no token sees is left out
          const int hi = (int)min(rows - c0, (long long)NR), all = (int)min(max(partly - c0, 0ll), (long long)NR), lo = (int)min(max(sees - c0, 0ll), (long long)NR);
          const int some = max(all - kTileTokens * group, 0);              // (the tile's first token sees rows from here on, or from further)
          const float times = factor * f;
          constexpr int STEP = 32;
          const int begin_c = some / STEP * STEP;
          if (begin_c >= hi) mbar_arrive(bar_sfree(st));
#pragma unroll 1
          for (int c = begin_c; c < hi; c += STEP) {
            uint32_t r[STEP];
            tmem_ld32_issue(lane_addr + C::kColS + st * NR + c, r);
            const float4* minus = reinterpret_cast<const float4*>(image + I::kMinus) + c / 4;
            tmem_ld32_wait(r);
            if (c + STEP >= hi) {
              tc_fence_before();
              mbar_arrive(bar_sfree(st));
            }
            auto add = [&](auto plain) {
              constexpr bool PLAIN = decltype(plain)::value;
              uint64_t times0 = pack_f2(times, times), times1 = times0;
#pragma unroll
              for (int e = 0; e < STEP; e += 4) {
                const float4 m = minus[e / 4];
                if constexpr (!PLAIN) {
                  const float4 g = reinterpret_cast<const float4*>(image + I::kFactors)[(c + e) / 4];
                  times0 = pack_f2(g.x * f, g.y * f);
                  times1 = pack_f2(g.z * f, g.w * f);
                }
                float x[4];
                unpack_f2(ffma2(pack_u2(r[e], r[e + 1]), times0, pack_f2(m.x, m.y)), x[0], x[1]);
                unpack_f2(ffma2(pack_u2(r[e + 2], r[e + 3]), times1, pack_f2(m.z, m.w)), x[2], x[3]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  x[k] = ex2(x[k]);
                  if constexpr (!PLAIN) x[k] = c + e + k >= lo && c + e + k < hi ? x[k] : 0.f;
                }
                sum2[0] = fadd2(sum2[0], pack_f2(x[0], x[1]));
                sum2[1] = fadd2(sum2[1], pack_f2(x[2], x[3]));
              }
            };
            if (c >= all && c + STEP <= hi && factor != 0.f) add(std::true_type());
            else add(std::false_type());
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_qfree(qs));
        }
        if (!ok) break;
        if (count > 1) {
          const int half = shared & 1, turn = shared >> 1;
          ++shared;
          if (!mine) {
            if (turn > 0) ok = warp_wait<18>(bar_partfree(half), (turn - 1) & 1, s_abort, status);
            if (!ok) break;
            s_part[half * 128 + t] = sum_of(sum2);
            mbar_arrive(bar_part(half));
            continue;
          }
          ok = warp_wait<19>(bar_part(half), turn & 1, s_abort, status);
          if (!ok) break;
          if (lane == 0) mbar_arrive(bar_keyfree(b));
          sum2[0] = pack_f2(sum_of(sum2), s_part[half * 128 + t]);
          sum2[1] = 0;
          mbar_arrive(bar_partfree(half));
        }
      }
      if (token < cap) p.out[at] = token < w.s.len ? (token < w.s.len - w.s.rows ? p.decay * old : 0.f) + (there ? sum_of(sum2) : 0.f) : 0.f;
    }
  } else if (warp < 16) {
    // ================= keys: a thread a token ==============================================================
    const int g = (warp >> 2) & 1, t = tid & 127;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    int keyed = 0;
    for (Walk w = walk_from<NR>(a, begin, end, s_next); !w.end && ok; walk_on<NR>(a, w, end, s_next)) {
      if (w.first >= w.images) continue;
      const int k = keyed++;
      if ((k & 1) != g) continue;
      const int rs = k % NRAW;
      const int token = w.j * kTileTokens + t;
      if (k >= 2) ok = warp_wait<23>(bar_keyfree(g), ((k >> 1) - 1) & 1, s_abort, status);
      if (ok) ok = warp_wait<24>(bar_raw(rs), (k / NRAW) & 1, s_abort, status);
      if (!ok) break;
      const bool there = token < w.s.len && (s_there[rs] >> (t / kBlockTokens) & 1);
      tc_fence_after();
      const uint8_t* raw = smem + C::kOffRaw + rs * C::kRaw;
      const float f = keys_to_tmem<D>(lane_addr + g * KeyCols<D>::kAll, raw + t / kBlockTokens * 8 * D, raw + C::kScales + t / kBlockTokens * 2 * D, t % kBlockTokens, there);
      s_factor[g * 128 + t] = there ? f : -1.f;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_rawfree(rs));
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(bar_key(g));
    }
  } else if (warp == 16) {
    // ================= products ============================================================================
    const bool el = elect_one();
    int images = 0, keyed = 0;
    for (Walk w = walk_from<NR>(a, begin, end, s_next); !w.end && ok; walk_on<NR>(a, w, end, s_next)) {
      if (w.first >= w.images) continue;
      const int b = keyed & 1;
      ok = warp_wait<25>(bar_key(b), (keyed >> 1) & 1, s_abort, status);
      ++keyed;
      for (int i = w.first; i < w.images && ok; ++i, ++images) {
        const int st = images % NS, qs = images % NQ;
        ok = warp_wait<26>(bar_q(qs), (images / NQ) & 1, s_abort, status);
        if (ok && images >= NS) ok = warp_wait<27>(bar_sfree(st), (images / NS - 1) & 1, s_abort, status);
        if (!ok) break;
        tc_fence_after();
        if (el) {
          scores_of_keys<D, NR>(tmem + C::kColS + st * NR, tmem + b * KeyCols<D>::kAll, ubase + C::kOffQ + qs * I::kBytes);
          umma_commit(bar_s(st));
          umma_commit(bar_qfree(qs));
          if (i + 1 == w.images) umma_commit(bar_keyfree(b));
        }
      }
    }
    __syncwarp();
  } else if (warp == 17) {
    // ================= copies of keys ======================================================================
    // A lane has a block of the next four tiles: its page is looked up before their turn comes.
    int keyed = 0;                                         // tiles that have been asked for
    Walk ahead = walk_from<NR>(a, begin, end, s_next);             // the first tile whose pages have not been looked up
    int left = 0, left1 = 0;                               // tiles that have been, of these four and the next
    struct Asked { int page, place; };                     // (the page's number is looked at when it is needed)
    auto look = [&](int& n) {
      Asked got = {-1, 0};
      n = 0;
#pragma unroll 1
      for (; n < 4 && !ahead.end; walk_on<NR>(a, ahead, end, s_next)) {
        if (ahead.first >= ahead.images) continue;
        if (lane / 8 == n) {
          const int token = ahead.j * kTileTokens + lane % 8 * kBlockTokens;
          if (token < ahead.s.len) {
            const int column = token / a.cache.page;
            got.place = ahead.head * subs + (token - column * a.cache.page) / kBlockTokens;
            got.page = a.table[(size_t)ahead.request * a.width + column];
          }
        }
        ++n;
      }
      return got;
    };
    Asked at0 = look(left), at1 = look(left1);
    while (ok && left > 0) {
      for (int n = 0; n < left; ++n, ++keyed) {
        const int rs = keyed % NRAW;
        const int page = __shfl_sync(0xffffffffu, at0.page, n * 8 + lane % 8), place = __shfl_sync(0xffffffffu, at0.place, n * 8 + lane % 8);
        const bool is = page >= 0 && page < a.cache.num_pages;
        const bool copies = lane < 8 && lane % p.run == 0 && is;
        const unsigned there = __ballot_sync(0xffffffffu, lane < 8 && is), runs = __ballot_sync(0xffffffffu, copies);
        if (keyed >= NRAW) ok = warp_wait<28>(bar_rawfree(rs), (keyed / NRAW - 1) & 1, s_abort, status);
        if (!ok) break;
        if (lane == 0) {
          s_there[rs] = there;
          mbar_arrive_expect(bar_raw(rs), __popc(runs) * p.run * C::kRawBlock);
        }
        __syncwarp();
        // (the blocks of a run that are beyond the request's tokens come along; a run has one page)
        if (copies) {
          const int row = page * a.cache.heads * subs + place;
          const uint32_t to = ubase + C::kOffRaw + rs * C::kRaw;
          tma_tile(to + lane * 8 * D, &maps.codes, 0, row, bar_raw(rs));
          tma_tile(to + C::kScales + lane * 2 * D, &maps.scales, 4 * D, row, bar_raw(rs));
        }
      }
      at0 = at1;
      left = left1;
      at1 = look(left1);
    }
    // nothing may be on its way into shared memory when the CTA ends
    for (int s = 0; s < NRAW && s < keyed; ++s) mbar_drain(bar_raw(s), ((keyed - 1 - s) / NRAW) & 1);
  } else {
    // ================= copies of images ====================================================================
    int images = 0;                                        // asked for
    for (Walk w = walk_from<NR>(a, begin, end, s_next); !w.end && ok; walk_on<NR>(a, w, end, s_next))
      for (int i = w.first; i < w.images && ok; ++i) {
        const int qs = images % NQ;
        if (images >= NQ) ok = warp_wait<29>(bar_qfree(qs), (images / NQ - 1) & 1, s_abort, status);
        if (!ok) break;
        if (lane == 0) {
          mbar_arrive_expect(bar_q(qs), I::kBytes);
          bulk_load(ubase + C::kOffQ + qs * I::kBytes, image_at(w, i), I::kBytes, bar_q(qs));
        }
        __syncwarp();
        ++images;
      }
    for (int s = 0; s < NQ && s < images; ++s) mbar_drain(bar_q(s), ((images - 1 - s) / NQ) & 1);
  }
  // ---- teardown ----
  tc_fence_before();
  __syncthreads();
  if (warp == 16) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// rows of an image: a product of 64 rows takes 48 clocks, of 128 rows 64; beside two tiles' keys of d = 128 TMEM has room for the scores of two images of 96
template <int D> constexpr int kImageRows = D == 64 ? 128 : 96;
// (what the few rows' kernels cannot count: all is for these)
Kinds weights_kinds(const hyperattn_weights_params& p, Kinds k) { return k.few && !few_rows_weights(p, k.many) ? Kinds{false, true} : k; }
long long slots_of(const hyperattn_weights_params& p, int least) {
  return image_slots(p.rows, p.requests, p.q_heads / p.cache.kv_heads, p.cache.d == 64 ? kImageRows<64> : kImageRows<128>, least) + 1;
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_cache_weights_workspace_bytes(const hyperattn_weights_params* p, size_t* bytes) {
  if (!bytes) return HYPERATTN_INVALID_ARGUMENT;
  if (int rc = check_chunk(p)) return rc;
  *bytes = 0;
  if (p->requests == 0) return HYPERATTN_OK;
  // (whatever a caller says about the most new tokens: without any word there are both kinds if there can be)
  const Kinds any = weights_kinds(*p, kinds_of(*p, 0));
  if (!any.many) return HYPERATTN_OK;
  const long long images = slots_of(*p, any.few ? most_of(*p) : -1) * p->cache.kv_heads;
  if (images > 0x7fffffffLL - 2 * kSms) return HYPERATTN_UNSUPPORTED_SHAPE;
  *bytes = (size_t)images * (p->cache.d == 64 ? Image<64, kImageRows<64>>::kBytes : Image<128, kImageRows<128>>::kBytes);
  return HYPERATTN_OK;
}

extern "C" int hyperattn_cache_weights(const hyperattn_weights_params* p) { return hyperattn_cache_weights_ex(p, 0); }

extern "C" int hyperattn_cache_weights_ex(const hyperattn_weights_params* p, int most_new) {
  size_t bytes = 0;
  if (most_new < 0) return HYPERATTN_INVALID_ARGUMENT;
  if (int rc = hyperattn_cache_weights_workspace_bytes(p, &bytes)) return rc;
  if (!p->cu_q && p->rows != p->requests) return HYPERATTN_INVALID_ARGUMENT;
  if (p->requests == 0) return HYPERATTN_OK;
  if ((p->rows && (!p->q || !p->lse)) || !p->weights_out || !p->table || !p->lengths || (bytes && !p->workspace)) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->q) || misaligned(p->weights) || misaligned(p->weights_out) || misaligned(p->workspace)) return HYPERATTN_MISALIGNED;
  if (p->workspace_bytes < bytes) return HYPERATTN_WORKSPACE_TOO_SMALL;
  const int subs = p->cache.page_tokens / kBlockTokens, d = p->cache.d;
  WeightArgs w = {chunk_args(*p), p->weights, p->weights_out, p->decay, subs % 8 == 0 ? 8 : subs & -subs};
  const Kinds kinds = weights_kinds(*p, kinds_of(*p, p->cu_q ? most_new : 1));
  KeyMaps maps;
  const long long blocks = (long long)p->cache.num_pages * p->cache.kv_heads * subs;
  if (kinds.many && (!encode_words_map(&maps.codes, p->cache.pages, blocks, 5 * d, 2 * d, w.run) || !encode_words_map(&maps.scales, p->cache.pages, blocks, 5 * d, d / 2, w.run))) return HYPERATTN_UNSUPPORTED_SHAPE;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  int* status = nullptr;
  if (int rc = device_status_word(st, &status)) return rc;
  int sms = 0;
  cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return status_of(e, "cache weights");
  if (kinds.few) {                               // (these write the zeros behind the tokens too)
    const int rc = launch_few_rows_weights(*p, kinds.many, status);
    if (rc || !kinds.many) return rc;
    w.c.least = most_of(*p);
  }
  auto go = [&](auto dim) {
    constexpr int D = decltype(dim)::value, NR = kImageRows<D>;
    using C = WCfg<D, NR>;
    cudaError_t e = allow_smem<weights_kernel<D, NR>>(C::kSmem);
    const int images = (int)(slots_of(*p, w.c.least) * p->cache.kv_heads);
    auto make = [&](auto kernel) { return launch(kernel, dim3((unsigned)images + (kinds.few ? 0 : 2 * kSms)), dim3(128), 0, st, w.c, p->lse, images, p->weights_out, kTileTokens); };
    if (e == cudaSuccess) e = p->dtype == HYPERATTN_BF16 ? make(image_kernel<D, NR, __nv_bfloat16>) : make(image_kernel<D, NR, __half>);
    const long long tiles = (long long)p->requests * p->cache.kv_heads * (((long long)p->table_width * p->cache.page_tokens + kTileTokens - 1) / kTileTokens);
    if (e == cudaSuccess) e = launch(weights_kernel<D, NR>, dim3((unsigned)(tiles < sms ? tiles : sms)), dim3(kWThreads), C::kSmem, st, w, maps, status);
    return status_of(e, "cache weights");
  };
  return d == 64 ? go(std::integral_constant<int, 64>()) : go(std::integral_constant<int, 128>());
}
