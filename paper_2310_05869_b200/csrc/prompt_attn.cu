// Exact attention over packed prompts with grouped heads, on the 5th-generation tensor cores.
//
// A work item is a key head and two neighbouring query tiles of a request.  A tile is 128 rows: 128 / G tokens with all G query heads
// that read the key head, so that the keys of a group are fetched once and a tile of many heads sees few keys in vain.  A
// CTA walks over the tiles of 128 keys from the last one that is seen down to the first:
//     S_i = Q_i K^T           tcgen05.mma, operands in 128B-swizzled shared memory (TMA boxes), S_i in TMEM
//     P_i = exp2(c S_i - m)   softmax warpgroup i, a thread a row; P_i in TMEM, in the inputs' type
//     O_i += P_i V            tcgen05.mma, P_i read from TMEM
// The tensor pipe works for one query tile while the other one's weights are made.  The reference m of a row is the maximum of its first
// tile (fp16: 2^7 below it, so that weights 2^-21 of the largest are still whole numbers of their type and down to 2^-32 are not nothing); it moves when a
// tile's weights sum to more than 2^15, and then O is multiplied in TMEM.  Tiles with keys that a row does not see are the first ones, so masks cost the
// later ones nothing.
//
// Values of keys that a row does not see are multiplied with zeros, which is not nothing where they are infinite or NaN.  In the tiles with such keys - of later tokens
// of the item, and beyond the request's end - infinities and NaN of keys that not all of its rows see are set to zero before they are multiplied, and the rows that do
// see them get them added at the end.
//
// Roundings: weights enter the products in the inputs' type (the tensor cores take both operands in one; a second term would be a second product), which is up to 2^-8 of each
// in bf16 and 2^-11 in fp16; sums of weights are taken before that, in fp32.  O is one chain of products over all keys, of whose sums the tensor cores cut up to 2^-23 each: within
// 2^-10 of a result at 131072 keys.
//
// What bounds it: at d = 128 the tensor pipe (64 % of its cycles) at the clock that the power limit leaves; 16384 tokens, 16 / 2 heads: 842 us, 1.3 PFLOP/s.  At d = 64 no unit
// is full (exponentials 57 %, issue 41 %, tensor pipe 32 %): two softmax warps a scheduler, each in one chain of loads, exponentials, stores and hand-overs; 6001
// tokens behind 5000 cached ones, 32 heads: 222 us, 0.6 PFLOP/s.  13 short prompts of 1021 tokens: 15.6 us, two items of a CTA one after the other.
//
// Warp roles (384 threads): 0-3 and 4-7 softmax and results of query tile 0 and 1, 8 issues the products (and allocates TMEM), 9 loads, 10 prepares items, 11 sees to
// values that are not finite.
// Every wait is bounded: a CTA that gives up raises the device status word, drains its copies, frees its TMEM and returns.
#include <climits>
#include <cstdio>
#include <type_traits>
#include "serving.cuh"
#include "tc_util.cuh"

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

// A lane's row at out[at]: the values that are not finite of keys key0 + from .. key0 + last (those that the row sees; none for last < from).  All lanes
// together: a lane looks at D / 32 coordinates of a key, and every row gathers, for each coordinate, whether there was an infinity of either sign (NaN: both).
template <int D, class T>
__device__ __noinline__ void add_unfinite(const PromptArgs& a, int kv, int key0, int from, int last, size_t at) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, end = __reduce_max_sync(0xffffffffu, last);
  const uint32_t* src = reinterpret_cast<const uint32_t*>(reinterpret_cast<const T*>(a.v) + (size_t)(key0 + from) * a.v_row + (size_t)kv * a.v_head) + lane * (E / 2);
  uint32_t up[E], down[E];
#pragma unroll
  for (int e = 0; e < E; ++e) up[e] = down[e] = 0;
#pragma unroll 4
  for (int key = from; key <= end; ++key, src += a.v_row / 2) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const float2 f = to_float2<T>(src[i]);
      const float x[2] = {f.x, f.y};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const unsigned p = __ballot_sync(0xffffffffu, !(x[e] < INFINITY)), m = __ballot_sync(0xffffffffu, !(x[e] > -INFINITY));
        if (key <= last) { up[2 * i + e] |= p; down[2 * i + e] |= m; }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    for (uint32_t any = up[e] | down[e]; any; any &= any - 1) {
      const int l = __ffs(any) - 1;
      const float x = (up[e] >> l & 1 ? INFINITY : 0.f) - (down[e] >> l & 1 ? INFINITY : 0.f);
      const size_t i = at * D + l * E + e;
      if (a.out_kind == HYPERATTN_FP32) reinterpret_cast<float*>(a.out)[i] += x;
      else reinterpret_cast<T*>(a.out)[i] = static_cast<T>(static_cast<float>(reinterpret_cast<T*>(a.out)[i]) + x);
    }
}

struct alignas(64) PromptMaps {
  CUtensorMap q, k, v;
};

constexpr int kTileRows = 128, kTileKeys = 128;
constexpr int kThreads = 384;
constexpr float kSumLimit = 32768.f;    // a tile whose weights sum to more has its reference moved (fp16 weights end at 2^16)
constexpr float kMostByArithmetic = 120.f;       // and one with a weight beyond 2 to that (which exp2_pair does not make; those up to it show in the sum)

template <int D>
struct Cfg {
  static constexpr uint32_t kSlab = 128 * 128;                         // 64 columns of 128 rows
  static constexpr uint32_t kTile = (D / 64) * kSlab;
  static constexpr int kStages = D == 64 ? 10 : 5;                     // tiles of K or V on their way
  static constexpr uint32_t kOffQ = 0, kOffRing = 2 * kTile, kOffMisc = kOffRing + kStages * kTile;
  static constexpr uint32_t kSmem = kOffMisc + 1024;
  // TMEM columns: S_0, S_1 (128 each), O_0, O_1; at d = 64 there is room for P_i beside S_i, so that the next scores do not wait for this tile's weights
  static constexpr bool kOwnP = D == 64;
  static constexpr uint32_t kColO = kOwnP ? 384 : 256, kStepO = kOwnP ? 64 : 128;
  static constexpr int kArithmetic = 8;                                // every so many-th pair of exponentials is made by arithmetic
  __host__ __device__ static constexpr uint32_t col_p(int i) { return kOwnP ? 256 + 64 * i : 128 * i; }
};

struct Item {
  int end;                               // no more items
  int row0;                              // first query row of the pair's first token
  int tokens[2];                         // tokens of either tile
  int tiles[2], most;                    // key tiles of either, of the longer one
  int key0, keys;                        // first key row, keys of the request
  int last;                              // last key that the pair's first token sees (may be negative)
  int kv;
  __device__ __forceinline__ int partly() const { return max(last + 1, 0); }                          // first key that not all rows see (from `keys` on: none does)
  __device__ __forceinline__ bool checked(int j) const { return (j + 1) * kTileKeys > partly(); }     // tile j has such keys
};

// Item `index`, decoded by a converged warp.  Items are ordered by request - of every 32 requests the one with most keys first - and in it from the last
// query on, so that the longest come first and little is left over at the end; key heads are next to each other.
__device__ __forceinline__ Item item_at(const PromptArgs& a, int index, int tile_tokens) {
  const int lane = threadIdx.x & 31;
  Item it = {};
  it.end = 1;
  if (index < 0) return it;
  const int block = index / a.kv_heads, pair_tokens = 2 * tile_tokens;
  it.kv = index - block * a.kv_heads;
  int before = 0;
  for (int r0 = 0; r0 < a.requests; r0 += 32) {
    int r = r0 + lane;
    int q0 = 0, nq = 0;
    if (a.requests > 1) {
      const int keys = r < a.requests ? a.cu_k[r + 1] - a.cu_k[r] : INT_MIN;
      int rank = 0, from = 0;
#pragma unroll
      for (int k = 0; k < 32; ++k) {
        const int other = __shfl_sync(0xffffffffu, keys, k);
        rank += other > keys || (other == keys && k < lane);
      }
#pragma unroll
      for (int k = 0; k < 32; ++k) from = __shfl_sync(0xffffffffu, rank, k) == lane ? k : from;
      r = r0 + from;
    }
    if (r < a.requests) {
      q0 = min(max(a.cu_q[r], 0), a.q_rows);
      nq = min(max(a.cu_q[r + 1], q0), a.q_rows) - q0;
    }
    const int mine = (nq + pair_tokens - 1) / pair_tokens;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, sum, o); if (lane >= o) sum += y; }
    const unsigned hit = __ballot_sync(0xffffffffu, before + sum > block);
    if (hit) {
      const int src = __ffs(hit) - 1;
      const int first = before + __shfl_sync(0xffffffffu, sum - mine, src), blocks = __shfl_sync(0xffffffffu, mine, src);
      q0 = __shfl_sync(0xffffffffu, q0, src);
      nq = __shfl_sync(0xffffffffu, nq, src);
      const int req = __shfl_sync(0xffffffffu, r, src), tok = (blocks - 1 - (block - first)) * pair_tokens;
      const int k0 = min(max(a.cu_k[req], 0), a.k_rows);
      it.end = 0;
      it.key0 = k0;
      it.keys = min(max(a.cu_k[req + 1], k0), a.k_rows) - k0;
      it.row0 = q0 + tok;
      it.last = a.causal ? min(it.keys - 1, tok + it.keys - nq) : it.keys - 1;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int left = nq - tok - i * tile_tokens;
        it.tokens[i] = min(max(left, 0), tile_tokens);
        const int seen = a.causal ? it.last + i * tile_tokens + it.tokens[i] : it.keys;       // keys that the tile's last token sees
        it.tiles[i] = it.tokens[i] > 0 && seen > 0 ? (min(seen, it.keys) + kTileKeys - 1) / kTileKeys : 0;
      }
      it.most = max(it.tiles[0], it.tiles[1]);
      return it;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return it;
}

template <class T> __device__ __forceinline__ constexpr uint32_t type_bits() { return sizeof(T) && std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u; }

// (NaN if one of them is)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// 2^x of two numbers up to 127 by arithmetic: x = n + f with n the nearest integer, 2^f by a polynomial of degree 4 (its coefficients a least-maximum
// fit of the relative error over -1/2 .. 1/2: 2.7e-6), n added to the exponent.  Below -125 x counts as that, and what it gives is taken off every result: zero for
// those, no difference to others.  (ZERO; where results become fp16 it is zero anyway, and sums do not show it.)  Above 2^127 the exponent does not hold n,
// so the caller looks at the largest x, which goes to `most` (NaN if one is).  The exponential unit makes 16 a clock and SM, which is what a tile of scores
// takes longest for; so some of them are made here.
template <bool ZERO>
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x2, float& most) {
  float x, y;
  unpack_f2(x2, x, y);
  most = max3(most, x, y);
  x2 = pack_f2(max3(x, -125.f, -125.f), max3(y, -125.f, -125.f));                       // (NaN stays, and becomes a huge number or NaN)
  const uint64_t t = fadd2(x2, pack_f2(12582912.f, 12582912.f));                      // 1.5 * 2^23 + n
  const uint64_t f = ffma2(fadd2(t, pack_f2(-12582912.f, -12582912.f)), pack_f2(-1.f, -1.f), x2);
  uint64_t p = ffma2(f, pack_f2(0.009570102207362652f, 0.009570102207362652f), pack_f2(0.05591786280274391f, 0.05591786280274391f));
  p = ffma2(f, p, pack_f2(0.240247443318367f, 0.240247443318367f));
  p = ffma2(f, p, pack_f2(0.6931217908859253f, 0.6931217908859253f));
  p = ffma2(f, p, pack_f2(0.9999992847442627f, 0.9999992847442627f));
  float p0, p1, t0, t1;
  unpack_f2(p, p0, p1);
  unpack_f2(t, t0, t1);
  const uint64_t w = pack_u2(__float_as_uint(p0) + (__float_as_uint(t0) << 23), __float_as_uint(p1) + (__float_as_uint(t1) << 23));
  constexpr float least = 0.9999992847442627f * 0x1p-125f;
  return ZERO ? fadd2(w, pack_f2(-least, -least)) : w;
}

// O of a row times alpha, in TMEM (rare).  All lanes together.
__device__ __noinline__ void rescale_o(uint32_t addr, int cols, float alpha) {
  uint32_t r[16];
  for (int c = 0; c < cols; c += 16) {
    tmem_ld16_issue(addr + c, r);
    tmem_ld16_wait(r);
#pragma unroll
    for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
    tmem_st16(addr + c, r);
  }
  tmem_wait_st();
}

template <int D, class T>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ PromptMaps maps, int group, int tile_tokens, int* status) {
  using C = Cfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t ubase = smem_u32(smem);
  Item* s_item = reinterpret_cast<Item*>(smem + C::kOffMisc);                    // [2]
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(smem + C::kOffMisc + 256);
  volatile int* s_abort = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 260);
  const uint32_t next0 = ubase + C::kOffMisc + 272, bar0 = next0 + 16;           // answer of next_index
  auto bar_item = [&](int set) { return bar0 + 8 * set; };                       // an item's description is written
  auto bar_itemfree = [&](int set) { return bar0 + 16 + 8 * set; };              // everybody is done with it
  const uint32_t bar_q = bar0 + 32, bar_qfree = bar0 + 40;                       // Q has landed; no product reads it any more
  auto bar_s = [&](int i) { return bar0 + 48 + 8 * i; };                         // S_i written
  auto bar_p = [&](int i) { return bar0 + 64 + 8 * i; };                         // P_i written
  auto bar_o = [&](int i) { return bar0 + 96 + 8 * i; };                         // O_i complete
  auto bar_ofree = [&](int i) { return bar0 + 112 + 8 * i; };                    // O_i read
  auto bar_sfree = [&](int i) { return bar0 + 128 + 8 * i; };                    // (P beside S) S_i read
  auto bar_pfree = [&](int i) { return bar0 + 144 + 8 * i; };                    // (P beside S) P_i multiplied
  const uint32_t bar_loaded = bar0 + 160, bar_next = bar0 + 168;                 // all loads of an item have been asked for; an answer has come
  auto bar_full = [&](int s) { return bar0 + 176 + 8 * s; };
  auto bar_empty = [&](int s) { return bar0 + 176 + 8 * (C::kStages + s); };
  auto bar_raw = [&](int s) { return bar0 + 176 + 8 * (2 * C::kStages + s); };   // values have landed that warp 11 checks before they are `full`
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

  // (a launch in which a wait gave up drains quickly; read before wait_for_stream() on purpose)
  if (tid == 0) *s_abort = *reinterpret_cast<volatile int*>(status);
  __syncthreads();
  if (*s_abort) return;
  __syncthreads();
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_item(i), 1);
      mbar_init(bar_itemfree(i), 256 + 3);
      mbar_init(bar_s(i), 1);
      mbar_init(bar_p(i), 128);
      mbar_init(bar_o(i), 1);
      mbar_init(bar_ofree(i), 128);
      mbar_init(bar_sfree(i), 128);
      mbar_init(bar_pfree(i), 1);
    }
    mbar_init(bar_q, 1);
    mbar_init(bar_qfree, 1);
    mbar_init(bar_loaded, 1);
    mbar_init(bar_next, 1);
    for (int s = 0; s < C::kStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); mbar_init(bar_raw(s), 1); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, *s_tmem, 0);
  wait_for_stream();
  // the number of a CTA that has not been launched and will not be, or -1 if there is none left
  auto next_index = [&](int& asked, int& index) {
    if (lane == 0)
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%1], 16;\n\t"
                   "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(next0), "r"(bar_next) : "memory");
    const bool ok = warp_wait<16>(bar_next, asked & 1, s_abort, status);
    ++asked;
    uint32_t x = 0, got = 0;
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b128 r;\n\tld.shared.b128 r, [%2];\n\tclusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\tselp.u32 %1, 1, 0, p;\n\t"
                 "mov.u32 %0, 0;\n\t@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n\t}" : "=r"(x), "=r"(got) : "r"(next0) : "memory");
    fence_async_smem();                                                    // (the next answer comes by the async proxy)
    __syncwarp();
    index = got ? (int)x : -1;
    return ok;
  };
  auto item_wait = [&](int it, auto site) { return warp_wait<decltype(site)::value>(bar_item(it & 1), (it >> 1) & 1, s_abort, status); };

  if (warp < 8) {
    // ================= softmax and results of query tile i: a thread a row =============================
    const int i = warp >> 2, row = tid & 127;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t scol = lane_addr + kTileKeys * i, pcol = lane_addr + C::col_p(i), ocol = lane_addr + C::kColO + C::kStepO * i;
    const int token = row / group, head = row - token * group;
    int done = 0;                        // key tiles of this query tile so far
    int items = 0;                       // items in which it had any
    bool ok = true;
    for (int it = 0; ok; ++it) {
      ok = item_wait(it, std::integral_constant<int, 0>{});
      if (!ok) break;
      const Item d = s_item[it & 1];
      if (d.end) break;
      const int tiles = i ? d.tiles[1] : d.tiles[0], tokens = i ? d.tokens[1] : d.tokens[0];
      const int tok = i * tile_tokens + token;                                   // in the pair
      const int limit = a.causal ? min(d.last + tok, d.keys - 1) : d.keys - 1;  // last key that the row sees
      const bool there = token < tokens && token < tile_tokens;                 // (other rows of the tile are other requests', or whatever shared memory held)
      const int least = a.causal ? min(d.last + i * tile_tokens, d.keys - 1) : d.keys - 1;       // the tile's first token
      float ref = -INFINITY;
      uint64_t sum2 = 0;
      for (int n = 0; n < tiles && ok; ++n) {
        const int j = tiles - 1 - n;
        ok = warp_wait<1>(bar_s(i), (done + n) & 1, s_abort, status);
        if (!ok) break;
        tc_fence_after();
        uint32_t r[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32_issue(scol + 32 * c, r[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32_wait(r[c]);
        if constexpr (C::kOwnP) {
          tc_fence_before();
          mbar_arrive(bar_sfree(i));
        }
        if (j * kTileKeys + kTileKeys - 1 > least) {
          const int rel = limit - j * kTileKeys;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (32 * c + e > rel) r[c][e] = 0xff800000u;
        }
        if constexpr (C::kOwnP) {
          if (done + n > 0) {                                              // the weights before these have been multiplied
            ok = warp_wait<13>(bar_pfree(i), (done + n - 1) & 1, s_abort, status);
            if (!ok) break;
            tc_fence_after();
          }
        }
        // The maximum is not taken of every tile: weights are made against the reference that the row has, and only where their sum shows that one of them may be
        // too large (or a score is not a number), or there is no reference yet, the maximum is taken, the reference moved to it, and the weights are made again -
        // in rows that need it: no row's result depends on which others it shares a warp with.
        constexpr float kBelow = std::is_same<T, __half>::value ? 7.f : 0.f;          // (128 weights of 2^7 are within the limit of a tile's sum)
        auto move_reference = [&](bool need) {
          float m[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            m[c] = max3(__uint_as_float(r[c][0]), __uint_as_float(r[c][1]), __uint_as_float(r[c][2]));
#pragma unroll
            for (int e = 3; e < 31; e += 2) m[c] = max3(m[c], __uint_as_float(r[c][e]), __uint_as_float(r[c][e + 1]));
            m[c] = max3(m[c], __uint_as_float(r[c][31]), __uint_as_float(r[c][31]));
          }
          const float top = max3(max3(m[0], m[1], m[2]), m[3], m[3]) * a.scale_log2 - kBelow;
          const bool move = need && top > ref;
          if (!__any_sync(0xffffffffu, move)) return;
          // (the products before this tile's are done - without P beside S because its scores came after them; the next one on O waits for this P)
          float alpha = 1.f;
          if (move) { alpha = ex2(ref - top); ref = top; }
          sum2 = fmul2(sum2, pack_f2(alpha, alpha));
          if (n > 0) rescale_o(ocol, D, alpha);
        };
        // (fp16: rows that saw few keys of their first tile are likely to be far below the second one's maximum, which leaves them 2^8 and not 2^15 - it is taken before the
        // weights are made for nothing.  6001 tokens in parts: 236 us without, 16 keys 229, 8 and 32 keys 230; 226 with a reference that is not below the maximum.)
        const bool first = there && (ref == -INFINITY || (std::is_same<T, __half>::value && n == 1 && limit - (j + 1) * kTileKeys < 16));
        if (__any_sync(0xffffffffu, first)) move_reference(first);
        const uint64_t sc2 = pack_f2(a.scale_log2, a.scale_log2);
        for (int attempt = 0;; ++attempt) {
          const float off = ref == -INFINITY ? 0.f : -ref;
          const uint64_t off2 = pack_f2(off, off);
          uint64_t tile2 = 0;
          float most = -INFINITY;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t p[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint64_t x2 = ffma2(pack_u2(r[c][2 * e], r[c][2 * e + 1]), sc2, off2);
              uint64_t w2;
              if (e % C::kArithmetic == C::kArithmetic - 1) w2 = exp2_pair<std::is_same<T, __nv_bfloat16>::value>(x2, most);
              else {
                float x, y;
                unpack_f2(x2, x, y);
                w2 = pack_f2(ex2(x), ex2(y));
              }
              tile2 = fadd2(tile2, w2);
              float x, y;
              unpack_f2(w2, x, y);
              p[e] = from_float2<T>(x, y);
            }
            tmem_st16(pcol + 16 * c, p);
          }
          float t0, t1;
          unpack_f2(tile2, t0, t1);
          const bool over = there && !(t0 + t1 <= kSumLimit && most <= kMostByArithmetic);
          if (attempt > 0 || !__any_sync(0xffffffffu, over)) {
            // (over it still: a score is no number, and the arithmetic has made one of it)
            if (attempt > 0 && !(most <= kMostByArithmetic)) tile2 = pack_f2(NAN, NAN);
            sum2 = fadd2(sum2, tile2);
            break;
          }
          move_reference(over);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(bar_p(i));
      }
      if (!ok) break;
      done += tiles;
      // ---- results ----
      float s0, s1;
      unpack_f2(sum2, s0, s1);
      const float sum = s0 + s1, inv = 1.f / sum;
      const bool none = ref == -INFINITY && sum == sum;                    // nothing was seen, or only scores of -infinity
      const size_t at = (size_t)(d.row0 + tok) * a.q_heads + d.kv * group + head;
      if (tiles > 0) {
        ok = warp_wait<2>(bar_o(i), items & 1, s_abort, status);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tmem_ld32_issue(ocol + 32 * c, o);
          tmem_ld32_wait(o);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = none ? 0u : __float_as_uint(__uint_as_float(o[e]) * inv);
          if (there) {
            if (a.out_kind == HYPERATTN_FP32) {
              float4* to = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at * D + 32 * c);
#pragma unroll
              for (int e = 0; e < 8; ++e)
                to[e] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
            } else {
              uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<T*>(a.out) + at * D + 32 * c);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = from_float2<T>(__uint_as_float(o[8 * e + 2 * k]), __uint_as_float(o[8 * e + 2 * k + 1]));
                to[e] = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          }
        }
        tc_fence_before();
        mbar_arrive(bar_ofree(i));
        ++items;
        if (there) a.lse[at] = none ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
      } else if (there) {
        a.lse[at] = -INFINITY;
        const int bytes = D * (a.out_kind == HYPERATTN_FP32 ? 4 : 2);
        for (int e = 0; e < bytes; e += 16) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(a.out) + at * bytes + e) = make_uint4(0, 0, 0, 0);
      }
      mbar_arrive(bar_itemfree(it & 1));
    }
  } else if (warp == 8) {
    // ================= products ============================================================================
    const bool el = elect_one();
    constexpr uint32_t idesc_s = (1u << 4) | type_bits<T>() | ((kTileKeys >> 3) << 17) | ((128u >> 4) << 24);
    constexpr uint32_t idesc_o = (1u << 4) | type_bits<T>() | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((128u >> 4) << 24);
    constexpr uint32_t desc_hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    const uint32_t dq_lo = ((ubase + C::kOffQ) >> 4) | (1u << 16);
    const uint32_t dk_lo = ((ubase + C::kOffRing) >> 4) | (1u << 16);
    const uint32_t dv_lo = ((ubase + C::kOffRing) >> 4) | ((C::kSlab >> 4) << 16);
    int ring = 0;                        // tiles of K and V before this item
    int done[2] = {0, 0}, items[2] = {0, 0}, qitems = 0;
    bool ok = true;
    for (int it = 0; ok; ++it) {
      ok = item_wait(it, std::integral_constant<int, 3>{});
      if (!ok) break;
      const Item& d = s_item[it & 1];
      auto uni = [&](int x) { return __shfl_sync(0xffffffffu, x, 0); };
      const bool end = uni(d.end) != 0;
      const int most = uni(d.most), tiles[2] = {uni(d.tiles[0]), uni(d.tiles[1])};
      __syncwarp();
      if (el) mbar_arrive(bar_itemfree(it & 1));
      if (end) break;
      if (most == 0) continue;
      ok = warp_wait<4>(bar_q, qitems & 1, s_abort, status);
      ++qitems;
      if (!ok) break;
      auto stage_of = [&](int j, int v) { return ring + 2 * (most - 1 - j) + v; };
      auto wait_tile = [&](int g) {
        if (ok) ok = warp_wait<5>(bar_full(g % C::kStages), (g / C::kStages) & 1, s_abort, status);
      };
      auto scores = [&](int i, int j) {
        const uint32_t k_lo = dk_lo + (uint32_t)(stage_of(j, 0) % C::kStages) * (C::kTile >> 4), q_lo = dq_lo + i * (C::kTile >> 4);
        if (el) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t step = ((ks >> 2) * C::kSlab + (ks & 3) * 32) >> 4;
            mma_ss2(tmem + kTileKeys * i, q_lo + step, k_lo + step, desc_hi, idesc_s, ks > 0);
          }
          umma_commit(bar_s(i));
        }
      };
      // scores of the first key tile
      wait_tile(stage_of(most - 1, 0));
      if (!ok) break;
      tc_fence_after();
      for (int i = 0; i < 2; ++i)
        if (tiles[i] == most) scores(i, most - 1);
      if (el) {
        umma_commit(bar_empty(stage_of(most - 1, 0) % C::kStages));
        if (most == 1) umma_commit(bar_qfree);
      }
      // O_i += P_i V of key tile j
      auto outputs = [&](int i, int j) {
        const uint32_t v_lo = dv_lo + (uint32_t)(stage_of(j, 1) % C::kStages) * (C::kTile >> 4);
        if (j == tiles[i] - 1 && items[i] > 0) ok = warp_wait<6>(bar_ofree(i), (items[i] - 1) & 1, s_abort, status);
        if (ok) ok = warp_wait<7>(bar_p(i), (done[i] + tiles[i] - 1 - j) & 1, s_abort, status);
        if (!ok) return;
        tc_fence_after();
        if (el) {
#pragma unroll
          for (int kk = 0; kk < kTileKeys / 16; ++kk)
            mma_ts2(tmem + C::kColO + C::kStepO * i, tmem + C::col_p(i) + kk * 8, v_lo + kk * (2048 >> 4), desc_hi, idesc_o, kk > 0 || j < tiles[i] - 1);
        }
        if (el) {
          if (C::kOwnP) umma_commit(bar_pfree(i));
          if (j == 0) umma_commit(bar_o(i));
        }
      };
      for (int j = most - 1; j >= 0 && ok; --j) {
        if constexpr (C::kOwnP) {
          // the next scores as soon as these have been read, then the products with V
          if (j > 0) {
            wait_tile(stage_of(j - 1, 0));
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (ok && j - 1 < tiles[i]) {
                if (j < tiles[i]) ok = warp_wait<14>(bar_sfree(i), (done[i] + tiles[i] - 1 - j) & 1, s_abort, status);
                if (!ok) break;
                tc_fence_after();
                scores(i, j - 1);
              }
            if (ok && el) {
              umma_commit(bar_empty(stage_of(j - 1, 0) % C::kStages));
              if (j == 1) umma_commit(bar_qfree);
            }
          }
          if (ok) wait_tile(stage_of(j, 1));
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (ok && j < tiles[i]) outputs(i, j);
          if (ok && el) umma_commit(bar_empty(stage_of(j, 1) % C::kStages));
        } else {
          wait_tile(stage_of(j, 1));
          if (j > 0) wait_tile(stage_of(j - 1, 0));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (ok && j < tiles[i]) outputs(i, j);
            if (ok && i == 1 && el) umma_commit(bar_empty(stage_of(j, 1) % C::kStages));
            if (ok && j > 0 && j - 1 < tiles[i]) scores(i, j - 1);
          }
          if (ok && j > 0 && el) {
            umma_commit(bar_empty(stage_of(j - 1, 0) % C::kStages));
            if (j == 1) umma_commit(bar_qfree);
          }
        }
      }
      ring += 2 * most;
      for (int i = 0; i < 2; ++i) { done[i] += tiles[i]; items[i] += tiles[i] > 0; }
    }
    __syncwarp();
  } else if (warp == 9) {
    // ================= loads ===============================================================================
    bool ok = true;
    int ring = 0, qitems = 0, armed = 0;           // armed: tiles that have been asked for
    uint32_t raw = 0, turns = 0;                   // by place in the ring: does the last one go through warp 11; parity of the next such one
    for (int it = 0; ok; ++it) {
      ok = item_wait(it, std::integral_constant<int, 8>{});
      if (!ok) break;
      const Item d = s_item[it & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_itemfree(it & 1));
      if (d.end) break;
      if (d.most == 0) {
        if (lane == 0) mbar_arrive(bar_loaded);
        continue;
      }
      if (qitems > 0) ok = warp_wait<9>(bar_qfree, (qitems - 1) & 1, s_abort, status);
      if (!ok) break;
      if (lane == 0) {
        const uint32_t bytes = (uint32_t)(tile_tokens * group) * 128u * (D / 64);
        mbar_expect_tx(bar_q, d.tokens[1] > 0 ? 2 * bytes : bytes);
        for (int i = 0; i < (d.tokens[1] > 0 ? 2 : 1); ++i)
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl)
            tma_heads_tile(ubase + C::kOffQ + i * C::kTile + sl * C::kSlab, &maps.q, sl * 64, d.kv * group, d.row0 + i * tile_tokens, bar_q);
        mbar_arrive(bar_q);
      }
      ++qitems;
      for (int n = 0; n < 2 * d.most && ok; ++n) {
        const int g = ring + n, s = g % C::kStages, j = d.most - 1 - (n >> 1);
        if (g >= C::kStages) ok = warp_wait<10>(bar_empty(s), (g / C::kStages - 1) & 1, s_abort, status);
        if (!ok) break;
        const uint32_t dst = ubase + C::kOffRing + s * C::kTile;
        const bool check = (n & 1) && d.checked(j);
        const uint32_t landed = check ? bar_raw(s) : bar_full(s);
        if (lane == 0) {
          mbar_expect_tx(landed, C::kTile);
#pragma unroll
          for (int sl = 0; sl < D / 64; ++sl)
            tma_heads_tile(dst + sl * C::kSlab, (n & 1) ? &maps.v : &maps.k, sl * 64, d.kv, d.key0 + j * kTileKeys, landed);
          mbar_arrive(landed);
        }
        armed = g + 1;
        raw = check ? raw | 1u << s : raw & ~(1u << s);
        turns ^= check ? 1u << s : 0u;
        __syncwarp();
      }
      if (lane == 0) mbar_arrive(bar_loaded);
      ring += 2 * d.most;
    }
    // nothing may be on its way into shared memory when the CTA ends
    for (int s = 0; s < C::kStages && s < armed; ++s)
      mbar_drain(raw >> s & 1 ? bar_raw(s) : bar_full(s), raw >> s & 1 ? ~(turns >> s) & 1 : ((armed - 1 - s) / C::kStages) & 1);
    if (qitems > 0) mbar_drain(bar_q, (qitems - 1) & 1);
  } else if (warp == 10) {
    // ================= items ===============================================================================
    // The grid has a CTA for every item that there can be.  A CTA that is done with its own takes the place of one that has not been launched (cluster launch
    // control), so that whoever is free takes the next item, in order; it asks when its loads of the present one are on their way, not earlier.
    bool ok = true;
    int asked = 0, index = blockIdx.x;
    for (int it = 0; ok; ++it) {
      Item d = item_at(a, index, tile_tokens);
      while (d.end && it > 0 && index >= 0 && ok) {                        // (numbers that are no item come last, and are taken out of the way)
        ok = next_index(asked, index);
        if (ok && index >= 0) d = item_at(a, index, tile_tokens);
      }
      if (ok && it >= 2) ok = warp_wait<11>(bar_itemfree(it & 1), ((it >> 1) - 1) & 1, s_abort, status);
      if (!ok) break;
      if (lane == 0) {
        s_item[it & 1] = d;
        mbar_arrive(bar_item(it & 1));
      }
      __syncwarp();
      if (d.end) break;
      ok = warp_wait<15>(bar_loaded, it & 1, s_abort, status);
      if (ok) ok = next_index(asked, index);
    }
    if (asked > 0) mbar_drain(bar_next, (asked - 1) & 1);
  } else {
    // ================= values that are not finite ==========================================================
    // (looked for while the weights of their tile are made)
    bool ok = true;
    int ring = 0;
    uint32_t turns = 0;                  // by place in the ring: parity of the next tile
    for (int it = 0; ok; ++it) {
      ok = item_wait(it, std::integral_constant<int, 17>{});
      if (!ok) break;
      const Item d = s_item[it & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_itemfree(it & 1));
      if (d.end) break;
      uint32_t add = 0;                  // some of keys that are seen
      for (int j = d.most - 1; j >= 0 && d.checked(j); --j) {
        const int s = (ring + 2 * (d.most - 1 - j) + 1) % C::kStages;
        ok = warp_wait<18>(bar_raw(s), turns >> s & 1, s_abort, status);
        if (!ok) break;
        turns ^= 1u << s;
        const int first = max(d.partly() - j * kTileKeys, 0), chunks = (kTileKeys - first) * 8, real = (d.keys - j * kTileKeys - first) * 8;     // (of 16 bytes, a slab)
        // an exponent of ones carries into the sign's place
        constexpr uint32_t kCarry = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
        auto bad_of = [&](uint32_t x) { return ((x & 0x7fff7fffu) + kCarry) & 0x80008000u; };
        uint32_t any = 0;
        for (int sl = 0; sl < D / 64; ++sl) {
          const uint4* at = reinterpret_cast<const uint4*>(smem + C::kOffRing + s * C::kTile + sl * C::kSlab + first * 128);
#pragma unroll 8
          for (int e = lane; e < chunks; e += 32) {
            const uint4 x = at[e];
            const uint32_t bad = bad_of(x.x) | bad_of(x.y) | bad_of(x.z) | bad_of(x.w);
            any |= bad;
            add |= e < real ? bad : 0u;
          }
        }
        if (__any_sync(0xffffffffu, any)) {
          for (int sl = 0; sl < D / 64; ++sl) {
            uint32_t* at = reinterpret_cast<uint32_t*>(smem + C::kOffRing + s * C::kTile + sl * C::kSlab + first * 128);
            for (int e = lane; e < 4 * chunks; e += 32) at[e] &= ~((bad_of(at[e]) >> 15) * 0xffffu);
          }
          fence_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_full(s));
      }
      ring += 2 * d.most;
      if (!ok || !__any_sync(0xffffffffu, add)) continue;
      ok = warp_wait<19>(bar_itemfree(it & 1), (it >> 1) & 1, s_abort, status);                // the results have been written
      if (!ok) break;
      for (int r = 0; r < 2 * kTileRows; r += 32) {
        const int i = r / kTileRows, row = r % kTileRows + lane, token = row / group, tok = i * tile_tokens + token;
        const size_t at = (size_t)(d.row0 + tok) * a.q_heads + d.kv * group + row - token * group;
        // (a row without weights stays zero)
        const bool sees = token < min(i ? d.tokens[1] : d.tokens[0], tile_tokens) && a.lse[at] != -INFINITY;
        add_unfinite<D, T>(a, d.kv, d.key0, d.partly(), sees ? min(a.causal ? d.last + tok : d.keys - 1, d.keys - 1) : -1, at);
      }
    }
  }

  // ---- teardown ----
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <int D, class T>
cudaError_t run_prompt(const PromptArgs& a, const PromptMaps& maps, int group, int tile_tokens, int* status, cudaStream_t st) {
  cudaError_t e = allow_smem<prompt_kernel<D, T>>(Cfg<D>::kSmem);
  if (e != cudaSuccess) return e;
  const long long items = ((long long)a.q_rows / (2 * tile_tokens) + a.requests) * a.kv_heads;       // at most
  if (items > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch(prompt_kernel<D, T>, dim3((unsigned)items), dim3(kThreads), Cfg<D>::kSmem, st, a, maps, group, tile_tokens, status);
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
    if (bad_stride(s) || s == 0) return HYPERATTN_UNSUPPORTED_SHAPE;
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
  const int group = p->q_heads / p->kv_heads, tile_tokens = kTileRows / group;
  const bool bf16 = p->dtype == HYPERATTN_BF16;
  PromptMaps maps;
  // (the stride of an axis of one entry does not matter, but has to be one; without keys the maps of K and V are not used)
  auto map = [&](CUtensorMap* m, const void* base, int rows, long long row, int heads, long long head, int box_rows, int box_heads) {
    return encode_heads_map(m, base, bf16, rows, rows > 1 ? row : (long long)heads * p->d, heads, heads > 1 ? head : p->d, p->d, box_rows, box_heads);
  };
  const bool keys = p->k_rows > 0;
  if (!map(&maps.q, p->q, p->q_rows, p->q_row_stride, p->q_heads, p->q_head_stride, tile_tokens, group) ||
      !map(&maps.k, keys ? p->k : p->q, keys ? p->k_rows : 1, p->k_row_stride, p->kv_heads, keys ? p->k_head_stride : p->d, kTileKeys, 1) ||
      !map(&maps.v, keys ? p->v : p->q, keys ? p->k_rows : 1, p->v_row_stride, p->kv_heads, keys ? p->v_head_stride : p->d, kTileKeys, 1))
    return HYPERATTN_UNSUPPORTED_SHAPE;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  int* status = nullptr;
  if (int rc = device_status_word(st, &status)) return rc;
  cudaError_t e;
  if (p->d == 64) e = bf16 ? run_prompt<64, __nv_bfloat16>(a, maps, group, tile_tokens, status, st) : run_prompt<64, __half>(a, maps, group, tile_tokens, status, st);
  else e = bf16 ? run_prompt<128, __nv_bfloat16>(a, maps, group, tile_tokens, status, st) : run_prompt<128, __half>(a, maps, group, tile_tokens, status, st);
  if (e == cudaSuccess) return HYPERATTN_OK;
  std::fprintf(stderr, "hyperattn: prompt attention failed: %s\n", cudaGetErrorString(e));
  return HYPERATTN_CUDA_ERROR;
}
