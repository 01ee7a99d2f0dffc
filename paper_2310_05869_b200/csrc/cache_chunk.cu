// Attention of several new tokens a request over the paged 4-bit cache, on the 5th-generation tensor cores.
//
// A segment is a request, a key head and 256 of its rows (tokens times the query heads that read the key head), in two units of 128.  A CTA walks over tiles of 64
// tokens, from the first one up:
//     K = (scale * code, what its rounding has lost, minimum), V = minimum + scale * code      from the cache's bytes to shared memory, by four warps for every other tile
//     S_i = Q_i K^T           tcgen05.mma, queries from TMEM; exact products (cache_tiles.cuh)
//     P_i = exp2(c S_i - m)   four warps a unit, a thread a row; P_i in TMEM, fp16
//     O_i += P_i V            tcgen05.mma
// The tensor pipe works for one unit while the other one's weights are made.  A segment of up to 128 rows has both units work for them, on every other tile each; unit 0's
// warps put the two results together (a lane of TMEM is the same row in both).  References move as in the attention of prompts (softmax.cuh); weights' references are 2^7 below
// the largest score.  K's scales and minima are multiplied by a power of two for their tile, V's by one that is a multiple of four octaves; a tile with larger values than O's has O multiplied, one with
// smaller ones its weights, so values of any size are as exact as any others.
//
// A NaN among a token's values becomes zero (0 * NaN would reach rows that do not see it), and the first such token of each group of 32 coordinates is kept: rows that see
// it get NaN there at the end.
//
// The tiles of all segments are one sequence, cut into equal parts, one for each CTA (a first launch of one CTA finds the cuts); pieces of segments that lie in several parts
// go to the workspace, and a last launch puts them together, in order.
//
// Roundings: weights and values enter the second product as fp16 (2^-11 of each), sums of weights before that; O is a chain of products over 96 or 512 tiles at most (kChain).  With fp16 queries, or fp32 results, what the weights'
// rounding has lost goes through the product too (results off by 2.8e-4 instead of 3.5e-4 of their size, where rounding them alone is 2.1e-4; 5 requests, 1501 rows 161 -> 200 us when
// that was added; bf16 results, 1.7e-3, do not show it).
//
// What bounds it: a tile of 64 tokens and 256 rows takes about 2300 clocks, near which lie its conversion, its 42 products (d = 128; half of those for scores are what exact keys cost) and the
// hand-overs of the softmax.  2048 rows over 30720 tokens, 32 / 8 heads of 128: 1261 us for a floor of 636 (tensor pipe 62 %, issue 56 %); 5 requests, 1501 rows over up to 5393 tokens, 32 heads
// of 64, fp16: 181 us (tensor pipe 36 %, issue 57 %), of which the first and the last launch take 10.  Two halves of a row block of up to 128 rows: 64 rows over 8000 tokens, 32 heads of 64, 8
// requests 297 -> 242 us.
//
// Warp roles (640 threads): 0-3 and 4-7 softmax and results of unit 0 and 1, 8-11 and 12-15 keys and values of even and odd tiles, 16 products (and TMEM), 17 copies, 18 segments, 19
// nothing (four warps give registers up together).
// Every wait is bounded: a CTA that gives up raises the device status word, drains its copies, frees its TMEM and returns.
#include <climits>
#include <type_traits>
#include "cache_rows.cuh"
#include "cache_tiles.cuh"
#include "softmax.cuh"

namespace hyperattn {
namespace {

constexpr int kUnitRows = 128, kBlockRows = 256, kKeys = 64, kCThreads = 640;
// Tiles of a unit's chain of products, at most.  The tensor cores cut their sums, always downwards, by 1.2 2^-23 of the partial sum for every 16 products on average: values of one sign came out 6e-4 too
// small after one chain over 131072 tokens, three times what rounding to fp16 does.  After chains of 96 tiles (6144 tokens) whose results are added in fp32 they are 4.3e-5 too small, after 512 tiles
// 1.4e-4, a twelfth of what rounding to bf16 does: that for bf16 results, which so hardly ever pay for it.  A longer segment is several pieces in a row; what they give is added up at the segment's place in
// the workspace, a thread its row.  us of 2048 rows over 30720 tokens, 32 / 8 heads of 128: without a limit 1267, 128 tiles 1314, 96 1348, 64 1396 (some 20 000 clocks a piece, in which
// nothing is multiplied).
template <bool FINE> constexpr int kChain = FINE ? 96 : 512;

struct ChunkOut {
  void* out;
  float* lse;
  int out_kind;
  // of the workspace
  long long* before;                     // [slots + 1] cost of the row blocks (of all key heads) before each
  int2* block;                           // [slots] request and row block, -1: none
  long long* start;                      // [parts + 1] where a part starts
  float4* part_o;                        // [2 parts][d / 4][256] pieces of outputs, by place
  float2* part_s;                        // [2 parts][256] their references and sums
  int slots, parts;
};
// a row block's rows, its 64-token tiles and what one costs
struct RowBlock { int row0, rows, tiles, cost; };
__device__ __forceinline__ RowBlock row_block(const ChunkArgs& a, const Span& s, int b) {
  const int group = a.q_heads / a.cache.heads;
  RowBlock k;
  k.row0 = b * kBlockRows;
  k.rows = min(s.rows * group - k.row0, kBlockRows);
  const int seen = a.causal ? s.len - s.rows + (k.row0 + k.rows - 1) / group + 1 : s.len;      // of the last row
  k.tiles = seen > 0 ? (min(seen, s.len) + kKeys - 1) / kKeys : 0;
  k.cost = k.rows > kUnitRows ? 5 : 3;
  return k;
}

constexpr int kShareThreads = 1024;
__global__ void __launch_bounds__(kShareThreads) share_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkOut o) {
  __shared__ long long s_warp[kShareThreads / 32];
  wait_for_stream();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = a.q_heads / a.cache.heads;
  for (int i = tid; i < o.slots; i += kShareThreads) o.block[i] = make_int2(-1, 0);
  __syncthreads();
  for (int r = warp; r < a.requests; r += kShareThreads / 32) {
    const Span s = span_of(a, r);
    const int blocks = is_for(a, s) ? (int)(((long long)s.rows * group + kBlockRows - 1) / kBlockRows) : 0;
    const long long first = image_slots(s.first, r, group, kBlockRows, a.least);
    for (int b = lane; b < blocks; b += 32) o.block[first + b] = make_int2(r, b);
  }
  __syncthreads();
  long long total = 0;
  for (int i0 = 0; i0 < o.slots; i0 += kShareThreads) {
    const int i = i0 + tid;
    long long cost = 0;
    if (i < o.slots) {
      const int2 x = o.block[i];
      if (x.x >= 0) {
        const RowBlock k = row_block(a, span_of(a, x.x), x.y);
        cost = (long long)k.tiles * k.cost * a.cache.heads;
      }
    }
    long long run = cost;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) { const long long y = __shfl_up_sync(0xffffffffu, run, d); if (lane >= d) run += y; }
    if (lane == 31) s_warp[warp] = run;
    __syncthreads();
    long long ahead = total + run - cost;
    for (int w = 0; w < kShareThreads / 32; ++w) { if (w < warp) ahead += s_warp[w]; total += s_warp[w]; }
    if (i < o.slots) o.before[i] = ahead;
    __syncthreads();
  }
  if (tid == 0) o.before[o.slots] = total;
  __syncthreads();
  const long long share = total / o.parts, extra = total % o.parts;
  for (int c = tid; c <= o.parts; c += kShareThreads) {
    long long x = share * c + min((long long)c, extra);
    if (x < total) {
      int lo = 0, hi = o.slots;                        // the last block that starts there or before (one with tiles: the ones after it start where it ends)
      while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (o.before[mid] <= x) lo = mid; else hi = mid; }
      const int2 b = o.block[lo];
      const RowBlock k = row_block(a, span_of(a, b.x), b.y);
      x = o.before[lo] + (x - o.before[lo] + k.cost - 1) / k.cost * k.cost;
    }
    o.start[c] = x;
  }
}

template <int D>
struct CCfg {
  static constexpr uint32_t kKeySlab = kKeys * 128, kP = (D / 64) * kKeySlab;                       // 64 columns of 64 tokens; scale * code of a tile
  static constexpr uint32_t kOffRest = kP, kOffV = 2 * kP, kOffMinima = kOffV + D * 128, kStage = kOffMinima + kKeys * 32;
  static constexpr int kStages = D == 128 ? 3 : 5, kRawStages = D == 128 ? 6 : 8;        // (even: a slot is the same group's every time)
  static constexpr uint32_t kRaw = 4 * Block<D>::kBytes, kSums = kUnitRows * 32;
  static constexpr uint32_t kOffRaw = kStages * kStage, kOffSums = kOffRaw + kRawStages * kRaw, kOffMisc = kOffSums + 2 * kSums;
  static constexpr uint32_t kSmem = kOffMisc + 1024 + 2048 + 1024;
  // TMEM columns: O_0, O_1, Q_0, Q_1, S_0, S_1; at d = 64 P_i beside S_i, so that the next scores do not wait for this tile's weights
  static constexpr bool kOwnP = D == 64;
  static constexpr uint32_t kColQ = 2 * D, kColS = 3 * D;
  __host__ __device__ static constexpr uint32_t col_p(int i) { return kColS + (kOwnP ? 2 * kKeys : 0) + kKeys * i; }
  static constexpr uint32_t kRest = kKeys / 2;                                   // (from P on: what its rounding has lost)
};

struct Piece {                           // of a segment, in a CTA's part
  int end;
  int request, kv, row0, units[2];       // rows of either unit
  Span s;
  int tile0, tile1;
  int split;                             // both units have the same rows, and every other tile
  int place;                             // in the workspace
  int begun, more, last;                 // the CTA had the segment's piece before this one, whose results are at that place; it has the next one; the segment is finished here
  __device__ __forceinline__ int last_seen(const ChunkArgs& a, int row) const {       // last token that a row of the segment sees
    const int token = (row0 + row) / (a.q_heads / a.cache.heads);
    return a.causal ? min(s.len - s.rows + token, s.len - 1) : s.len - 1;
  }
};

// FINE: what rounding the weights to fp16 has lost goes through the product too
template <int D, class T, bool FINE>
__global__ void __launch_bounds__(kCThreads, 1) chunk_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkOut o, int run, int* status) {
  using C = CCfg<D>;
  using B = Block<D>;
  constexpr int G = D / kGroup, NS = C::kStages, NRAW = C::kRawStages;
  constexpr int kAtOnce = FINE ? 16 : 32;        // weights that go to TMEM at a time (their number and the scores, which may be needed once more, are what registers hold)
  extern __shared__ uint8_t smem_[];
  uint8_t* smem = smem_ + (1024 - (smem_u32(smem_) & 1023)) % 1024;
  const uint32_t ubase = smem_u32(smem);
  uint8_t* misc = smem + C::kOffMisc;
  Piece* s_piece = reinterpret_cast<Piece*>(misc);                               // [2]
  int* s_nan = reinterpret_cast<int*>(misc + 192);                               // [2][4] first token with a NaN among the values of a group
  int* s_exp = reinterpret_cast<int*>(misc + 224);                               // [2][2][4] the blocks' exponents, of even and odd tiles
  uint32_t* s_there = reinterpret_cast<uint32_t*>(misc + 288);                   // [kRawStages] which of a tile's blocks are in the cache
  float4* s_tile = reinterpret_cast<float4*>(misc + 320);                        // [kStages] factor of the scores, octaves that V is multiplied by, blocks
  float4* s_merge = reinterpret_cast<float4*>(misc + 1024);                      // [128] split: reference, sum and octaves of unit 1's rows
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc + 400);
  volatile int* s_abort = reinterpret_cast<volatile int*>(misc + 404);
  const uint32_t bar0 = ubase + C::kOffMisc + 408;
  auto bar_piece = [&](int set) { return bar0 + 8 * set; };
  auto bar_piecefree = [&](int set) { return bar0 + 16 + 8 * set; };
  auto bar_q = [&](int i) { return bar0 + 32 + 8 * i; };                         // Q_i is in TMEM
  auto bar_qfree = [&](int i) { return bar0 + 48 + 8 * i; };
  auto bar_s = [&](int i) { return bar0 + 64 + 8 * i; };                         // S_i written
  auto bar_p = [&](int i) { return bar0 + 80 + 8 * i; };                         // P_i written
  auto bar_o = [&](int i) { return bar0 + 96 + 8 * i; };                         // O_i complete
  auto bar_ofree = [&](int i) { return bar0 + 112 + 8 * i; };                    // O_i read
  auto bar_sfree = [&](int i) { return bar0 + 128 + 8 * i; };                    // (P beside S) S_i read
  auto bar_pfree = [&](int i) { return bar0 + 144 + 8 * i; };                    // (P beside S) P_i multiplied
  auto bar_op = [&](int s) { return bar0 + 160 + 8 * s; };                       // a tile's operands are there
  auto bar_opfree = [&](int s) { return bar0 + 160 + 8 * (NS + s); };
  auto bar_raw = [&](int s) { return bar0 + 160 + 8 * (2 * NS + s); };
  auto bar_rawfree = [&](int s) { return bar0 + 160 + 8 * (2 * NS + NRAW + s); };
  const uint32_t bar_merge = bar0 + 160 + 8 * (2 * NS + 2 * NRAW);               // split: unit 1's references and sums are there
  static_assert(408 + 160 + 8 * (2 * NS + 2 * NRAW + 1) <= 1024 && sizeof(Piece) <= 96, "room for the barriers");
  const int tid = threadIdx.x, lane = tid & 31;
  const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) *s_abort = *reinterpret_cast<volatile int*>(status);
  __syncthreads();
  if (*s_abort) {
    wait_for_stream();                                 // (the last launch reads what the first one wrote: this one may not be over before it)
    return;
  }
  __syncthreads();
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_piece(i), 1);
      mbar_init(bar_piecefree(i), 256 + 8 + 2);
      mbar_init(bar_q(i), 128); mbar_init(bar_qfree(i), 1);
      mbar_init(bar_s(i), 1); mbar_init(bar_p(i), 128);
      mbar_init(bar_o(i), 1); mbar_init(bar_ofree(i), 128);
      mbar_init(bar_sfree(i), 128); mbar_init(bar_pfree(i), 1);
    }
    mbar_init(bar_merge, 128);
    for (int s = 0; s < NS; ++s) { mbar_init(bar_op(s), 128); mbar_init(bar_opfree(s), 1); }
    for (int s = 0; s < NRAW; ++s) { mbar_init(bar_raw(s), 1); mbar_init(bar_rawfree(s), 4); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __reduce_max_sync(0xffffffffu, *s_tmem);      // (in a uniform register, as the products want their operands)
  wait_for_stream();
  const int group = a.q_heads / a.cache.heads, subs = a.cache.page / kBlockTokens;
  auto piece_wait = [&](int it, auto site) { return warp_wait<decltype(site)::value>(bar_piece(it & 1), (it >> 1) & 1, s_abort, status); };

  // Registers: 96 a thread at launch; 136 for the softmax, 80 for keys and values, 48 for the others (together as many).
  if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
  else if (warp < 16) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");

  if (warp < 8) {
    // ================= softmax and results of unit i: a thread a row =======================================
    const int i = warp >> 2, row = tid & 127;
    const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t scol = lane_addr + C::kColS + kKeys * i, pcol = lane_addr + C::col_p(i), ocol = lane_addr + D * i, qcol = lane_addr + C::kColQ + (D / 2) * i;
    int done = 0, pieces = 0, tiles = 0;       // tiles of this unit, pieces with rows of it, tiles of the CTA so far
    int others = 0, splits = 0, loaded = 0;    // pieces with rows of unit 1, that were split; queries that this unit has had
    float scale = 0.f;
    bool ok = true;
    for (int it = 0; ok; ++it) {
      ok = piece_wait(it, std::integral_constant<int, 0>{});
      if (!ok) break;
      const Piece d = s_piece[it & 1];
      if (d.end) break;
      const int all = d.tile1 - d.tile0, rows = i && !d.split ? d.units[1] : d.units[0];
      const int from = d.split ? i : 0, step = d.split ? 2 : 1, count = (all - from + step - 1) / step, base = d.split ? 0 : i * kUnitRows;       // its tiles; its first row
      if (rows > 0) {
        const bool there = row < rows;
        const int in_block = base + row, token = (d.row0 + in_block) / group, head = d.row0 + in_block - token * group;
        const int limit = there ? d.last_seen(a, in_block) : -1;               // last token that the row sees
        const int least = d.last_seen(a, base);                                // the unit's first row
        const size_t at = (size_t)(d.s.first + token) * a.q_heads + d.kv * group + head;
        // ---- the row's query (that of the piece before is there still) ----
        if (!d.begun) {
          uint32_t raw[D / 2];
          const T* from = reinterpret_cast<const T*>(a.q) + (long long)(d.s.first + token) * a.q_row + (long long)(d.kv * group + head) * a.q_head;
#pragma unroll
          for (int c = 0; c < D / 8; ++c) {
            const uint4 v = there ? reinterpret_cast<const uint4*>(from)[c] : make_uint4(0, 0, 0, 0);
            raw[4 * c] = v.x; raw[4 * c + 1] = v.y; raw[4 * c + 2] = v.z; raw[4 * c + 3] = v.w;
          }
          float top = 0.f;
#pragma unroll
          for (int c = 0; c < D / 2; ++c) { const float2 f = to_float2<T>(raw[c]); top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y))); }
          // (as for the images in cache_tiles.cuh)
          int e = (int)(__float_as_uint(top) >> 23) - 127 - 9;
          e = top == 0.f || !(top < INFINITY) ? 0 : min(max(e, -126), 126);
          const float down = __uint_as_float((uint32_t)(127 - e) << 23);
          scale = __uint_as_float((uint32_t)(127 + e) << 23) * a.scale_log2;
          uint32_t sums[8] = {};
          float parts[3][G];
#pragma unroll
          for (int g = 0; g < G; ++g) {
            float sum = 0.f;
#pragma unroll
            for (int c = 16 * g; c < 16 * g + 16; ++c) {
              const float2 f = to_float2<T>(raw[c]);
              raw[c] = from_float2<__half>(f.x * down, f.y * down);
              const float2 r = to_float2<__half>(raw[c]);
              sum += r.x + r.y;
            }
            parts[0][g] = __half2float(__float2half_rn(sum));
            parts[1][g] = __half2float(__float2half_rn(sum - parts[0][g]));
            parts[2][g] = sum - parts[0][g] - parts[1][g];
          }
#pragma unroll
          for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int g = 0; g < G; g += 2) sums[(p * G + g) / 2] = from_float2<__half>(parts[p][g], parts[p][g + 1]);
          if (loaded > 0) ok = warp_wait<1>(bar_qfree(i), (loaded - 1) & 1, s_abort, status);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < D / 2; c += 16) {
            uint32_t w[16];
#pragma unroll
            for (int x = 0; x < 16; ++x) w[x] = raw[c + x];
            tmem_st16(qcol + c, w);
          }
          uint8_t* to = smem + C::kOffSums + i * C::kSums;
          *reinterpret_cast<uint4*>(to + row * 16) = make_uint4(sums[0], sums[1], sums[2], sums[3]);
          *reinterpret_cast<uint4*>(to + (kUnitRows + row) * 16) = make_uint4(sums[4], sums[5], sums[6], sums[7]);
          tmem_wait_st();
          fence_async_smem();
          tc_fence_before();
          mbar_arrive(bar_q(i));
          ++loaded;
        }
        float ref = -INFINITY;
        uint64_t sum2 = 0;
        int lift = 127;                                                        // octaves that O's values are multiplied by (none yet)
        for (int n = 0; n < count && ok; ++n) {
          const int tile_n = from + n * step, key0 = (d.tile0 + tile_n) * kKeys, st = (tiles + tile_n) % NS;
          ok = warp_wait<3>(bar_s(i), (done + n) & 1, s_abort, status);
          // (the tile's operands were there for its scores; this thread sees what was written beside them.  Not before: a unit that has had no rows may be phases behind)
          if (ok) ok = warp_wait<2>(bar_op(st), ((tiles + tile_n) / NS) & 1, s_abort, status);
          if (!ok) break;
          const float4 tile = s_tile[st];
          tc_fence_after();
          uint32_t r[2][32];
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_ld32_issue(scol + 32 * c, r[c]);
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_ld32_wait(r[c]);
          if constexpr (C::kOwnP) {
            tc_fence_before();
            mbar_arrive(bar_sfree(i));
          }
          const uint32_t blocks = __float_as_uint(tile.z);
          if (key0 + kKeys - 1 > least || blocks != 15u) {
            const int rel = limit - key0;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (32 * c + e > rel || !(blocks >> (2 * c + e / 16) & 1)) r[c][e] = 0xff800000u;
          }
          if constexpr (C::kOwnP) {
            if (done + n > 0) {
              ok = warp_wait<4>(bar_pfree(i), (done + n - 1) & 1, s_abort, status);
              if (!ok) break;
              tc_fence_after();
            }
          }
          const float scale_log2 = scale * tile.x;
          // V's octaves: smaller than O's so far: O follows; larger: this tile's weights do
          const int mine = __float_as_int(tile.y);
          if (mine < lift) {
            if (n > 0) rescale_o(ocol, D, exp2f((float)(mine - lift)));
            lift = mine;
          }
          const float less = (float)(mine - lift);                            // octaves that weights are smaller by
          constexpr float kBelow = 7.f;                                        // (as for fp16 prompts)
          auto move_reference = [&](bool need) {
            float m[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              m[c] = max3(__uint_as_float(r[c][0]), __uint_as_float(r[c][1]), __uint_as_float(r[c][2]));
#pragma unroll
              for (int e = 3; e < 31; e += 2) m[c] = max3(m[c], __uint_as_float(r[c][e]), __uint_as_float(r[c][e + 1]));
              m[c] = max3(m[c], __uint_as_float(r[c][31]), __uint_as_float(r[c][31]));
            }
            const float top = max3(m[0], m[1], m[1]) * scale_log2 - kBelow;
            const bool move = need && top > ref;
            if (!__any_sync(0xffffffffu, move)) return;
            float alpha = 1.f;
            if (move) { alpha = ex2(ref - top); ref = top; }
            sum2 = fmul2(sum2, pack_f2(alpha, alpha));
            if (n > 0) rescale_o(ocol, D, alpha);
          };
          const bool first = there && ref == -INFINITY;
          if (__any_sync(0xffffffffu, first)) move_reference(first);
          const uint64_t sc2 = pack_f2(scale_log2, scale_log2);
          for (int attempt = 0;; ++attempt) {
            const float off = (ref == -INFINITY ? 0.f : -ref) - less;
            const uint64_t off2 = pack_f2(off, off);
            uint64_t tile2 = 0;
#pragma unroll
            for (int c = 0; c < 64 / kAtOnce; ++c) {
              uint32_t p[kAtOnce / 2], rest[kAtOnce / 2];
#pragma unroll
              for (int e = 0; e < kAtOnce / 2; ++e) {
                const int at = kAtOnce * c + 2 * e;
                const uint64_t x2 = ffma2(pack_u2(r[at / 32][at % 32], r[at / 32][at % 32 + 1]), sc2, off2);
                float x, y;
                unpack_f2(x2, x, y);
                x = ex2(x);
                y = ex2(y);
                tile2 = fadd2(tile2, pack_f2(x, y));
                p[e] = from_float2<__half>(x, y);
                if constexpr (FINE) {
                  const float2 r2 = to_float2<__half>(p[e]);
                  rest[e] = from_float2<__half>(x - r2.x, y - r2.y);
                }
              }
              if constexpr (FINE) {
                tmem_st8(pcol + kAtOnce / 2 * c, p);
                tmem_st8(pcol + C::kRest + kAtOnce / 2 * c, rest);
              } else tmem_st16(pcol + kAtOnce / 2 * c, p);
            }
            float t0, t1;
            unpack_f2(tile2, t0, t1);
            const bool over = there && !(t0 + t1 <= kSumLimit);
            if (attempt > 0 || !__any_sync(0xffffffffu, over)) {
              const float back = exp2f(less);
              sum2 = ffma2(tile2, pack_f2(back, back), sum2);
              break;
            }
            move_reference(over);
          }
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(bar_p(i));
        }
        if (!ok) break;
        done += count;
        // ---- results ----
        float s0, s1;
        unpack_f2(sum2, s0, s1);
        float sum = s0 + s1;
        if (d.split && i == 1) {                                               // unit 0 does the rest
          s_merge[row] = make_float4(ref, sum, (float)lift, 0.f);
          mbar_arrive(bar_merge);
          ++pieces;
          tiles += all;
          mbar_arrive(bar_piecefree(it & 1));
          continue;
        }
        bool none = ref == -INFINITY && sum == sum;
        ok = warp_wait<5>(bar_o(i), pieces & 1, s_abort, status);
        if (!ok) break;
        float times = exp2f((float)-lift), times1 = 0.f;                       // of O; of unit 1's
        if (d.split) {
          ok = warp_wait<18>(bar_o(1), others & 1, s_abort, status);
          if (ok) ok = warp_wait<19>(bar_merge, splits & 1, s_abort, status);
          if (!ok) break;
          ++splits;
          const float4 x = s_merge[row];
          const bool none1 = x.x == -INFINITY && x.y == x.y;
          const float top = fmaxf(ref, x.x);
          // (a sum without a reference: NaN)
          const float f0 = ref == -INFINITY ? (none ? 0.f : 1.f) : ex2(ref - top), f1 = x.x == -INFINITY ? (none1 ? 0.f : 1.f) : ex2(x.x - top);
          sum = sum * f0 + x.y * f1;
          times *= f0;
          times1 = exp2f(-x.z) * f1;
          ref = top;
          none = none && none1;
        }
        tc_fence_after();
        const size_t place = (size_t)d.place * kBlockRows + in_block;
        uint32_t nan = 0;                                                      // groups with a NaN that the row sees
#pragma unroll
        for (int g = 0; g < G; ++g) nan |= (uint32_t)(s_nan[(it & 1) * 4 + g] <= limit && !none) << g;
        // the pieces of the segment before this one, which this thread has put at the place
        const bool begun = d.begun && there;
        float past = 0.f;                                                      // of what is there
        if (begun) {
          const float2 x = o.part_s[place];
          const bool none1 = x.x == -INFINITY && x.y == 0.f;
          const float top = fmaxf(ref, x.x), f = ref == -INFINITY ? (none ? 0.f : 1.f) : ex2(ref - top);
          past = x.x == -INFINITY ? (none1 ? 0.f : 1.f) : ex2(x.x - top);
          sum = (none ? 0.f : sum * f) + x.y * past;
          times *= f;
          times1 *= f;
          ref = top;
          none = none && none1;
        }
        if (d.last) { const float inv = none ? 0.f : 1.f / sum; times *= inv; times1 *= inv; past *= inv; }
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_ld32_issue(ocol + 32 * c, v);
          tmem_ld32_wait(v);
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * times);
          if (d.split) {
            uint32_t v1[32];
            tmem_ld32_issue(ocol + D + 32 * c, v1);
            tmem_ld32_wait(v1);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(fmaf(__uint_as_float(v1[e]), times1, __uint_as_float(v[e])));
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = none ? 0u : nan >> c & 1 ? 0x7fffffffu : v[e];
          if (begun) {
            const float4* x = o.part_o + ((size_t)d.place * (D / 4) + 8 * c) * kBlockRows + in_block;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float4 y = x[e * kBlockRows];
              v[4 * e] = __float_as_uint(fmaf(y.x, past, __uint_as_float(v[4 * e])));
              v[4 * e + 1] = __float_as_uint(fmaf(y.y, past, __uint_as_float(v[4 * e + 1])));
              v[4 * e + 2] = __float_as_uint(fmaf(y.z, past, __uint_as_float(v[4 * e + 2])));
              v[4 * e + 3] = __float_as_uint(fmaf(y.w, past, __uint_as_float(v[4 * e + 3])));
            }
          }
          if (there) {
            if (!d.last || o.out_kind == HYPERATTN_FP32) {
              float4* to = d.last ? reinterpret_cast<float4*>(o.out) + at * (D / 4) + 8 * c : o.part_o + ((size_t)d.place * (D / 4) + 8 * c) * kBlockRows + in_block;
              const int step = d.last ? 1 : kBlockRows;
#pragma unroll
              for (int e = 0; e < 8; ++e)
                to[e * step] = make_float4(__uint_as_float(v[4 * e]), __uint_as_float(v[4 * e + 1]), __uint_as_float(v[4 * e + 2]), __uint_as_float(v[4 * e + 3]));
            } else {
              uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<T*>(o.out) + at * D + 32 * c);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = from_float2<T>(__uint_as_float(v[8 * e + 2 * k]), __uint_as_float(v[8 * e + 2 * k + 1]));
                to[e] = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          }
        }
        tc_fence_before();
        mbar_arrive(bar_ofree(i));
        if (d.split) mbar_arrive(bar_ofree(1));
        ++pieces;
        if (there) {
          if (!d.last) o.part_s[place] = make_float2(none ? -INFINITY : ref, none ? 0.f : sum);
          else o.lse[at] = none ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
        }
      }
      others += d.split || d.units[1] > 0;
      tiles += all;
      mbar_arrive(bar_piecefree(it & 1));
    }
  } else if (warp < 16) {
    // ================= keys and values: a warp a block of 16 tokens ========================================
    const int group_kv = (warp >> 2) & 1, sub = warp & 3, c4 = lane & 3, r8 = lane >> 2;
    // (what one of the four gives up on, all do: they meet at a barrier that has no limit)
    auto all_ok = [&](bool mine) {
      uint32_t all;
      asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"((uint32_t)mine), "r"(1 + group_kv) : "memory");
      return all != 0;
    };
    int tiles = 0;
    bool ok = true;
    for (int it = 0; ok; ++it) {
      ok = all_ok(piece_wait(it, std::integral_constant<int, 6>{}));
      if (!ok) break;
      const Piece d = s_piece[it & 1];
      if (d.end) break;
      for (int n = d.tile0; n < d.tile1; ++n, ++tiles) {
        if ((tiles & 1) != group_kv) continue;
        const int st = tiles % NS, rs = tiles % NRAW;
        int* exponents = s_exp + (2 * group_kv + (tiles >> 1 & 1)) * 4;
        bool mine = tiles < NS || warp_wait<7>(bar_opfree(st), (tiles / NS - 1) & 1, s_abort, status);
        if (mine) mine = warp_wait<8>(bar_raw(rs), (tiles / NRAW) & 1, s_abort, status);
        const uint32_t blocks = s_there[rs];
        const uint8_t* raw = smem + C::kOffRaw + rs * C::kRaw + sub * B::kBytes;
        const int valid = blocks >> sub & 1 ? min(max(d.s.len - n * kKeys - sub * kBlockTokens, 0), kBlockTokens) : 0;
        // scales and minima: K's of tokens r8 and 8 + r8 (pairs, of which one is the lane's), V's of tokens 2 c4, 2 c4 + 1 and 8 + those
        uint32_t sk[2][G], mk[2][G], sv[2][G], mv[2][G];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int g = 0; g < G; g += 2) {
            const uint4 x = *reinterpret_cast<const uint4*>(raw + B::kScaleK + (half * 4 + lane / 8) * G * 8 + g * 8);
            const uint4 y = *reinterpret_cast<const uint4*>(raw + B::kScaleV + (half * 4 + c4) * G * 8 + g * 8);
            sk[half][g] = x.x; mk[half][g] = x.y; sk[half][g + 1] = x.z; mk[half][g + 1] = x.w;
            sv[half][g] = y.x; mv[half][g] = y.y; sv[half][g + 1] = y.z; mv[half][g + 1] = y.w;
          }
        if (valid < kBlockTokens) {                                            // whatever the places behind the last token hold
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int tk = half * 8 + lane / 8 * 2, tv = half * 8 + 2 * c4;
            const uint32_t keep_k = (tk < valid ? 0xffffu : 0u) | (tk + 1 < valid ? 0xffff0000u : 0u), keep_v = (tv < valid ? 0xffffu : 0u) | (tv + 1 < valid ? 0xffff0000u : 0u);
#pragma unroll
            for (int g = 0; g < G; ++g) { sk[half][g] &= keep_k; mk[half][g] &= keep_k; sv[half][g] &= keep_v; mv[half][g] &= keep_v; }
          }
        }
        auto bad_of = [](uint32_t x) { return ((x & 0x7fff7fffu) + 0x04000400u) & 0x80008000u; };          // an exponent of ones carries into the sign's place
        // values that are no numbers
        {
          uint32_t any = 0;
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int g = 0; g < G; ++g) any |= bad_of(sv[half][g]) | bad_of(mv[half][g]);
          if (__any_sync(0xffffffffu, any)) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int g = 0; g < G; ++g) {
                const uint32_t bad = bad_of(sv[half][g]) | bad_of(mv[half][g]), gone = (bad >> 15) * 0xffffu;
                sv[half][g] &= ~gone;
                mv[half][g] &= ~gone;
                if (bad) atomicMin(&s_nan[(it & 1) * 4 + g], n * kKeys + sub * kBlockTokens + half * 8 + 2 * c4 + (bad & 0x8000u ? 0 : 1));
              }
          }
        }
        __half2 top_s = as_half2(0u), top_m = as_half2(0u), vtop_s = as_half2(0u), vtop_m = as_half2(0u);      // (of a number and NaN the number)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int g = 0; g < G; ++g) {
            top_s = __hmax2(top_s, as_half2(sk[half][g])); top_m = __hmax2(top_m, __habs2(as_half2(mk[half][g])));
            vtop_s = __hmax2(vtop_s, as_half2(sv[half][g])); vtop_m = __hmax2(vtop_m, __habs2(as_half2(mv[half][g])));
          }
        int mine_k = exponent_of(as_u32(top_s), as_u32(top_m));
        // (K's infinities are still there, and one would hide the other tokens' numbers: then one by one.  V's are gone)
        if (__any_sync(0xffffffffu, bad_of(as_u32(top_s)) | bad_of(as_u32(top_m)))) {
          mine_k = 0;
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int g = 0; g < G; ++g) mine_k = max(mine_k, exponent_of(sk[half][g], mk[half][g]));
        }
        const int ek = __reduce_max_sync(0xffffffffu, mine_k), ev = __reduce_max_sync(0xffffffffu, exponent_of(as_u32(vtop_s), as_u32(vtop_m)));
        if (lane == 0) exponents[sub] = ek | ev << 8;
        ok = all_ok(mine);
        if (!ok) break;
        int tile_k = 0, tile_v = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) { const int e = exponents[w]; tile_k = max(tile_k, e & 255); tile_v = max(tile_v, e >> 8); }
        const int lift_k = lift_of(tile_k), lift_v = lift_of(tile_v) & ~3;
        const __half2 up_k = lift2(lift_k), up_v = lift2(lift_v);
        uint8_t* to = smem + st * C::kStage;
        if (sub == 0 && lane == 0) s_tile[st] = make_float4(__uint_as_float((uint32_t)(127 - lift_k) << 23), __int_as_float(lift_v), __uint_as_float(blocks), 0.f);
        // K: 8 codes of a token are 16 bytes.  (Tokens of odd rows take the groups of a pair the other way round, so that eight lanes write to all banks.)
        const uint32_t same = r8 & 1 ? 0x3232u : 0x1010u;
        const bool swap = r8 & 1;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t kw[G], m[G];
          if constexpr (D == 128) {
            const uint4 v = *reinterpret_cast<const uint4*>(raw + half * 512 + lane * 16);
            kw[0] = v.x; kw[1] = v.y; kw[2] = v.z; kw[3] = v.w;
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(raw + lane * 16 + half * 8);
            kw[0] = v.x; kw[1] = v.y;
          }
          const int krow = sub * kBlockTokens + half * 8 + r8;
#pragma unroll
          for (int g = 0; g < G; ++g) m[g] = as_u32(__hmul2(as_half2(__byte_perm(mk[half][g], 0, same)), up_k));
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const uint32_t w = swap ? kw[g ^ 1] : kw[g], s = swap ? sk[half][g ^ 1] : sk[half][g];
            const __half2 sc = __hmul2(as_half2(__byte_perm(s, 0, same)), up_k);
            uint32_t k[4], p[4], rest[4];
            half_codes(w, k);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const __half2 y = __hmul2(as_half2(k[x]), sc);
              p[x] = as_u32(y);
              rest[x] = as_u32(__hfma2(as_half2(k[x]), sc, __hneg2(y)));
            }
            const uint32_t at = (uint32_t)(g / 2) * C::kKeySlab + krow * 128 + (((((g & 1) ^ (int)swap) * 4 + c4) ^ r8) << 4);
            *reinterpret_cast<uint4*>(to + at) = make_uint4(p[0], p[1], p[2], p[3]);
            *reinterpret_cast<uint4*>(to + C::kOffRest + at) = make_uint4(rest[0], rest[1], rest[2], rest[3]);
          }
          // minima, three times: for the three parts of the queries' sums.  Lanes 2 half and 2 half + 1 of a token's four write its 32 bytes
          if (c4 >> 1 == half) {
            const uint32_t m01 = __byte_perm(m[0], m[1], 0x5410), m23 = __byte_perm(m[G - 2], m[G - 1], 0x5410);
            const uint4 first = G == 4 ? make_uint4(m01, m23, m01, m23) : make_uint4(m01, m01, m01, 0u), second = G == 4 ? make_uint4(m01, m23, 0u, 0u) : make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(to + C::kOffMinima + (c4 & 1) * (kKeys * 16) + krow * 16) = c4 & 1 ? second : first;
          }
        }
        // V: pairs of tokens of a coordinate
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int g = 0; g < G; ++g) {
            sv[half][g] = as_u32(__hmul2(as_half2(sv[half][g]), up_v));
            mv[half][g] = as_u32(__hmul2(as_half2(mv[half][g]), up_v));
          }
#pragma unroll
        for (int i4 = 0; i4 < D / 64; ++i4) {
          const uint4 v = *reinterpret_cast<const uint4*>(raw + B::kV + i4 * 512 + lane * 16);
          const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int u = 4 * i4 + j, g = u / 2;
            uint32_t k[4];
            half_codes(vw[j], k);
#pragma unroll
            for (int x = 0; x < 4; ++x) {                                      // tokens 2 c4, + 1 (x >= 2: 8 + those) of coordinate 16 u + r8 (odd x: 8 more)
              const int half = x / 2, coordinate = 16 * u + 8 * (x & 1) + r8;
              *reinterpret_cast<uint32_t*>(to + C::kOffV + coordinate * 128 + (((2 * sub + half) ^ r8) << 4) + c4 * 4) =
                  as_u32(__hfma2(as_half2(k[x]), as_half2(sv[half][g]), as_half2(mv[half][g])));
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_rawfree(rs));
        fence_async_smem();
        mbar_arrive(bar_op(st));
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_piecefree(it & 1));
    }
  } else if (warp == 16) {
    // ================= products ============================================================================
    const bool el = elect_one();
    constexpr uint32_t idesc_s = (1u << 4) | ((uint32_t)(kKeys >> 3) << 17) | ((128u >> 4) << 24);
    constexpr uint32_t idesc_o = (1u << 4) | ((uint32_t)(D >> 3) << 17) | ((128u >> 4) << 24);
    int tiles = 0, done[2] = {0, 0}, pieces[2] = {0, 0}, queries[2] = {0, 0};
    bool ok = true;
    for (int it = 0; ok; ++it) {
      ok = piece_wait(it, std::integral_constant<int, 9>{});
      if (!ok) break;
      const Piece& d = s_piece[it & 1];
      auto uni = [&](int x) { return __reduce_max_sync(0xffffffffu, x); };
      const bool end = uni(d.end) != 0, split = uni(d.split) != 0, has[2] = {uni(d.units[0]) > 0, split || uni(d.units[1]) > 0};
      const bool begun = uni(d.begun) != 0, more = uni(d.more) != 0;
      const int count = uni(d.tile1 - d.tile0), step = split ? 2 : 1;
      __syncwarp();
      if (el) mbar_arrive(bar_piecefree(it & 1));
      if (end) break;
      // (Queries of the piece before: the first scores come as soon as the last ones have been read.  Unit 1 cannot be at its piece's end before unit 0 has put the last piece's results together: both have
      // tens of tiles then, and the second one's scores come after O has been read.)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (ok && has[i]) {
          if (!begun) ok = warp_wait<10>(bar_q(i), queries[i]++ & 1, s_abort, status);
          else if constexpr (C::kOwnP) ok = warp_wait<14>(bar_sfree(i), (done[i] - 1) & 1, s_abort, status);
        }
      if (!ok) break;
      auto wait_tile = [&](int n) { if (ok) ok = warp_wait<11>(bar_op((tiles + n) % NS), ((tiles + n) / NS) & 1, s_abort, status); };
      // tile n, the unit's last one if there is none `step` further
      auto scores = [&](int i, int n) {
        const uint32_t stage = (ubase + (uint32_t)((tiles + n) % NS) * C::kStage) >> 4, to = tmem + C::kColS + kKeys * i;
        if (el) {
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              mma_ts2(to, tmem + C::kColQ + (D / 2) * i + 8 * ks, (stage | (1u << 16)) + ((part * C::kOffRest + (ks >> 2) * C::kKeySlab + (ks & 3) * 32) >> 4), kDescSwizzled, idesc_s, part + ks > 0);
          mma_ss2(to, ((ubase + C::kOffSums + i * C::kSums) >> 4) | (((kUnitRows * 16u) >> 4) << 16), (stage + (C::kOffMinima >> 4)) | (((kKeys * 16u) >> 4) << 16), kDescPlain, idesc_s, 1);
          umma_commit(bar_s(i));
          if (n + step >= count && !more) umma_commit(bar_qfree(i));
        }
      };
      // (k: tiles of the unit before it)
      auto outputs = [&](int i, int n, int k) {
        if (k == 0 && pieces[i] > 0) ok = warp_wait<12>(bar_ofree(i), (pieces[i] - 1) & 1, s_abort, status);
        if (ok) ok = warp_wait<13>(bar_p(i), (done[i] + k) & 1, s_abort, status);
        if (!ok) return;
        tc_fence_after();
        const uint32_t v_lo = ((ubase + (uint32_t)((tiles + n) % NS) * C::kStage + C::kOffV) >> 4) | (1u << 16);
        if (el) {
#pragma unroll
          for (int kk = 0; kk < kKeys / 16; ++kk) mma_ts2(tmem + D * i, tmem + C::col_p(i) + kk * 8, v_lo + kk * (32 >> 4), kDescSwizzled, idesc_o, kk > 0 || k > 0);
          if constexpr (FINE) {
#pragma unroll
            for (int kk = 0; kk < kKeys / 16; ++kk) mma_ts2(tmem + D * i, tmem + C::col_p(i) + C::kRest + kk * 8, v_lo + kk * (32 >> 4), kDescSwizzled, idesc_o, 1);
          }
          if (C::kOwnP) umma_commit(bar_pfree(i));
          if (n + step >= count) umma_commit(bar_o(i));
        }
      };
      auto next_scores = [&](int i, int n, int k) {                              // of tile n, k tiles of the unit before it
        if constexpr (C::kOwnP) {
          ok = warp_wait<14>(bar_sfree(i), (done[i] + k - 1) & 1, s_abort, status);
          if (!ok) return;
          tc_fence_after();
        }
        scores(i, n);
      };
      wait_tile(0);
      if (split && count > 1) wait_tile(1);
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (has[i]) scores(i, split ? i : 0);
      if (split) {
        for (int n0 = 0; n0 < count && ok; n0 += 2) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int n = n0 + i, k = n0 / 2;
            if (!ok || n >= count) break;
            auto next = [&] {
              if (n + 2 >= count) return;
              wait_tile(n + 2);
              if (!ok) return;
              tc_fence_after();
              next_scores(i, n + 2, k + 1);
            };
            // (P in the place of S; and of three stages, tile n + 2 gets that of tile n - 1: its keys come while this tile's weights are multiplied)
            if (C::kOwnP) next();
            if (ok) outputs(i, n, k);
            if (ok && el) umma_commit(bar_opfree((tiles + n) % NS));
            if (ok && !C::kOwnP) next();
          }
        }
        tiles += count;
        done[0] += (count + 1) / 2;
        done[1] += count / 2;
        ++pieces[0];
        ++pieces[1];
        continue;
      }
      for (int n = 0; n < count && ok; ++n) {
        if (n + 1 < count) wait_tile(n + 1);
        if (!ok) break;
        tc_fence_after();
        if constexpr (C::kOwnP) {
          // the next scores as soon as these have been read, then the products with V
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (ok && n + 1 < count && has[i]) next_scores(i, n + 1, n + 1);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (ok && has[i]) outputs(i, n, n);
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (ok && has[i]) {
              outputs(i, n, n);
              if (ok && n + 1 < count) next_scores(i, n + 1, n + 1);
            }
        }
        if (ok && el) umma_commit(bar_opfree((tiles + n) % NS));
      }
      tiles += count;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (has[i]) { done[i] += count; ++pieces[i]; }
    }
    __syncwarp();
  } else if (warp == 17) {
    // ================= copies ==============================================================================
    // A lane has a block of the next eight tiles: its page is looked up before their turn comes.
    int tiles = 0;
    bool ok = true;
    for (int it = 0; ok; ++it) {
      ok = piece_wait(it, std::integral_constant<int, 15>{});
      if (!ok) break;
      const Piece d = s_piece[it & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_piecefree(it & 1));
      if (d.end) break;
      int place = 0, place1 = 0;
      auto look = [&](int from, int& at) {
        const int n = from + lane / 4, token = n * kKeys + lane % 4 * kBlockTokens;
        at = 0;
        if (n >= d.tile1 || token >= d.s.len) return -1;
        const int column = token / a.cache.page;
        at = d.kv * subs + (token - column * a.cache.page) / kBlockTokens;
        return a.table[(size_t)d.request * a.width + column];
      };
      int page = look(d.tile0, place);
      for (int n0 = d.tile0; n0 < d.tile1 && ok; n0 += 8) {
        const int page1 = look(n0 + 8, place1);
        for (int n = n0; n < min(n0 + 8, d.tile1); ++n, ++tiles) {
          const int rs = tiles % NRAW;
          const int p = __shfl_sync(0xffffffffu, page, (n - n0) * 4 + lane % 4), at = __shfl_sync(0xffffffffu, place, (n - n0) * 4 + lane % 4);
          const bool is = lane < 4 && p >= 0 && p < a.cache.num_pages, copies = is && lane % run == 0;
          const unsigned there = __ballot_sync(0xffffffffu, is), runs = __ballot_sync(0xffffffffu, copies);
          if (tiles >= NRAW) ok = warp_wait<16>(bar_rawfree(rs), (tiles / NRAW - 1) & 1, s_abort, status);
          if (!ok) break;
          if (lane == 0) {
            s_there[rs] = there;
            mbar_arrive_expect(bar_raw(rs), __popc(runs) * run * B::kBytes);
          }
          __syncwarp();
          // (the blocks of a run that are beyond the request's tokens come along; a run has one page)
          if (copies) bulk_load(ubase + C::kOffRaw + rs * C::kRaw + lane * B::kBytes, a.cache.pages + ((size_t)p * a.cache.heads * subs + at) * B::kBytes, run * B::kBytes, bar_raw(rs));
        }
        page = page1;
        place = place1;
      }
    }
    // nothing may be on its way into shared memory when the CTA ends
    for (int s = 0; s < NRAW && s < tiles; ++s) mbar_drain(bar_raw(s), ((tiles - 1 - s) / NRAW) & 1);
  } else if (warp == 18) {
    // ================= segments ============================================================================
    const long long begin = o.start[blockIdx.x], end = o.start[blockIdx.x + 1];
    int slot = 0;
    if (begin < end) {
      int hi = o.slots;                                    // the last row block that starts there or before
      while (hi - slot > 1) { const int mid = (slot + hi) >> 1; if (o.before[mid] <= begin) slot = mid; else hi = mid; }
    }
    long long x = begin;
    bool ok = true;
    for (int it = 0; ok; ++it) {
      Piece d = {};
      d.end = x >= end;
      if (!d.end) {
        while (o.before[slot + 1] <= x) ++slot;
        const int2 b = o.block[slot];
        d.request = b.x;
        d.s = span_of(a, b.x);
        const RowBlock k = row_block(a, d.s, b.y);
        const long long rest = x - o.before[slot], whole = (long long)k.tiles * k.cost;
        d.kv = (int)(rest / whole);
        d.row0 = k.row0;
        d.units[0] = min(k.rows, kUnitRows);
        d.units[1] = k.rows - d.units[0];
        const long long first = x - (rest - d.kv * whole), last = first + whole;               // the segment's
        d.tile0 = (int)((x - first) / k.cost);
        const int tiles = (int)((min(last, end) - first) / k.cost) - d.tile0, most = d.units[1] ? kChain<FINE> : 2 * kChain<FINE>, pieces = (tiles + most - 1) / most;        // (that are left here)
        d.tile1 = d.tile0 + (tiles + pieces - 1) / pieces;
        d.split = d.units[1] == 0 && d.tile1 - d.tile0 > 1;
        // (a segment that is finished here as a whole has the place of the part's end for that long)
        const bool inside = first >= begin && last <= end;
        d.begun = x > first && x > begin;
        d.more = pieces > 1;
        d.last = inside && pieces == 1;
        d.place = 2 * (int)blockIdx.x + (inside || first > begin ? 1 : 0);
        x = first + (long long)d.tile1 * k.cost;
      }
      if (it >= 2) ok = warp_wait<17>(bar_piecefree(it & 1), ((it >> 1) - 1) & 1, s_abort, status);
      if (!ok) break;
      if (lane < 4) s_nan[(it & 1) * 4 + lane] = INT_MAX;
      __syncwarp();
      if (lane == 0) {
        s_piece[it & 1] = d;
        mbar_arrive(bar_piece(it & 1));
      }
      __syncwarp();
      if (d.end) break;
    }
  }
  // ---- teardown ----
  tc_fence_before();
  __syncthreads();
  if (warp == 16) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// Puts the pieces of segments together that lie in several parts; rows without any tile get their zeros.
constexpr int kPutThreads = 256;
template <int D> constexpr int kPutRows = kPutThreads / (D / 4);        // (a row for every 32 or 16 threads: with 32 rows a CTA it took 20 us)

template <int D, class T>
__global__ void __launch_bounds__(kPutThreads) put_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ ChunkOut o) {
  wait_for_stream();
  const int kv = blockIdx.x % a.cache.heads, slot = blockIdx.x / a.cache.heads, group = a.q_heads / a.cache.heads, tid = threadIdx.x;
  const int2 b = o.block[slot];
  if (b.x < 0) return;
  const Span s = span_of(a, b.x);
  const RowBlock k = row_block(a, s, b.y);
  if ((int)blockIdx.y * kPutRows<D> >= k.rows) return;
  const long long whole = (long long)k.tiles * k.cost, first = o.before[slot] + kv * whole, last = first + whole;
  int p0 = 0, p1 = 0;                                  // its first and last part
  if (k.tiles > 0) {
    // (starts ascend: as many as are not behind it, less one)
    for (int c = 0; c < o.parts; c += kPutThreads) {
      p0 += __syncthreads_count(c + tid < o.parts && o.start[c + tid] <= first);
      p1 += __syncthreads_count(c + tid < o.parts && o.start[c + tid] < last);
    }
    --p0;
    --p1;
    if (p0 == p1) return;                              // finished there
  }
  const int lane = tid / kPutRows<D>;
  for (int row = blockIdx.y * kPutRows<D> + tid % kPutRows<D>; row < k.rows; row += gridDim.y * kPutRows<D>) {
    float ref = -INFINITY, sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (k.tiles > 0)
#pragma unroll 4
      for (int c = p0; c <= p1; ++c) {
        if (o.start[c] == o.start[c + 1]) continue;
        const size_t place = 2 * c + (c == p0 && o.start[c] < first ? 1 : 0);
        const float2 x = o.part_s[place * kBlockRows + row];
        const float4 y = o.part_o[(place * (D / 4) + lane) * kBlockRows + row];
        const float m = fmaxf(ref, x.x);
        const float f = x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : ex2(x.x - m), g = ref == -INFINITY ? (sum == 0.f ? 0.f : 1.f) : ex2(ref - m);
        ref = m;
        sum = sum * g + x.y * f;
        v = make_float4(v.x * g + y.x * f, v.y * g + y.y * f, v.z * g + y.z * f, v.w * g + y.w * f);
      }
    const int token = (k.row0 + row) / group;
    const size_t at = (size_t)(s.first + token) * a.q_heads + kv * group + k.row0 + row - token * group;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    v = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    if (o.out_kind == HYPERATTN_FP32) reinterpret_cast<float4*>(reinterpret_cast<float*>(o.out) + at * D)[lane] = v;
    else reinterpret_cast<uint2*>(reinterpret_cast<T*>(o.out) + at * D)[lane] = make_uint2(from_float2<T>(v.x, v.y), from_float2<T>(v.z, v.w));
    if (lane == 0) o.lse[at] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.6931471805599453f;
  }
}

// What a call's launches look like, and where its workspace has what
struct ChunkShape { long long slots; int parts; size_t block, start, part_s, part_o, bytes; };
ChunkShape chunk_shape(const hyperattn_chunk_params& p, int least) {
  ChunkShape s;
  s.slots = image_slots(p.rows, p.requests, p.q_heads / p.cache.kv_heads, kBlockRows, least) + 1;
  const long long tiles = s.slots * p.cache.kv_heads * (((long long)p.table_width * p.cache.page_tokens + kKeys - 1) / kKeys);
  s.parts = (int)(tiles < kSms ? tiles : kSms);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  s.block = up((size_t)(s.slots + 1) * 8);
  s.start = s.block + up((size_t)s.slots * 8);
  s.part_s = s.start + up((size_t)(s.parts + 1) * 8);
  s.part_o = s.part_s + (size_t)s.parts * 2 * kBlockRows * 8;
  s.bytes = s.part_o + (size_t)s.parts * 2 * kBlockRows * p.cache.d * 4;
  return s;
}
// The kernels of a call, and what its workspace has for those of few rows (what they cannot count: all is for these)
Kinds chunk_kinds(const hyperattn_chunk_params& p, Kinds k, size_t* few) {
  *few = 0;
  if (k.few && !few_rows_attention(p, k.many, few)) { *few = 0; return {false, true}; }
  *few = (*few + 255) / 256 * 256;
  return k;
}

int check(const hyperattn_chunk_params* p) {
  if (int rc = check_chunk(p)) return rc;
  if (p->out_dtype != p->dtype && p->out_dtype != HYPERATTN_FP32) return HYPERATTN_INVALID_ARGUMENT;
  return HYPERATTN_OK;
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_cache_chunk_attention_workspace_bytes(const hyperattn_chunk_params* p, size_t* bytes) {
  if (!bytes) return HYPERATTN_INVALID_ARGUMENT;
  if (int rc = check(p)) return rc;
  *bytes = 0;
  if (p->requests == 0 || p->rows == 0) return HYPERATTN_OK;
  // (whatever a caller says about the most new tokens: without any word there are both kinds if there can be)
  size_t few, alone = 0;
  const Kinds any = chunk_kinds(*p, kinds_of(*p, 0), &few);
  if (any.many) chunk_kinds(*p, {true, false}, &alone);
  *bytes = few > alone ? few : alone;
  if (!any.many) return HYPERATTN_OK;
  const ChunkShape s = chunk_shape(*p, any.few ? most_of(*p) : -1);
  if (s.slots * p->cache.kv_heads > 0x7fffffffLL) return HYPERATTN_UNSUPPORTED_SHAPE;
  *bytes += s.bytes;
  return HYPERATTN_OK;
}

extern "C" int hyperattn_cache_chunk_attention(const hyperattn_chunk_params* p) { return hyperattn_cache_chunk_attention_ex(p, 0); }

extern "C" int hyperattn_cache_chunk_attention_ex(const hyperattn_chunk_params* p, int most_new) {
  size_t bytes = 0;
  if (most_new < 0) return HYPERATTN_INVALID_ARGUMENT;
  if (int rc = hyperattn_cache_chunk_attention_workspace_bytes(p, &bytes)) return rc;
  if (!p->cu_q && p->rows != p->requests) return HYPERATTN_INVALID_ARGUMENT;
  if (p->requests == 0 || p->rows == 0) return HYPERATTN_OK;
  if (!p->q || !p->out || !p->lse || !p->table || !p->lengths || !p->workspace) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->q) || misaligned(p->out) || misaligned(p->workspace)) return HYPERATTN_MISALIGNED;
  if (p->workspace_bytes < bytes) return HYPERATTN_WORKSPACE_TOO_SMALL;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(p->stream);
  int* status = nullptr;
  if (int rc = device_status_word(st, &status)) return rc;
  ChunkArgs a = chunk_args(*p);
  char* ws = reinterpret_cast<char*>(p->workspace);
  size_t few;
  const Kinds kinds = chunk_kinds(*p, kinds_of(*p, p->cu_q ? most_new : 1), &few);
  if (kinds.few) {
    const int rc = launch_few_rows_attention(*p, kinds.many, status);
    if (rc || !kinds.many) return rc;
    a.least = most_of(*p);
    ws += few;
  }
  const ChunkShape s = chunk_shape(*p, a.least);
  const ChunkOut o = {p->out, p->lse, p->out_dtype, reinterpret_cast<long long*>(ws), reinterpret_cast<int2*>(ws + s.block), reinterpret_cast<long long*>(ws + s.start),
                      reinterpret_cast<float4*>(ws + s.part_o), reinterpret_cast<float2*>(ws + s.part_s), (int)s.slots, s.parts};
  const int subs = p->cache.page_tokens / kBlockTokens, run = subs % 4 == 0 ? 4 : subs & -subs;
  auto go = [&](auto dim, auto type, auto fine) {
    constexpr int D = decltype(dim)::value;
    using T = decltype(type);
    constexpr auto kernel = chunk_kernel<D, T, decltype(fine)::value>;
    cudaError_t e = allow_smem<kernel>(CCfg<D>::kSmem);
    if (e == cudaSuccess) e = launch(share_kernel, dim3(1), dim3(kShareThreads), 0, st, a, o);
    if (e == cudaSuccess) e = launch(kernel, dim3((unsigned)s.parts), dim3(kCThreads), CCfg<D>::kSmem, st, a, o, run, status);
    // (as many CTAs as the GPU holds several times over, at most: 64 requests of few rows, 8 heads, had 17 664, most with nothing to do)
    const long long blocks = s.slots * p->cache.kv_heads, most = kBlockRows / kPutRows<D>, want = (32 * kSms + blocks - 1) / blocks;
    if (e == cudaSuccess) e = launch(put_kernel<D, T>, dim3((unsigned)blocks, (unsigned)(want < most ? want : most)), dim3(kPutThreads), 0, st, a, o);
    return status_of(e, "chunk attention");
  };
  auto of_type = [&](auto dim) {
    return p->dtype != HYPERATTN_BF16 ? go(dim, __half(), std::true_type()) : p->out_dtype == HYPERATTN_FP32 ? go(dim, __nv_bfloat16(), std::true_type()) : go(dim, __nv_bfloat16(), std::false_type());
  };
  return p->cache.d == 64 ? of_type(std::integral_constant<int, 64>()) : of_type(std::integral_constant<int, 128>());
}
