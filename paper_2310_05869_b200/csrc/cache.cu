// The paged 4-bit cache: pages (plan), storing, reading.
#include <cstdio>
#include "serving.cuh"
#include "tc_util.cuh"

namespace hyperattn {
namespace {

// ---- plan ------------------------------------------------------------------------------------------------------------------
// Everything follows from three running sums over the requests (new tokens, pages needed, pages released), which every CTA makes for
// itself in shared memory - reading a few KB again costs less than a launch to make them first.  Then it does one thing: some CTAs
// write the tables, some the rows, some the stack, one the requests' new state, so that their latencies do not add up.  256 requests with tables of 129 pages: 5.0 us,
// latency (7.0 with the four in a row); 1024 requests with 2049 pages: 11.6 us, bound by the instructions of the sums (two 64-bit divisions a request, in each of 519 CTAs).
constexpr int kPlanColumns = 512;        // table entries of a warp at a time

struct PlanParts { int tables, rows, stack; };           // CTAs for each

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ hyperattn_plan p, PlanParts parts) {
  extern __shared__ int smem[];
  __shared__ int s_warp[3][kPlanWarps], s_given;
  wait_for_stream();
  const int R = p.requests, W = p.table_width, P = p.page_tokens, F = p.num_free;
  // running sums (inclusive); pages that a request has, 1 << 29: there is room for it, 1 << 30: it has ended; its length
  int *s_add = smem, *s_need = smem + R, *s_rel = smem + 2 * R, *s_have = smem + 3 * R, *s_len = smem + 4 * R;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n_free = min(max(p.n_free[0], 0), F);
  if (tid == 0) s_given = 0;

  // a thread takes consecutive requests
  const int per = (R + kPlanThreads - 1) / kPlanThreads, r0 = min(R, tid * per), r1 = min(R, r0 + per);
  int sum[3] = {0, 0, 0};
  for (int r = r0; r < r1; ++r) {
    const int len = max(p.lengths[r], 0), add = p.new_tokens[r];
    const int have = min((int)(((long long)len + P - 1) / P), W);
    const long long pages = ((long long)len + max(add, 0) + P - 1) / P;
    const bool ended = add < 0, fits = !ended && pages <= W;
    const int need = fits ? max((int)pages - have, 0) : 0;
    sum[0] = plus(sum[0], max(add, 0)); sum[1] += need; sum[2] += ended ? have : 0;
    s_add[r] = sum[0]; s_need[r] = sum[1]; s_rel[r] = sum[2];
    s_have[r] = have | (fits ? 1 << 29 : 0) | (ended ? 1 << 30 : 0);
    s_len[r] = len;
  }
  sums_before(sum, s_warp);
  for (int r = r0; r < r1; ++r) { s_add[r] = plus(s_add[r], sum[0]); s_need[r] += sum[1]; s_rel[r] += sum[2]; }
  __syncthreads();
  const int total = n_free + s_rel[R - 1];             // pages on the stack before any is taken

  auto before = [](const int* a, int r) { return r ? a[r - 1] : 0; };
  auto have_of = [&](int r) { return s_have[r] & 0xfffffff; };
  auto ended = [&](int r) { return (s_have[r] >> 30 & 1) != 0; };
  auto need_of = [&](int r) { return s_need[r] - before(s_need, r); };
  auto admitted = [&](int r) { return (s_have[r] >> 29 & 1) && (need_of(r) == 0 || s_need[r] <= total); };
  auto stack = [&](int i) {                            // entry of the stack: a free page, or a released one
    if (i < 0) return -1;
    if (i < n_free) return p.free_pages[i];
    const int r = upper_bound(s_rel, R, i - n_free);
    return r < R ? p.table[(size_t)r * W + (i - n_free - before(s_rel, r))] : -1;
  };
  auto fresh = [&](int r, int k) { return stack(total - 1 - (before(s_need, r) + k)); };      // request r's k-th new page

  int cta = blockIdx.x;
  if (cta < parts.tables) {
    // block tables: a warp takes pieces of rows
    const int pieces = (W + kPlanColumns - 1) / kPlanColumns;
    for (int u = cta * kPlanWarps + warp; u < R * pieces; u += parts.tables * kPlanWarps) {
      const int r = u / pieces, c0 = (u - r * pieces) * kPlanColumns;
      const int have = have_of(r), keep = ended(r) ? 0 : have, end = admitted(r) ? have + need_of(r) : keep;
      const int32_t* from = p.table + (size_t)r * W;
      int32_t* to = p.table_out + (size_t)r * W;
      int v[kPlanColumns / 32];
#pragma unroll
      for (int i = 0; i < kPlanColumns / 32; ++i) { const int c = c0 + 32 * i + lane; v[i] = c < keep ? from[c] : -1; }
#pragma unroll
      for (int i = 0; i < kPlanColumns / 32; ++i) {
        const int c = c0 + 32 * i + lane;
        if (c >= keep && c < end) v[i] = fresh(r, c - have);
        if (c < W) to[c] = v[i];
      }
    }
    return;
  }
  cta -= parts.tables;
  if (cta < parts.rows) {
    // rows of the packed batch
    for (int i = cta * kPlanThreads + tid; i < p.rows; i += parts.rows * kPlanThreads) {
      const int r = upper_bound(s_add, R, i);
      int slot = -1, pos = -1;
      if (r < R && admitted(r)) {
        pos = s_len[r] + i - before(s_add, r);
        const int c = pos / P, have = have_of(r);
        const int page = c < have ? p.table[(size_t)r * W + c] : fresh(r, c - have);
        if (page >= 0) slot = page * P + (pos - c * P);
      }
      p.slots[i] = slot;
      p.positions[i] = pos;
    }
    return;
  }
  cta -= parts.rows;
  // pages that are taken: those of the admitted requests, which are the first ones that need any
  int given = 0;
  for (int r = r0; r < r1; ++r)
    if (admitted(r) && need_of(r) > 0) given = s_need[r];
  if (given) atomicMax(&s_given, given);
  __syncthreads();
  const int left = min(total - s_given, F);
  if (cta < parts.stack) {
    const bool quads = ((reinterpret_cast<uintptr_t>(p.free_pages) | reinterpret_cast<uintptr_t>(p.free_out)) & 15) == 0;
    for (int i = 4 * (cta * kPlanThreads + tid); i < F; i += 4 * parts.stack * kPlanThreads) {
      if (quads && i + 4 <= F && (i >= left || i + 4 <= min(left, n_free))) {
        *reinterpret_cast<int4*>(p.free_out + i) = i >= left ? make_int4(-1, -1, -1, -1) : *reinterpret_cast<const int4*>(p.free_pages + i);
      } else {
        for (int k = i; k < min(i + 4, F); ++k) p.free_out[k] = k < left ? stack(k) : -1;
      }
    }
    return;
  }
  // the requests' state
  int run[1] = {0};
  auto length_after = [&](int r) { return ended(r) ? 0 : admitted(r) ? s_len[r] + p.new_tokens[r] : s_len[r]; };
  for (int r = r0; r < r1; ++r) {
    const int out = length_after(r);
    p.lengths_out[r] = out;
    p.cu_new[r + 1] = s_add[r];
    run[0] = plus(run[0], out);
  }
  sums_before(run, s_warp);
  for (int r = r0; r < r1; ++r) {
    run[0] = plus(run[0], length_after(r));
    p.cu_lengths[r + 1] = run[0];
  }
  if (tid == 0) { p.cu_new[0] = 0; p.cu_lengths[0] = 0; p.n_free_out[0] = left; }
}

// ---- store -----------------------------------------------------------------------------------------------------------------
// A CTA takes the runs that begin among its rows: rows that follow each other into consecutive slots of one block (so a run is at most a block, and
// for prompts nearly always is one).  A warp makes a run's part of a block in shared memory, first K, then V - a row of d numbers is d / 8 lanes with 8
// numbers each, a group of 32 the numbers of four neighbouring lanes - and writes a whole block with 16-byte stores, a part of one by the pieces that its
// tokens own.  What bounds it is the arithmetic of the codes.  Blocks that a run covers whole take a path without tests (32768 tokens of 32 heads of 64, fp16, 352 MB, with
// the reading back: 201 us; with this path, codes clamped as pairs of integers, the divisions and the lengths of runs by fewer operations 163;
// K rows of the next item asked for beside V 153, where those in registers made it slower, 175, and V's as well no faster, 154;
// scales and minima of four rows by four lanes, each for one, and not by all four for each, 150; all V rows asked for at once spill and are no faster, 149 but d = 128 138 for 137).
constexpr int kStoreRows = 64, kStoreWarps = 8;

struct StoreArgs {
  CacheView cache;
  const void *k, *v;
  long long k_row, k_head, v_row, v_head;
  int rows;
  const int32_t* slots;
};

template <class T> struct Pair;          // two numbers of a 16-bit type
template <> struct Pair<__half> { using type = __half2; };
template <> struct Pair<__nv_bfloat16> { using type = __nv_bfloat162; };
template <class T> __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {      // (NaN if one of two is)
  using P = typename Pair<T>::type;
  P r = __hmin2_nan(*reinterpret_cast<P*>(&a), *reinterpret_cast<P*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}
template <class T> __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  using P = typename Pair<T>::type;
  P r = __hmax2_nan(*reinterpret_cast<P*>(&a), *reinterpret_cast<P*>(&b));
  return *reinterpret_cast<uint32_t*>(&r);
}

// x / 15 as the division rounds it (P. Markstein, 1990: one correction of a product with the rounded reciprocal).  Results below 2^-126 are not: they become zero in fp16.
__device__ __forceinline__ float fifteenth(float x) {
  constexpr float c = 1.f / 15.f;
  const float q = x * c;
  return fmaf(fmaf(-15.f, q, x), c, q);
}
// 1 / s for an s from fp16: the approximate reciprocal and one step of Newton's; for each of them what 1.f / s gives.
__device__ __forceinline__ float reciprocal(float s) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
  return fmaf(y, fmaf(-s, y, 1.f), y);
}
// Smallest and minus largest of the lane's 8 numbers, as a pair.
template <class T>
__device__ __forceinline__ uint32_t extremes(const uint4& in) {
  const uint32_t low = min2<T>(min2<T>(in.x, in.y), min2<T>(in.z, in.w)), high = max2<T>(max2<T>(in.x, in.y), max2<T>(in.z, in.w)) ^ 0x80008000u;
  return min2<T>(__byte_perm(low, high, 0x5410), __byte_perm(low, high, 0x7632));
}
// What a group is held with: scale and minimum (fp16), minus the minimum and one over the scale as its codes take them.
struct Held { __half s, m; float minus, r; };
// Of four rows' extremes, each over four neighbouring lanes: lane j of the four gets row j's, and what follows from them.
template <class T>
__device__ __forceinline__ Held held_of(const uint32_t (&e)[4]) {
  const bool b0 = threadIdx.x & 1, b1 = threadIdx.x & 2;
  const uint32_t x0 = min2<T>(b1 ? e[2] : e[0], __shfl_xor_sync(0xffffffffu, b1 ? e[0] : e[2], 2)), x1 = min2<T>(b1 ? e[3] : e[1], __shfl_xor_sync(0xffffffffu, b1 ? e[1] : e[3], 2));
  const float2 f = to_float2<T>(min2<T>(b0 ? x1 : x0, __shfl_xor_sync(0xffffffffu, b0 ? x0 : x1, 1)));
  Held h;
  h.s = __float2half_rn(fifteenth(-f.y - f.x));
  h.m = __float2half_rn(f.x);
  float fs = __half2float(h.s), fm = __half2float(h.m);
  if (!(fabsf(fs) < INFINITY) || !(fabsf(fm) < INFINITY)) {            // (a number that is not finite shows in one of the two)
    h.s = h.m = __ushort_as_half(0x7fff);
    fs = fm = 0.f;
  }
  h.r = fs == 0.f ? 0.f : reciprocal(fs);
  h.minus = -fm;
  return h;
}
// The codes of the lane's 8 numbers, of row j of held_of's four: c[i] = number A(i) and, 16 bits higher, number B(i).
template <class T, class A, class B>
__device__ __forceinline__ void codes8(const uint4& in, const Held& h, int j, A first, B second, uint32_t (&c)[4]) {
  const float m = __shfl_sync(0xffffffffu, h.minus, j, 4), r = __shfl_sync(0xffffffffu, h.r, j, 4);
  const uint64_t minus = pack_f2(m, m), times = pack_f2(r, r);
  const uint32_t w[4] = {in.x, in.y, in.z, in.w};
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = to_float2<T>(w[i]);
    float t0, t1;
    // 1.5 * 2^23 + t is rounded to the nearest integer, ties to even, and has it in its lowest bits (|t| < 32: where s is rounded to a multiple of 2^-24 it is at least two
    // thirds of what it stands for, and m is off by half of one)
    unpack_f2(fmul2(fadd2(pack_f2(x.x, x.y), minus), times), t0, t1);
    u[2 * i] = __float_as_uint(__fadd_rn(t0, 12582912.f));              // (not as a pair: product and sum of pairs become one operation, rounded once)
    u[2 * i + 1] = __float_as_uint(__fadd_rn(t1, 12582912.f));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = __vimin_s16x2_relu(__byte_perm(u[first(i)], u[second(i)], 0x5410), 0x000f000fu);
}

template <int D, class T>
__global__ void __launch_bounds__(32 * kStoreWarps, D == 64 ? 4 : 3) store_kernel(const __grid_constant__ StoreArgs a) {
  using B = Block<D>;
  constexpr int LANES = D / 8, PER = 32 / LANES, STEPS = kBlockTokens / PER, kWindow = kStoreRows + kBlockTokens;     // PER: rows at a time
  __shared__ int s_slot[kWindow + 1], s_run[kStoreRows], s_count[kStoreRows];
  __shared__ unsigned s_begin[kStoreRows / 32], s_break[3];
  __shared__ __align__(16) uint8_t s_block[kStoreWarps][B::kBytes];
  wait_for_stream();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long w0 = (long long)blockIdx.x * kStoreRows;
  // slots of the row before, of the CTA's rows, and of those that a run may reach into
  for (int i = tid; i <= kWindow; i += 32 * kStoreWarps) {
    const long long row = w0 + i - 1;
    const int slot = row >= 0 && row < a.rows ? a.slots[row] : -1;
    s_slot[i] = slot >= 0 && slot / a.cache.page < a.cache.num_pages ? slot : -1;
  }
  __syncthreads();
  auto follows = [&](int i) { return s_slot[i] >= 0 && s_slot[i - 1] >= 0 && s_slot[i] == s_slot[i - 1] + 1 && s_slot[i] % kBlockTokens != 0; };
  // the runs in order (all CTAs of a window have to number them alike), and their lengths: a run ends before the next row that does not follow
  static_assert(kWindow <= 96 && kStoreRows == 64, "three warps look, the first two for beginnings");
  const bool breaks = tid < 96 && !(tid < kWindow && follows(tid + 1)), begins = breaks && tid < kStoreRows && s_slot[tid + 1] >= 0;
  const unsigned flags = __ballot_sync(0xffffffffu, begins), ends = __ballot_sync(0xffffffffu, breaks);
  if (warp < 3 && lane == 0) s_break[warp] = ends;
  if (warp < 2 && lane == 0) s_begin[warp] = flags;
  __syncthreads();
  if (begins) {
    const int run = __popc(flags & ((1u << lane) - 1u)) + (warp ? __popc(s_begin[0]) : 0);
    s_run[run] = tid + 1;
    s_count[run] = __ffs((int)__funnelshift_rc(ends, s_break[warp + 1], lane + 1));       // (at most a block, whose end breaks it)
  }
  __syncthreads();
  const int items = (__popc(s_begin[0]) + __popc(s_begin[1])) * a.cache.heads, warps = kStoreWarps * gridDim.y;
  const int next_run = warps / a.cache.heads, next_head = warps - next_run * a.cache.heads;
  uint8_t* block = s_block[warp];
  const int o = lane % LANES, sub = lane / LANES;
  const int first = blockIdx.y * kStoreWarps + warp;
  int run = first / a.cache.heads, head = first - run * a.cache.heads;
  // The K rows of an item come while the item before is at its V, each lane's into places that it alone reads (zeros for rows that are not the run's).
  extern __shared__ __align__(16) uint8_t s_next[];
  uint8_t* const next = s_next + (warp * STEPS * 32 + lane) * 16;
  auto ask_k = [&](int r, int h) {
    const int at = s_run[r], t0 = s_slot[at] % kBlockTokens, t1 = t0 + s_count[r];               // (a page is whole blocks)
    const T* from = reinterpret_cast<const T*>(a.k) + h * a.k_head + o * 8 + (w0 + at - 1 - t0 + sub) * a.k_row;
#pragma unroll
    for (int i = 0; i < STEPS; ++i, from += PER * a.k_row) {
      const int t = i * PER + sub;
      const bool in = t >= t0 && t < t1;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(next + i * 512)), "l"(in ? from : reinterpret_cast<const T*>(a.k)), "r"(in ? 16 : 0) : "memory");
    }
  };
  if (first < items) ask_k(run, head);
  for (int item = first; item < items; item += warps) {
    const int at = s_run[run], n = s_count[run];
    const int slot = s_slot[at], page = slot / a.cache.page, in_page = slot - page * a.cache.page, t0 = in_page % kBlockTokens;
    const long long row0 = w0 + at - 1 - t0;                               // (the row of the block's token 0)
    auto mine = [&](int t) { return t >= t0 && t < t0 + n; };
    // K: tokens sub, sub + PER, ...; V: a lane takes the four tokens of a word one after the other
    auto k_token = [&](int i) { return i * PER + sub; };
    auto v_token = [&](int i) { return 2 * (sub * (STEPS / 4) + i / 4) + i % 4 / 2 + (i & 1) * 8; };
    auto scales = [&](int at0, int t, __half s, __half m) {
      __half* to = reinterpret_cast<__half*>(block + at0 + ((t / 2) * B::kGroups + o / 4) * 8 + (t % 2) * 2);
      to[0] = s;
      to[2] = m;
    };
    int then_run = run + next_run, then_head = head + next_head;
    if (then_head >= a.cache.heads) { then_head -= a.cache.heads; ++then_run; }
    // (whole: no token of the block is left out)
    auto make = [&](auto whole) {
      constexpr bool WHOLE = decltype(whole)::value;
      const T* vs = reinterpret_cast<const T*>(a.v) + head * a.v_head + o * 8 + (row0 + v_token(0)) * a.v_row;
      uint4 in[STEPS];
      asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
      for (int i4 = 0; i4 < STEPS; i4 += 4) {
        auto row = [&](int i) { return *reinterpret_cast<const uint4*>(next + i * 512); };
        uint32_t e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = extremes<T>(row(i4 + i));
        const Held h = held_of<T>(e);
        scales(B::kScaleK, k_token(i4 + o % 4), h.s, h.m);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = i4 + j, t = k_token(i);
          if (WHOLE || __any_sync(0xffffffffu, mine(t))) {
            uint32_t c[4];
            codes8<T>(row(i), h, j, [](int x) { return 2 * x; }, [](int x) { return 2 * x + 1; }, c);
            // nibble e of the codes is (e % 2) * 4 + e / 2 of the word
            const uint32_t word = c[0] + 16 * c[1] + 256 * (c[2] + 16 * c[3]);
            const int ln = (t % 8) * 4 + o % 4;
            *reinterpret_cast<uint32_t*>(block + (D == 128 ? (t / 8) * 512 + ln * 16 : ln * 16 + (t / 8) * 8) + (o / 4) * 4) = word;
          }
          in[i] = WHOLE || mine(v_token(i)) ? *reinterpret_cast<const uint4*>(vs + (i & 1) * 8 * a.v_row) : make_uint4(0, 0, 0, 0);
          if (i & 1) vs += a.v_row;
        }
      }
      if (item + warps < items) ask_k(then_run, then_head);
#pragma unroll
      for (int i4 = 0; i4 < STEPS; i4 += 4) {
        uint32_t w[4], e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = extremes<T>(in[i4 + i]);
        const Held h = held_of<T>(e);
        scales(B::kScaleV, v_token(i4 + o % 4), h.s, h.m);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = v_token(i4 + i);
          w[i] = 0;
          if (WHOLE || __any_sync(0xffffffffu, mine(t))) {
            uint32_t c[4];
            codes8<T>(in[i4 + i], h, i, [](int x) { return x / 2 * 4 + x % 2; }, [](int x) { return x / 2 * 4 + x % 2 + 2; }, c);
            // the octets of a byte are neighbours: the even lane makes coordinates 0..3 of both, the odd one 4..7
            const uint32_t low = c[0] + 256 * c[1], high = c[2] + 256 * c[3];
            const uint32_t other = __shfl_xor_sync(0xffffffffu, o & 1 ? low : high, 1);
            w[i] = o & 1 ? other + 16 * high : low + 16 * other;
          }
        }
        // four tokens of four coordinates, the other way round
        const uint32_t x0 = __byte_perm(w[0], w[1], 0x5140), x1 = __byte_perm(w[2], w[3], 0x5140), x2 = __byte_perm(w[0], w[1], 0x7362), x3 = __byte_perm(w[2], w[3], 0x7362);
        const int u = o / 2, quad = sub * (STEPS / 4) + i4 / 4;
        uint32_t* to = reinterpret_cast<uint32_t*>(block + B::kV + (u / 4) * 512 + ((o & 1) * 16 + quad) * 16 + (u % 4) * 4);
        to[0] = __byte_perm(x0, x1, 0x5410); to[16] = __byte_perm(x0, x1, 0x7632); to[32] = __byte_perm(x2, x3, 0x5410); to[48] = __byte_perm(x2, x3, 0x7632);
      }
    };
    if (n == kBlockTokens) make(std::true_type());
    else make(std::false_type());
    __syncwarp();
    uint8_t* out = block_at<D>(a.cache, page, head, in_page / kBlockTokens);
    if (n == kBlockTokens) {
#pragma unroll
      for (int i = 0; i < B::kBytes; i += 512) {
        const int x = i + lane * 16;
        if (x < B::kBytes) *reinterpret_cast<uint4*>(out + x) = *reinterpret_cast<const uint4*>(block + x);
      }
    } else {
      // K: D / 2 bytes a token, in pieces of 8 bytes
      for (int i = lane; i < D; i += 32) {
        const int t = D == 128 ? i / 64 * 8 + i % 64 / 8 : i / 8 + (i & 1) * 8;
        if (mine(t)) *reinterpret_cast<uint2*>(out + i * 8) = *reinterpret_cast<const uint2*>(block + i * 8);
      }
      // V: a word has tokens 2 c, 8 + 2 c, 2 c + 1, 9 + 2 c in its bytes
      for (int i = lane; i < 2 * D; i += 32) {
        const int c = i / 4 % 4;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (mine(2 * c + k / 2 + (k & 1) * 8)) out[B::kV + i * 4 + k] = block[B::kV + i * 4 + k];
      }
      // scales and minima: (2 i, 2 i + 1) of a group, twice
      for (int i = lane; i < 2 * D; i += 32) {
        const int t = i / 4 / B::kGroups % 8 * 2 + (i & 1);
        if (mine(t)) reinterpret_cast<__half*>(out + B::kScaleK)[i] = reinterpret_cast<const __half*>(block + B::kScaleK)[i];
      }
    }
    __syncwarp();
    run = then_run;
    head = then_head;
  }
}

// ---- read ------------------------------------------------------------------------------------------------------------------
// A CTA takes some rows of the result, a warp a block of 16 tokens of one head at a time: 16-byte loads of codes and scales; V's words, which hold four
// tokens of two coordinates, are turned by movmatrix so that a lane has neighbouring coordinates of a token, as it has for K.  Rows leave through shared memory.
// 65536 tokens of 8 heads of 128, bf16, 352 MB: 65 us, 5.4 TB/s (84 % of copy bandwidth).
struct ReadArgs {
  CacheView cache;
  const int32_t *table, *cu, *first;
  int requests, width, rows;
  void *k, *v;
};
constexpr int kReadRows = 64, kReadWarps = 4;

template <int D, class T>
__global__ void __launch_bounds__(32 * kReadWarps) read_kernel(const __grid_constant__ ReadArgs a) {
  using B = Block<D>;
  constexpr int G = B::kGroups, kPitch = D * (int)sizeof(T) + 16;        // bytes of a row in shared memory
  __shared__ __align__(16) uint8_t s_rows[kReadWarps][kBlockTokens * kPitch];
  wait_for_stream();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = lane & 3;
  uint8_t* rows = s_rows[warp];
  // The CTA's rows as pieces: rows of one request in one block, numbered in order (several CTAs share the rows of few)
  __shared__ int s_request[kReadRows], s_token[kReadRows], s_piece[kReadRows + 1];
  __shared__ unsigned s_begin[kReadRows / 32];
  static_assert(kReadRows == 64 && kReadWarps >= 2, "two warps look");
  const int tid = threadIdx.x, w0 = blockIdx.x * kReadRows, in_window = min(kReadRows, a.rows - w0), subs = a.cache.page / kBlockTokens;
  if (tid < kReadRows) {
    const int row = w0 + tid, r = upper_bound(a.cu + 1, a.requests, row);
    s_request[tid] = r;
    s_token[tid] = r < a.requests ? (a.first ? a.first[r] : 0) + row - a.cu[r] : tid;               // (beyond the requests: blocks of 16 rows)
  }
  __syncthreads();
  const bool begins = tid < in_window && (tid == 0 || s_request[tid] != s_request[tid - 1] || (s_token[tid] & 15) == 0);
  const unsigned flags = __ballot_sync(0xffffffffu, begins);
  if (tid < kReadRows && lane == 0) s_begin[warp] = flags;
  __syncthreads();
  const int pieces = __popc(s_begin[0]) + __popc(s_begin[1]);
  if (begins) s_piece[__popc(flags & ((1u << lane) - 1u)) + (warp ? __popc(s_begin[0]) : 0)] = tid;
  if (tid == 0) s_piece[pieces] = in_window;
  __syncthreads();
  for (int i = blockIdx.y * kReadWarps + warp; i < pieces * a.cache.heads; i += kReadWarps * gridDim.y) {
    const int piece = i / a.cache.heads, head = i - piece * a.cache.heads, from = s_piece[piece], r = s_request[from], token = s_token[from], b = token >> 4;
    int page = -1;
    if (r < a.requests && b >= 0 && b / subs < a.width) page = a.table[(size_t)r * a.width + b / subs];
    const bool there = page >= 0 && page < a.cache.num_pages;
    const int t_first = token & 15, t_end = t_first + s_piece[piece + 1] - from;                    // tokens of the block that are asked for
    const long long row0 = (long long)w0 + from - t_first;               // (the result's row of the block's token 0)
    auto flush = [&](void* out) {
      __syncwarp();
      constexpr int CHUNKS = D * (int)sizeof(T) / 16;
      for (int e = lane; e < kBlockTokens * CHUNKS; e += 32) {
        const int t = e / CHUNKS, x = e - t * CHUNKS;
        if (t >= t_first && t < t_end)
          reinterpret_cast<uint4*>(reinterpret_cast<T*>(out) + ((row0 + t) * a.cache.heads + head) * D)[x] = there ? *reinterpret_cast<const uint4*>(rows + t * kPitch + x * 16) : make_uint4(0, 0, 0, 0);
      }
      __syncwarp();
    };
    auto put2 = [&](int t, int x, float f0, float f1) {                   // coordinates x, x + 1
      if constexpr (sizeof(T) == 4) *reinterpret_cast<float2*>(rows + t * kPitch + x * 4) = make_float2(f0, f1);
      else *reinterpret_cast<uint32_t*>(rows + t * kPitch + x * 2) = from_float2<T>(f0, f1);
    };
    if (!there) { flush(a.k); flush(a.v); continue; }
    const uint8_t* block = block_at<D>(a.cache, page, head, b % subs);
    uint32_t kw[2][G], vw[D / 16];
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
#pragma unroll
    for (int i4 = 0; i4 < D / 64; ++i4) {
      const uint4 v = *reinterpret_cast<const uint4*>(block + B::kV + i4 * 512 + lane * 16);
      vw[4 * i4] = v.x; vw[4 * i4 + 1] = v.y; vw[4 * i4 + 2] = v.z; vw[4 * i4 + 3] = v.w;
    }
    uint32_t sk[2][2 * G], sv[2][2 * G];                                 // (scales, minima) of the token pair of token lane / 4 (+ 8), by group
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i4 = 0; i4 < G / 2; ++i4) {
        const int at = (half * 4 + lane / 8) * G * 8 + i4 * 16;
        const uint4 x = *reinterpret_cast<const uint4*>(block + B::kScaleK + at), y = *reinterpret_cast<const uint4*>(block + B::kScaleV + at);
        sk[half][4 * i4] = x.x; sk[half][4 * i4 + 1] = x.y; sk[half][4 * i4 + 2] = x.z; sk[half][4 * i4 + 3] = x.w;
        sv[half][4 * i4] = y.x; sv[half][4 * i4 + 1] = y.y; sv[half][4 * i4 + 2] = y.z; sv[half][4 * i4 + 3] = y.w;
      }
    const int odd = (lane >> 2) & 1;                                     // the lane's token is the pair's second
    auto half_of = [&](uint32_t two) { return __half2float(__ushort_as_half((unsigned short)(odd ? two >> 16 : two))); };
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int w = 0; w < G; ++w) {
        const float s = half_of(sk[half][2 * w]), m = half_of(sk[half][2 * w + 1]);
#pragma unroll
        for (int e = 0; e < 4; ++e)                                      // coordinates 2 e, 2 e + 1 of the octet: nibbles e and e + 4
          put2(lane / 4 + 8 * half, 32 * w + 8 * c + 2 * e, fmaf(s, (float)((kw[half][w] >> (4 * e)) & 15u), m), fmaf(s, (float)((kw[half][w] >> (4 * e + 16)) & 15u), m));
      }
    flush(a.k);
#pragma unroll
    for (int u = 0; u < D / 16; ++u) {
      const int w = u / 2;
#pragma unroll
      for (int q = 0; q < 4; ++q) {                                      // nibbles q and q + 4: tokens 2 c, 2 c + 1 (+ 8 for q >= 2) of coordinate 16 u + lane / 4 (+ 8 for odd q)
        uint32_t codes = (vw[u] >> (4 * q)) & 0x000f000fu;
        asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(codes) : "r"(codes));
        // now coordinates 2 c, 2 c + 1 of token lane / 4
        const int half = q / 2;
        const float s = half_of(sv[half][2 * w]), m = half_of(sv[half][2 * w + 1]);
        put2(lane / 4 + 8 * half, 16 * u + 8 * (q & 1) + 2 * c, fmaf(s, (float)(codes & 0xffffu), m), fmaf(s, (float)(codes >> 16), m));
      }
    }
    flush(a.v);
  }
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_cache_plan(const hyperattn_plan* p) {
  if (!p || p->requests < 0 || p->table_width <= 0 || p->num_free < 0 || p->rows < 0 || p->page_tokens <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (p->requests > HYPERATTN_PLAN_MAX_REQUESTS || (long long)p->table_width * p->page_tokens > 0x7fffffffLL || p->table_width >= 1 << 28 ||
      (long long)p->requests * p->table_width + p->num_free > 0x7fffffffLL)
    return HYPERATTN_UNSUPPORTED_SHAPE;
  if (p->requests == 0) return HYPERATTN_OK;
  if (!p->lengths || !p->new_tokens || !p->table || (p->num_free && (!p->free_pages || !p->free_out)) || !p->n_free || (p->rows && (!p->slots || !p->positions)) ||
      !p->cu_new || !p->cu_lengths || !p->lengths_out || !p->table_out || !p->n_free_out)
    return HYPERATTN_INVALID_ARGUMENT;
  if (p->lengths_out == p->lengths || p->table_out == p->table || (p->num_free && p->free_out == p->free_pages) || p->n_free_out == p->n_free) return HYPERATTN_MISALIGNED;
  const int smem = 5 * p->requests * (int)sizeof(int);
  if (smem > 40 * 1024)
    if (int rc = status_of(allow_smem<plan_kernel>(5 * HYPERATTN_PLAN_MAX_REQUESTS * (int)sizeof(int)), "plan: shared memory")) return rc;
  auto ctas = [](long long work, int per, int most) { return (int)(work <= 0 ? 0 : (work + per - 1) / per < most ? (work + per - 1) / per : most); };
  const PlanParts parts = {ctas((long long)p->requests * ((p->table_width + kPlanColumns - 1) / kPlanColumns), kPlanWarps, 2 * kSms), ctas(p->rows, kPlanThreads, kSms / 2),
                           ctas(p->num_free, 8 * kPlanThreads, kSms)};
  return status_of(launch(plan_kernel, dim3((unsigned)(parts.tables + parts.rows + parts.stack + 1)), dim3(kPlanThreads), smem, reinterpret_cast<cudaStream_t>(p->stream), *p, parts), "plan");
}

extern "C" int hyperattn_cache_store(const hyperattn_cache* cache, const void* k, const void* v, int dtype, int rows, long long k_row_stride,
                                     long long k_head_stride, long long v_row_stride, long long v_head_stride, const int32_t* slots, void* stream) {
  int rc;
  if (!cache || rows < 0) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_cache(*cache, &rc)) return rc;
  if (dtype != HYPERATTN_BF16 && dtype != HYPERATTN_FP16) return dtype == HYPERATTN_FP32 ? HYPERATTN_UNSUPPORTED_SHAPE : HYPERATTN_INVALID_ARGUMENT;
  if (rows == 0) return HYPERATTN_OK;
  if (!k || !v || !slots) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_stride(k_row_stride) || bad_stride(k_head_stride) || bad_stride(v_row_stride) || bad_stride(v_head_stride)) return HYPERATTN_UNSUPPORTED_SHAPE;
  if (misaligned(k) || misaligned(v)) return HYPERATTN_MISALIGNED;
  const StoreArgs a = {view_of(*cache), k, v, k_row_stride, k_head_stride, v_row_stride, v_head_stride, rows, slots};
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  // The heads of a window over several CTAs, until there are a few rounds of them: 32768 tokens of 32 heads (d = 64) with twice as many CTAs as SMs at least
  // 181 us, six times 114, twelve times 100 (the first form); with the reading back eight and twelve times 153, 24 times 156 (the form before the last).
  // The kernel needs the registers of four CTAs an SM (d = 128: three); d = 64 with five: 160 for 153.
  const int windows = (rows + kStoreRows - 1) / kStoreRows, most = (kStoreRows * cache->kv_heads + kStoreWarps - 1) / kStoreWarps;
  int split = (12 * kSms + windows - 1) / windows;
  if (split > most) split = most;
  const int smem = kStoreWarps * kBlockTokens * cache->d * 2;
  auto go = [&](auto dim, auto type) {
    constexpr auto kernel = store_kernel<decltype(dim)::value, decltype(type)>;
    cudaError_t e = allow_smem<kernel>(smem);
    if (e == cudaSuccess) e = launch(kernel, dim3((unsigned)windows, (unsigned)split), dim3(32 * kStoreWarps), smem, st, a);
    return status_of(e, "store");
  };
  auto of_type = [&](auto dim) { return dtype == HYPERATTN_BF16 ? go(dim, __nv_bfloat16()) : go(dim, __half()); };
  return cache->d == 64 ? of_type(std::integral_constant<int, 64>()) : of_type(std::integral_constant<int, 128>());
}

extern "C" int hyperattn_cache_read(const hyperattn_cache* cache, const int32_t* table, int requests, int table_width, const int32_t* cu,
                                    const int32_t* first, int rows, void* k, void* v, int dtype, void* stream) {
  int rc;
  if (!cache || rows < 0 || requests < 0 || table_width <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (bad_cache(*cache, &rc)) return rc;
  if (dtype != HYPERATTN_BF16 && dtype != HYPERATTN_FP16 && dtype != HYPERATTN_FP32) return HYPERATTN_INVALID_ARGUMENT;
  if (rows == 0) return HYPERATTN_OK;
  if ((requests && !table) || !cu || !k || !v) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(k) || misaligned(v)) return HYPERATTN_MISALIGNED;
  // (likewise: 65536 tokens of 8 heads (d = 128) 68.0 us with eight times as many CTAs as SMs at least, 65.2 with 24 times, 66.5 with 48)
  const int windows = (rows + kReadRows - 1) / kReadRows, most = (kReadRows * cache->kv_heads + kReadWarps - 1) / kReadWarps;
  int split = (24 * kSms + windows - 1) / windows;
  if (split > most) split = most;
  const ReadArgs a = {view_of(*cache), table, cu, first, requests, table_width, rows, k, v};
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto kernel) { return status_of(launch(kernel, dim3((unsigned)windows, (unsigned)split), dim3(32 * kReadWarps), 0, st, a), "read"); };
  if (cache->d == 64)
    return dtype == HYPERATTN_BF16 ? go(read_kernel<64, __nv_bfloat16>) : dtype == HYPERATTN_FP16 ? go(read_kernel<64, __half>) : go(read_kernel<64, float>);
  return dtype == HYPERATTN_BF16 ? go(read_kernel<128, __nv_bfloat16>) : dtype == HYPERATTN_FP16 ? go(read_kernel<128, __half>) : go(read_kernel<128, float>);
}
