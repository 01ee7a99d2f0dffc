// The paged 4-bit cache: pages (plan), storing, reading.
#include <cstdio>
#include "serving.cuh"

namespace hyperattn {
namespace {

// ---- plan ------------------------------------------------------------------------------------------------------------------
// Everything follows from three running sums over the requests (new tokens, pages needed, pages released), which every CTA makes for
// itself in shared memory - reading a few KB again costs less than a launch to make them first - and then takes its share of the tables,
// the stack and the rows.
constexpr int kPlanThreads = 512;

struct PlanShared {      // [R] each, running sums inclusive
  int *add, *need, *rel, *info;      // info: pages the request has, | 1 << 30: admitted, | 1 << 31: ended
};

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(hyperattn_plan p) {
  extern __shared__ int smem[];
  __shared__ int s_warp[3][kPlanThreads / 32];
  wait_for_stream();
  const int R = p.requests, W = p.table_width, P = p.page_tokens, F = p.num_free;
  int *s_add = smem, *s_need = smem + R, *s_rel = smem + 2 * R, *s_have = smem + 3 * R;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n_free = min(max(p.n_free[0], 0), F);

  // a thread takes consecutive requests
  const int per = (R + kPlanThreads - 1) / kPlanThreads, r0 = min(R, tid * per), r1 = min(R, r0 + per);
  int sum[3] = {0, 0, 0};
  for (int r = r0; r < r1; ++r) {
    const int len = max(p.lengths[r], 0), add = p.new_tokens[r];
    const int have = min((len + P - 1) / P, W);
    const long long pages = ((long long)len + max(add, 0) + P - 1) / P;
    const bool ended = add < 0, fits = !ended && pages <= W;
    const int need = fits ? max((int)pages - have, 0) : 0;
    sum[0] += max(add, 0); sum[1] += need; sum[2] += ended ? have : 0;
    s_add[r] = sum[0]; s_need[r] = sum[1]; s_rel[r] = sum[2];
    s_have[r] = have | (fits ? 1 << 29 : 0) | (ended ? 1 << 30 : 0);
  }
  int base[3];
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    int x = sum[q];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
    if (lane == 31) s_warp[q][warp] = x;
    base[q] = x - sum[q];
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < 3; ++q)
    for (int w = 0; w < warp; ++w) base[q] += s_warp[q][w];
  for (int r = r0; r < r1; ++r) { s_add[r] += base[0]; s_need[r] += base[1]; s_rel[r] += base[2]; }
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

  const int threads = gridDim.x * kPlanThreads, gid = blockIdx.x * kPlanThreads + tid;
  // block tables: a thread writes four entries of a row, or one where rows do not start on 16 bytes
  const bool quads = W % 4 == 0 && ((reinterpret_cast<uintptr_t>(p.table) | reinterpret_cast<uintptr_t>(p.table_out)) & 15) == 0;
  const int step = quads ? 4 : 1, row_units = W / step;
  for (long long u = gid; u < (long long)R * row_units; u += threads) {
    const int r = (int)(u / row_units), c = (int)(u - (long long)r * row_units) * step;
    const int have = have_of(r), keep = ended(r) ? 0 : have, end = admitted(r) ? have + need_of(r) : keep;
    const size_t at = (size_t)r * W + c;
    if (quads) {
      int4 v = make_int4(-1, -1, -1, -1);
      if (c < keep) v = *reinterpret_cast<const int4*>(p.table + at);
      int* e = reinterpret_cast<int*>(&v);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i >= keep) e[i] = c + i < end ? fresh(r, c + i - have) : -1;
      *reinterpret_cast<int4*>(p.table_out + at) = v;
    } else {
      p.table_out[at] = c < keep ? p.table[at] : c < end ? fresh(r, c - have) : -1;
    }
  }
  // rows of the packed batch
  for (int i = gid; i < p.rows; i += threads) {
    const int r = upper_bound(s_add, R, i);
    int slot = -1, pos = -1;
    if (r < R && admitted(r)) {
      pos = max(p.lengths[r], 0) + i - before(s_add, r);
      const int c = pos / P, have = have_of(r);
      const int page = c < have ? p.table[(size_t)r * W + c] : fresh(r, c - have);
      if (page >= 0) slot = page * P + (pos - c * P);
    }
    p.slots[i] = slot;
    p.positions[i] = pos;
  }
  // pages that are taken: those of the admitted requests, which are the first ones that need any
  __shared__ int s_given, s_long[kPlanThreads / 32];
  if (tid == 0) s_given = 0;
  __syncthreads();
  int given = 0;
  for (int r = r0; r < r1; ++r)
    if (admitted(r) && need_of(r) > 0) given = s_need[r];
  if (given) atomicMax(&s_given, given);
  __syncthreads();
  const int left = min(total - s_given, F);
  for (int i = gid; i < F; i += threads) p.free_out[i] = i < left ? stack(i) : -1;
  if (blockIdx.x == 0) {
    int len_sum = 0;
    for (int r = r0; r < r1; ++r) {
      const int len = max(p.lengths[r], 0);
      const int out = ended(r) ? 0 : admitted(r) ? len + s_add[r] - before(s_add, r) : len;
      p.lengths_out[r] = out;
      p.cu_new[r + 1] = s_add[r];
      len_sum += out;
    }
    int x = len_sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
    if (lane == 31) s_long[warp] = x;
    __syncthreads();
    int run = x - len_sum;
    for (int w = 0; w < warp; ++w) run += s_long[w];
    for (int r = r0; r < r1; ++r) {
      run += p.lengths_out[r];                          // (written by this thread)
      p.cu_lengths[r + 1] = run;
    }
    if (tid == 0) { p.cu_new[0] = 0; p.cu_lengths[0] = 0; p.n_free_out[0] = left; }
  }
}

// ---- store -----------------------------------------------------------------------------------------------------------------
// A row of d numbers is d / 8 lanes with 8 numbers each, a group of 32 the numbers of four neighbouring lanes.
template <class T>
struct Packed8 {                        // 8 numbers as loaded
  uint4 v;
  __device__ __forceinline__ void floats(float (&x)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 f = to_float2<T>(w[i]); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
  }
};

// codes of the lane's 8 numbers, 4 bits each from bit 0 on; scale and minimum (fp16) of its group
template <class T>
__device__ __forceinline__ uint32_t quantise8(const Packed8<T>& in, __half& s, __half& m) {
  float x[8];
  in.floats(x);
  float lo = x[0], hi = x[0];
  bool finite = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]);
    finite = finite && fabsf(x[i]) < INFINITY;          // (false for NaN)
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const unsigned all = __ballot_sync(0xffffffffu, finite);
  const unsigned mine = 0xfu << (threadIdx.x & 28);
  s = __float2half_rn((hi - lo) / 15.f);
  m = __float2half_rn(lo);
  if ((all & mine) != mine || __hisinf(s) || __hisinf(m)) {
    s = m = __ushort_as_half(0x7fff);
    return 0;
  }
  const float fs = __half2float(s), fm = __half2float(m);
  const float r = fs == 0.f ? 0.f : 1.f / fs;
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = fminf(fmaxf(rintf((x[i] - fm) * r), 0.f), 15.f);
    codes |= (uint32_t)c << (4 * i);
  }
  return codes;
}

struct StoreArgs {
  CacheView cache;
  const void *k, *v;
  long long k_row, k_head, v_row, v_head;
  int rows;
  const int32_t* slots;
};

// A warp takes K and V of one (row, head) at d = 128, of two at d = 64.
template <int D, class T>
__global__ void __launch_bounds__(256) store_kernel(StoreArgs a) {
  wait_for_stream();
  constexpr int LANES = D / 8;                          // lanes of a row
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * (256 / (2 * LANES)) + threadIdx.x / (2 * LANES);
  const bool is_v = (lane / LANES) & 1;
  const int o = lane % LANES;                           // octet of the row
  const long long row = item / a.cache.heads;
  const int head = (int)(item - row * a.cache.heads);
  const int slot = row < a.rows ? a.slots[row] : -1;
  const int page = slot < 0 ? -1 : slot / a.cache.page;
  const bool there = page >= 0 && page < a.cache.num_pages;
  Packed8<T> in = {make_uint4(0, 0, 0, 0)};
  if (there) {
    const T* src = is_v ? reinterpret_cast<const T*>(a.v) + row * a.v_row + head * a.v_head : reinterpret_cast<const T*>(a.k) + row * a.k_row + head * a.k_head;
    in.v = *reinterpret_cast<const uint4*>(src + o * 8);
  }
  __half s, m;
  const uint32_t codes = quantise8(in, s, m);
  const uint32_t other = __shfl_xor_sync(0xffffffffu, codes, 1);
  if (!there) return;
  const int in_page = slot - page * a.cache.page, t = in_page % kBlockTokens;
  uint8_t* block = block_at<D>(a.cache, page, head, in_page / kBlockTokens);
  if (!is_v) {
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) word |= ((codes >> (4 * e)) & 15u) << (4 * ((e % 2) * 4 + e / 2));
    const int ln = (t % 8) * 4 + o % 4;
    const int at = (D == 128 ? (t / 8) * 512 + ln * 16 : ln * 16 + (t / 8) * 8) + (o / 4) * 4;
    *reinterpret_cast<uint32_t*>(block + at) = word;
  } else {
    // the octets of a byte are neighbours: the even lane writes coordinates 0..3 of both, the odd one 4..7
    const uint32_t low = (o & 1) ? other : codes, high = (o & 1) ? codes : other;
    const int u = o / 2;
    uint8_t* at = block + Block<D>::kV + (u / 4) * 512 + (t % 8 / 2) * 16 + (u % 4) * 4 + (t % 2) * 2 + t / 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (o & 1) * 4 + i;
      at[r * 64] = (uint8_t)(((low >> (4 * r)) & 15u) | (((high >> (4 * r)) & 15u) << 4));
    }
  }
  if (o % 4 == 0) {
    __half* at = reinterpret_cast<__half*>(block + (is_v ? Block<D>::kScaleV : Block<D>::kScaleK) + ((t / 2) * Block<D>::kGroups + o / 4) * 8 + (t % 2) * 2);
    at[0] = s;
    at[2] = m;
  }
}

// ---- read ------------------------------------------------------------------------------------------------------------------
struct ReadArgs {
  CacheView cache;
  const int32_t *table, *cu, *first;
  int requests, width, rows;
  void *k, *v;
};

template <class T> __device__ __forceinline__ void put8(T* to, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(to) = make_uint4(from_float2<T>(x[0], x[1]), from_float2<T>(x[2], x[3]), from_float2<T>(x[4], x[5]), from_float2<T>(x[6], x[7]));
}
template <> __device__ __forceinline__ void put8<float>(float* to, const float (&x)[8]) {
  reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

template <int D, class T>
__global__ void __launch_bounds__(256) read_kernel(ReadArgs a) {
  wait_for_stream();
  constexpr int LANES = D / 8;
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * (256 / (2 * LANES)) + threadIdx.x / (2 * LANES);
  const bool is_v = (lane / LANES) & 1;
  const int o = lane % LANES;
  const long long row = item / a.cache.heads;
  const int head = (int)(item - row * a.cache.heads);
  if (row >= a.rows) return;
  const int r = upper_bound(a.cu + 1, a.requests, (int)row);
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  int page = -1, token = 0;
  if (r < a.requests) {
    token = (int)row - a.cu[r] + (a.first ? a.first[r] : 0);
    const int c = token / a.cache.page;
    if (token >= 0 && c < a.width) page = a.table[(size_t)r * a.width + c];
  }
  if (page >= 0 && page < a.cache.num_pages) {
    const int in_page = token % a.cache.page, t = in_page % kBlockTokens;
    const uint8_t* block = block_at<D>(a.cache, page, head, in_page / kBlockTokens);
    const __half* sc = reinterpret_cast<const __half*>(block + (is_v ? Block<D>::kScaleV : Block<D>::kScaleK) + ((t / 2) * Block<D>::kGroups + o / 4) * 8 + (t % 2) * 2);
    const float s = __half2float(sc[0]), m = __half2float(sc[2]);
    if (!is_v) {
      const int ln = (t % 8) * 4 + o % 4;
      const int at = (D == 128 ? (t / 8) * 512 + ln * 16 : ln * 16 + (t / 8) * 8) + (o / 4) * 4;
      const uint32_t word = *reinterpret_cast<const uint32_t*>(block + at);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fmaf(s, (float)((word >> (4 * ((e % 2) * 4 + e / 2))) & 15u), m);
    } else {
      const int u = o / 2;
      const uint8_t* at = block + Block<D>::kV + (u / 4) * 512 + (t % 8 / 2) * 16 + (u % 4) * 4 + (t % 2) * 2 + t / 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fmaf(s, (float)((at[i * 64] >> (4 * (o & 1))) & 15u), m);
    }
  }
  put8<T>(reinterpret_cast<T*>(is_v ? a.v : a.k) + (row * a.cache.heads + head) * D + o * 8, x);
}

CacheView view_of(const hyperattn_cache& c) { return {reinterpret_cast<uint8_t*>(c.pages), c.num_pages, c.page_tokens, c.kv_heads}; }
int status_of(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return HYPERATTN_OK;
  std::fprintf(stderr, "hyperattn: %s failed: %s\n", what, cudaGetErrorString(e));
  return HYPERATTN_CUDA_ERROR;
}

}  // namespace
}  // namespace hyperattn

using namespace hyperattn;

extern "C" int hyperattn_cache_plan(const hyperattn_plan* p) {
  if (!p || p->requests < 0 || p->table_width <= 0 || p->num_free < 0 || p->rows < 0 || p->page_tokens <= 0) return HYPERATTN_INVALID_ARGUMENT;
  if (p->requests > HYPERATTN_PLAN_MAX_REQUESTS || (long long)p->table_width * p->page_tokens > 0x7fffffffLL) return HYPERATTN_UNSUPPORTED_SHAPE;
  if (p->requests == 0) return HYPERATTN_OK;
  if (!p->lengths || !p->new_tokens || !p->table || (p->num_free && (!p->free_pages || !p->free_out)) || !p->n_free || (p->rows && (!p->slots || !p->positions)) ||
      !p->cu_new || !p->cu_lengths || !p->lengths_out || !p->table_out || !p->n_free_out)
    return HYPERATTN_INVALID_ARGUMENT;
  if (p->lengths_out == p->lengths || p->table_out == p->table || (p->num_free && p->free_out == p->free_pages) || p->n_free_out == p->n_free) return HYPERATTN_MISALIGNED;
  const int smem = 4 * p->requests * (int)sizeof(int);
  if (smem > 40 * 1024)
    if (int rc = status_of(allow_smem<plan_kernel>(4 * HYPERATTN_PLAN_MAX_REQUESTS * (int)sizeof(int)), "plan: shared memory")) return rc;
  const long long work = (long long)p->requests * p->table_width / 4 + p->rows + p->num_free / 4;
  long long grid = (work + 2 * kPlanThreads - 1) / (2 * kPlanThreads);
  if (grid > 2 * kSms) grid = 2 * kSms;
  if (grid < 1) grid = 1;
  return status_of(launch(plan_kernel, dim3((unsigned)grid), dim3(kPlanThreads), smem, reinterpret_cast<cudaStream_t>(p->stream), *p), "plan");
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
  const int per = 256 / (cache->d / 4);
  const long long grid = ((long long)rows * cache->kv_heads + per - 1) / per;
  if (grid > 0x7fffffffLL) return HYPERATTN_UNSUPPORTED_SHAPE;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto kernel) { return status_of(launch(kernel, dim3((unsigned)grid), dim3(256), 0, st, a), "store"); };
  if (cache->d == 64) return dtype == HYPERATTN_BF16 ? go(store_kernel<64, __nv_bfloat16>) : go(store_kernel<64, __half>);
  return dtype == HYPERATTN_BF16 ? go(store_kernel<128, __nv_bfloat16>) : go(store_kernel<128, __half>);
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
  const ReadArgs a = {view_of(*cache), table, cu, first, requests, table_width, rows, k, v};
  const int per = 256 / (cache->d / 4);
  const long long grid = ((long long)rows * cache->kv_heads + per - 1) / per;
  if (grid > 0x7fffffffLL) return HYPERATTN_UNSUPPORTED_SHAPE;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  auto go = [&](auto kernel) { return status_of(launch(kernel, dim3((unsigned)grid), dim3(256), 0, st, a), "read"); };
  if (cache->d == 64)
    return dtype == HYPERATTN_BF16 ? go(read_kernel<64, __nv_bfloat16>) : dtype == HYPERATTN_FP16 ? go(read_kernel<64, __half>) : go(read_kernel<64, float>);
  return dtype == HYPERATTN_BF16 ? go(read_kernel<128, __nv_bfloat16>) : dtype == HYPERATTN_FP16 ? go(read_kernel<128, __half>) : go(read_kernel<128, float>);
}
