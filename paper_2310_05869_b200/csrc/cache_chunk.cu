// Attention of several new tokens a request over the paged 4-bit cache.
#include "cache_rows.cuh"
#include "cache_tiles.cuh"

using namespace hyperattn;

namespace {
int check(const hyperattn_chunk_params* p) {
  if (int rc = check_chunk(p)) return rc;
  if (p->out_dtype != p->dtype && p->out_dtype != HYPERATTN_FP32) return HYPERATTN_INVALID_ARGUMENT;
  return HYPERATTN_OK;
}
}  // namespace

extern "C" int hyperattn_cache_chunk_attention_workspace_bytes(const hyperattn_chunk_params* p, size_t* bytes) {
  if (!bytes) return HYPERATTN_INVALID_ARGUMENT;
  if (int rc = check(p)) return rc;
  *bytes = 0;
  if (p->requests == 0 || p->rows == 0) return HYPERATTN_OK;
  if (!few_rows_attention(*p, bytes)) return HYPERATTN_UNSUPPORTED_SHAPE;
  return HYPERATTN_OK;
}

extern "C" int hyperattn_cache_chunk_attention(const hyperattn_chunk_params* p) {
  size_t bytes = 0;
  if (int rc = hyperattn_cache_chunk_attention_workspace_bytes(p, &bytes)) return rc;
  if (!p->cu_q && p->rows != p->requests) return HYPERATTN_INVALID_ARGUMENT;
  if (p->requests == 0 || p->rows == 0) return HYPERATTN_OK;
  if (!p->q || !p->out || !p->lse || !p->table || !p->lengths || !p->workspace) return HYPERATTN_INVALID_ARGUMENT;
  if (misaligned(p->q) || misaligned(p->out) || misaligned(p->workspace)) return HYPERATTN_MISALIGNED;
  if (p->workspace_bytes < bytes) return HYPERATTN_WORKSPACE_TOO_SMALL;
  int* status = nullptr;
  if (int rc = device_status_word(reinterpret_cast<cudaStream_t>(p->stream), &status)) return rc;
  return launch_few_rows_attention(*p, status);
}
