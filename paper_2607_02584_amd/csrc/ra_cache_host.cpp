// ra_cache_host.cpp -- entry points of the 4-bit paged KV cache: argument
// validation and launches.  Everything is checked before the GPU is touched;
// nothing here allocates or throws.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "../../include/rotate_attn.h"
#include "ra_cache.h"

namespace {

using ra::set_error;

int hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return RA_OK;
  char msg[160];
  std::snprintf(msg, sizeof msg, "%s: %s", what, hipGetErrorString(e));
  return set_error(RA_ERR_HIP, msg);
}

int log2_of(int x) {
  int n = 0;
  while ((1 << n) < x) ++n;
  return n;
}

int validate(const ra_cache_params* p) {
  if (!p) return set_error(RA_ERR_INVALID, "params is NULL");
  if (p->D != 64 && p->D != 128) return set_error(RA_ERR_UNSUPPORTED, "the cache supports D == 64 and D == 128");
  if (p->Hq < 1 || p->Hkv < 1) return set_error(RA_ERR_INVALID, "Hq and Hkv must be >= 1");
  if (p->Hq > 1024) return set_error(RA_ERR_UNSUPPORTED, "Hq above 1024 is not supported");
  if (p->Hq % p->Hkv) return set_error(RA_ERR_INVALID, "Hq must be a multiple of Hkv");
  if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128 && p->page_size != 256)
    return set_error(RA_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256");
  if (p->num_pages < 1 || p->max_blocks < 1) return set_error(RA_ERR_INVALID, "num_pages and max_blocks must be >= 1");
  // slots and positions are 32-bit numbers
  if (static_cast<int64_t>(p->num_pages) * p->page_size > 0x7fffffff)
    return set_error(RA_ERR_UNSUPPORTED, "num_pages * page_size must stay below 2^31");
  if (static_cast<int64_t>(p->max_blocks) * p->page_size > (1 << 30))
    return set_error(RA_ERR_UNSUPPORTED, "max_blocks * page_size must not exceed 2^30");
  if (p->rotation != RA_ROT_NONE && p->rotation != RA_ROT_HADAMARD)
    return set_error(RA_ERR_UNSUPPORTED, "the cache rotates by RA_ROT_NONE or RA_ROT_HADAMARD");
  if (p->v_rotation != RA_VROT_NONE && p->v_rotation != RA_VROT_HADAMARD)
    return set_error(RA_ERR_INVALID, "unknown v_rotation");
  if (p->causal != 0 && p->causal != 1) return set_error(RA_ERR_INVALID, "causal must be 0 or 1");
  if (p->window < 0) return set_error(RA_ERR_INVALID, "window must be >= 0");
  if (p->window > (1 << 30)) return set_error(RA_ERR_UNSUPPORTED, "window must not exceed 2^30");
  if (p->window && !p->causal) return set_error(RA_ERR_UNSUPPORTED, "a window needs causal attention");
  if (!(p->sm_scale >= 0.0f) || !std::isfinite(p->sm_scale)) return set_error(RA_ERR_INVALID, "sm_scale must be >= 0");
  if (p->in_dtype != RA_BF16 && p->in_dtype != RA_FP16)
    return set_error(RA_ERR_INVALID, "in_dtype must be BF16 or FP16");
  if (p->out_dtype != RA_BF16 && p->out_dtype != RA_FP16 && p->out_dtype != RA_FP32)
    return set_error(RA_ERR_INVALID, "out_dtype must be BF16, FP16 or FP32");
  return RA_OK;
}

int64_t page_bytes(const ra_cache_params* p) {
  return static_cast<int64_t>(p->Hkv) * p->page_size * (p->D + 8);
}

ra::CacheGeom geom(const ra_cache_params* p, void* cache) {
  ra::CacheGeom g;
  g.cache = static_cast<uint8_t*>(cache);
  g.page_bytes = page_bytes(p);
  g.num_pages = p->num_pages;
  g.page = p->page_size;
  g.page_log = log2_of(p->page_size);
  g.Hkv = p->Hkv;
  return g;
}

bool aligned(const void* ptr, unsigned n) { return reinterpret_cast<uintptr_t>(ptr) % n == 0; }

// Rows of 16-bit values are read in 16-byte pieces.
int check_rows(const char* name, const void* ptr, int64_t token_stride, int64_t head_stride) {
  char msg[120];
  if (!aligned(ptr, 16)) {
    std::snprintf(msg, sizeof msg, "%s must be 16-byte aligned", name);
    return set_error(RA_ERR_INVALID, msg);
  }
  if (token_stride < 0 || head_stride < 0 || token_stride % 8 || head_stride % 8) {
    std::snprintf(msg, sizeof msg, "the strides of %s must be multiples of 8 elements", name);
    return set_error(RA_ERR_INVALID, msg);
  }
  return RA_OK;
}

int check_rope(const ra_cache_params* p, const float* rope, int32_t rope_rows) {
  (void)p;
  if (!rope) return RA_OK;
  if (!aligned(rope, 16)) return set_error(RA_ERR_INVALID, "rope must be 16-byte aligned");
  if (rope_rows < 1) return set_error(RA_ERR_INVALID, "rope_rows must be >= 1");
  return RA_OK;
}

int check_counts(int32_t R, int32_t T) {
  if (R < 0 || T < 0) return set_error(RA_ERR_INVALID, "R and T must be >= 0");
  if (R > 65536) return set_error(RA_ERR_UNSUPPORTED, "R above 65536 requests is not supported");
  if (T > (1 << 24)) return set_error(RA_ERR_UNSUPPORTED, "T above 2^24 tokens is not supported");
  return RA_OK;
}

// A launch holds 2^32 work-items along the grid, 256 per workgroup: a request's
// tiles of 128 rows (or its only one) for every KV head, and up to 1024 + Hkv
// more for the parts of split ones.  Rows of a request then stay below 2^31, too.
int check_pieces(const ra_cache_params* p, int32_t R, int32_t T) {
  const int64_t pieces = static_cast<int64_t>(R) * p->Hkv + static_cast<int64_t>(T) * p->Hq / 128;
  if (pieces >= (1 << 24) - 4096)
    return set_error(RA_ERR_UNSUPPORTED, "R * Hkv + T * Hq / 128 must stay below 2^24 - 4096");
  return RA_OK;
}

}  // namespace

extern "C" {

int rotate_attn_cache_layout(const ra_cache_params* p, ra_cache_sizes* out) {
  const int rc = validate(p);
  if (rc) return rc;
  if (!out) return set_error(RA_ERR_INVALID, "out is NULL");
  out->head_bytes = static_cast<int64_t>(p->page_size) * (p->D + 8);
  out->page_bytes = page_bytes(p);
  out->cache_bytes = page_bytes(p) * p->num_pages;
  out->v_codes = static_cast<int64_t>(p->page_size) * p->D / 2;
  out->k_scales = static_cast<int64_t>(p->page_size) * p->D;
  out->v_scales = out->k_scales + 4 * static_cast<int64_t>(p->page_size);
  return RA_OK;
}

int rotate_attn_cache_workspace_size(const ra_cache_params* p, int32_t R, int32_t T, int32_t max_q, size_t* bytes) {
  int rc = validate(p);
  if (rc) return rc;
  if ((rc = check_counts(R, T))) return rc;
  if ((rc = check_pieces(p, R, T))) return rc;
  if (max_q < 0) return set_error(RA_ERR_INVALID, "max_q must be >= 0");
  if (!bytes) return set_error(RA_ERR_INVALID, "bytes is NULL");
  size_t ml;
  *bytes = ra::cache_attn_partial_bytes(p->D, p->Hkv, p->Hq / p->Hkv, max_q, &ml);
  return RA_OK;
}

int rotate_attn_cache_plan(const ra_cache_params* p, int32_t R, int32_t T, const int32_t* seq_lens,
                           const int32_t* new_lens, const int32_t* release, int32_t* block_table, int32_t* free_pages,
                           const int32_t* free_count, int32_t* seq_out, int32_t* count_out, int32_t* q_start,
                           int32_t* positions, int32_t* slots, int32_t* status, void* stream) {
  int rc = validate(p);
  if (rc) return rc;
  if ((rc = check_counts(R, T))) return rc;
  if (!free_pages || !free_count || !count_out || !q_start || !status ||
      (R && (!seq_lens || !new_lens || !block_table || !seq_out)) || (T && (!positions || !slots)))
    return set_error(RA_ERR_INVALID, "NULL tensor pointer");
  // lengths and count may be updated in place; new_lens is read after seq_out is written
  if (R && (seq_out == new_lens || seq_out == release)) return set_error(RA_ERR_INVALID, "seq_out must not be new_lens or release");
  ra::PlanArgs a;
  a.seq_lens = seq_lens;
  a.new_lens = new_lens;
  a.release = release;
  a.block_table = block_table;
  a.free_pages = free_pages;
  a.free_count = free_count;
  a.seq_out = seq_out;
  a.count_out = count_out;
  a.q_start = q_start;
  a.positions = positions;
  a.slots = slots;
  a.status = status;
  a.R = R;
  a.T = T;
  a.max_blocks = p->max_blocks;
  a.num_pages = p->num_pages;
  a.page = p->page_size;
  a.page_log = log2_of(p->page_size);
  return hip_status(ra::launch_cache_plan(a, static_cast<hipStream_t>(stream)), "cache_plan");
}

int rotate_attn_cache_append(const ra_cache_params* p, int32_t T, const void* k, int64_t k_token_stride,
                             int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride,
                             const int32_t* slots, const int32_t* positions, const float* rope, int32_t rope_rows,
                             void* cache, void* stream) {
  int rc = validate(p);
  if (rc) return rc;
  if ((rc = check_counts(0, T))) return rc;
  if (T == 0) return RA_OK;
  if (!k || !v || !slots || !cache) return set_error(RA_ERR_INVALID, "NULL tensor pointer");
  if (rope && !positions) return set_error(RA_ERR_INVALID, "rope needs positions");
  if ((rc = check_rows("k", k, k_token_stride, k_head_stride))) return rc;
  if ((rc = check_rows("v", v, v_token_stride, v_head_stride))) return rc;
  if ((rc = check_rope(p, rope, rope_rows))) return rc;
  if (!aligned(cache, 128)) return set_error(RA_ERR_INVALID, "cache must be 128-byte aligned");
  ra::AppendArgs a;
  a.g = geom(p, cache);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.k_ts = k_token_stride;
  a.k_hs = k_head_stride;
  a.v_ts = v_token_stride;
  a.v_hs = v_head_stride;
  a.slots = slots;
  a.positions = positions;
  a.rope = rope;
  a.rope_rows = rope_rows;
  a.T = T;
  a.is_fp16 = p->in_dtype == RA_FP16;
  a.heads = 1;
  return hip_status(ra::launch_cache_append(a, p->D, p->rotation == RA_ROT_HADAMARD, p->v_rotation == RA_VROT_HADAMARD,
                                            static_cast<hipStream_t>(stream)), "cache_append");
}

int rotate_attn_cache_read(const ra_cache_params* p, int32_t T, const void* cache, const int32_t* slots, void* k,
                           void* v, void* stream) {
  int rc = validate(p);
  if (rc) return rc;
  if ((rc = check_counts(0, T))) return rc;
  if (T == 0) return RA_OK;
  if (!k || !v || !slots || !cache) return set_error(RA_ERR_INVALID, "NULL tensor pointer");
  if (!aligned(k, 16) || !aligned(v, 16)) return set_error(RA_ERR_INVALID, "k and v must be 16-byte aligned");
  if (!aligned(cache, 128)) return set_error(RA_ERR_INVALID, "cache must be 128-byte aligned");
  ra::ReadArgs a;
  a.g = geom(p, const_cast<void*>(cache));
  a.slots = slots;
  a.k = k;
  a.v = v;
  a.T = T;
  a.out_dtype = p->out_dtype;
  a.heads = 1;
  return hip_status(ra::launch_cache_read(a, p->D, p->rotation == RA_ROT_HADAMARD, p->v_rotation == RA_VROT_HADAMARD,
                                          static_cast<hipStream_t>(stream)), "cache_read");
}

int rotate_attn_cache_attn(const ra_cache_params* p, int32_t R, int32_t T, int32_t max_q, const void* q,
                           int64_t q_token_stride, int64_t q_head_stride, const void* cache,
                           const int32_t* block_table, const int32_t* q_start, const int32_t* seq_lens,
                           const float* rope, int32_t rope_rows, void* o, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
  int rc = validate(p);
  if (rc) return rc;
  if ((rc = check_counts(R, T))) return rc;
  if ((rc = check_pieces(p, R, T))) return rc;
  if (max_q < 0) return set_error(RA_ERR_INVALID, "max_q must be >= 0");
  if (R == 0 || T == 0 || max_q == 0) return RA_OK;
  if (max_q > T) max_q = T;
  if (!q || !cache || !block_table || !q_start || !seq_lens || !o) return set_error(RA_ERR_INVALID, "NULL tensor pointer");
  if ((rc = check_rows("q", q, q_token_stride, q_head_stride))) return rc;
  if ((rc = check_rope(p, rope, rope_rows))) return rc;
  if (!aligned(cache, 128)) return set_error(RA_ERR_INVALID, "cache must be 128-byte aligned");
  if (!aligned(o, 16)) return set_error(RA_ERR_INVALID, "o must be 16-byte aligned");
  size_t ml;
  const int G = p->Hq / p->Hkv;
  const size_t need = ra::cache_attn_partial_bytes(p->D, p->Hkv, G, max_q, &ml);
  if (!workspace) return set_error(RA_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(workspace, 256)) return set_error(RA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace_bytes < need) {
    char msg[96];
    std::snprintf(msg, sizeof msg, "workspace too small: need %zu bytes", need);
    return set_error(RA_ERR_WORKSPACE, msg);
  }
  ra::CacheAttnArgs a;
  a.g = geom(p, const_cast<void*>(cache));
  a.q = static_cast<const uint16_t*>(q);
  a.q_ts = q_token_stride;
  a.q_hs = q_head_stride;
  a.block_table = block_table;
  a.q_start = q_start;
  a.seq_lens = seq_lens;
  a.rope = rope;
  a.rope_rows = rope_rows;
  a.o = o;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + ml);
  const double scale = p->sm_scale == 0.0f ? 1.0 / std::sqrt(static_cast<double>(p->D)) : p->sm_scale;
  const double norm = p->rotation == RA_ROT_HADAMARD ? 1.0 / std::sqrt(static_cast<double>(p->D)) : 1.0;
  a.c = static_cast<float>(scale * norm * 1.4426950408889634);   // base 2
  a.R = R;
  a.T = T;
  a.max_q = max_q;
  a.Hq = p->Hq;
  a.G = G;
  a.max_blocks = p->max_blocks;
  a.causal = p->causal;
  a.window = p->window;
  a.is_fp16 = p->in_dtype == RA_FP16;
  a.out_dtype = p->out_dtype;
  a.had = p->rotation == RA_ROT_HADAMARD;
  a.vhad = p->v_rotation == RA_VROT_HADAMARD;
  a.target = a.target_rows = 0;
  return hip_status(ra::launch_cache_attn(a, p->D, static_cast<hipStream_t>(stream)), "cache_attn");
}

}  // extern "C"
