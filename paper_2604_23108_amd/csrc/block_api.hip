// Host side of mohge_block.h: argument checks and dispatch to the launchers.
#include "block.h"

using namespace mohge;

#define NEED(p) do { int rc_ = need((p), #p, true); if (rc_) return rc_; } while (0)
#define OPT(p) do { int rc_ = need((p), #p, false); if (rc_) return rc_; } while (0)

namespace {

int check_norm(const mohge_norm_config* c) {
  if (!c) { set_error("cfg is NULL"); return MOHGE_ENULL; }
  if (c->T < 0 || c->T > 1 << 21) { set_error("T = %d outside 0..2^21", c->T); return MOHGE_EINVAL; }
  if (c->d < 8 || c->d % 8 || c->d > 32768) {
    set_error("d = %d must be a multiple of 8 in 8..32768", c->d); return MOHGE_EINVAL; }
  if (c->dtype != MOHGE_F32 && c->dtype != MOHGE_BF16) { set_error("dtype = %d unknown", c->dtype); return MOHGE_EINVAL; }
  if (c->y_dtype != c->dtype && c->y_dtype != MOHGE_E4M3) {
    set_error("y_dtype = %d must be dtype or MOHGE_E4M3", c->y_dtype); return MOHGE_EINVAL; }
  if (!(c->eps >= 0.f)) { set_error("eps = %g must not be negative", c->eps); return MOHGE_EINVAL; }
  return MOHGE_OK;
}

int check_cache(const mohge_cache_config* c) {
  if (!c) { set_error("cfg is NULL"); return MOHGE_ENULL; }
  if (c->n_seqs < 0) { set_error("n_seqs = %d is negative", c->n_seqs); return MOHGE_EINVAL; }
  if (c->n_kv_heads < 1 || c->n_heads < 1 || c->n_heads % c->n_kv_heads) {
    set_error("n_heads = %d must be a positive multiple of n_kv_heads = %d", c->n_heads, c->n_kv_heads);
    return MOHGE_EINVAL; }
  if (c->n_heads > 1024) { set_error("n_heads = %d outside 1..1024", c->n_heads); return MOHGE_EINVAL; }
  if ((int64_t)c->n_seqs * c->n_heads >= (int64_t)1 << 24) {
    set_error("n_seqs*n_heads = %lld must be less than 2^24", (long long)c->n_seqs * c->n_heads); return MOHGE_EINVAL; }
  if (c->head_size != 64 && c->head_size != 128 && c->head_size != 256) {
    set_error("head_size = %d must be 64, 128 or 256", c->head_size); return MOHGE_EINVAL; }
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) {
    set_error("page_size = %d must be 16, 32, 64, 128 or 256", c->page_size); return MOHGE_EINVAL; }
  if (c->n_pages < 1 || c->max_pages < 1) { set_error("n_pages and max_pages must be positive"); return MOHGE_EINVAL; }
  // (positions are int32, and the attention rounds them up to its units)
  if ((int64_t)c->max_pages * c->page_size > (int64_t)1 << 30) {
    set_error("max_pages*page_size must be at most 2^30: positions are int32"); return MOHGE_EINVAL; }
  // (the attention numbers its units of 64 positions or more in 32 bits)
  if ((int64_t)c->n_seqs * c->n_heads * ((int64_t)c->max_pages * c->page_size / 64 + 1) >= (int64_t)1 << 31) {
    set_error("n_seqs*n_heads*max_pages*page_size must be less than 2^37"); return MOHGE_EINVAL; }
  if (c->dtype != MOHGE_F32 && c->dtype != MOHGE_BF16) { set_error("dtype = %d unknown", c->dtype); return MOHGE_EINVAL; }
  if (c->cache_dtype != c->dtype && !(c->cache_dtype == MOHGE_E4M3 && c->dtype == MOHGE_BF16)) {
    set_error("cache_dtype = %d must be dtype, or MOHGE_E4M3 with MOHGE_BF16", c->cache_dtype); return MOHGE_EINVAL; }
  return MOHGE_OK;
}

// distance between rows of `width` elements
int check_stride(int64_t stride, int64_t width, const char* name) {
  if (stride < width) { set_error("%s = %lld is less than a row of %lld", name, (long long)stride, (long long)width); return MOHGE_EINVAL; }
  if (stride % 8) { set_error("%s = %lld is not a multiple of 8", name, (long long)stride); return MOHGE_EALIGN; }
  return MOHGE_OK;
}

int check_cache_pointers(const mohge_cache_config* cfg, const int32_t* block_table, const int32_t* seq_lens,
                         const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale) {
  NEED(block_table); NEED(seq_lens); NEED(k_pages); NEED(v_pages);
  if (cfg->cache_dtype == MOHGE_E4M3) { NEED(k_scale); NEED(v_scale); }
  else if (k_scale || v_scale) { set_error("k_scale / v_scale given for a cache without scales"); return MOHGE_EINVAL; }
  return MOHGE_OK;
}

int check_proj(const mohge_proj_config* c) {
  if (!c) { set_error("cfg is NULL"); return MOHGE_ENULL; }
  if (c->T < 0 || c->T > 32) { set_error("T = %d outside 0..32", c->T); return MOHGE_EINVAL; }
  if (c->group != 32 && c->group != 64 && c->group != 128) {
    set_error("group = %d must be 32, 64 or 128", c->group); return MOHGE_EINVAL; }
  if (c->n_in < c->group || c->n_in % c->group || c->n_in > 1 << 20) {
    set_error("n_in = %d must be a multiple of group = %d in 1..2^20", c->n_in, c->group); return MOHGE_EINVAL; }
  if (c->n_out < 1 || c->n_out > 1 << 24) { set_error("n_out = %d outside 1..2^24", c->n_out); return MOHGE_EINVAL; }
  if (c->x_dtype != MOHGE_BF16 && c->x_dtype != MOHGE_E4M3) {
    set_error("x_dtype = %d must be MOHGE_BF16 or MOHGE_E4M3", c->x_dtype); return MOHGE_EINVAL; }
  if (c->y_dtype != MOHGE_BF16 && c->y_dtype != MOHGE_F32) {
    set_error("y_dtype = %d must be MOHGE_BF16 or MOHGE_F32", c->y_dtype); return MOHGE_EINVAL; }
  return MOHGE_OK;
}

}  // namespace

extern "C" {

int mohge_rmsnorm(const mohge_norm_config* cfg, const void* x, const void* residual, const float* weight,
                  void* sum_out, void* y, float* y_scale, float* rstd, void* stream) {
  int rc = check_norm(cfg);
  if (rc) return rc;
  if (cfg->T == 0) return MOHGE_OK;
  NEED(x); OPT(residual); NEED(weight); OPT(sum_out); NEED(y); OPT(rstd);
  if (cfg->y_dtype == MOHGE_E4M3) NEED(y_scale);
  else if (y_scale) { set_error("y_scale given for an output without scales"); return MOHGE_EINVAL; }
  return hip_rc(launch_rmsnorm(*cfg, x, residual, weight, sum_out, y, y_scale, rstd, (hipStream_t)stream),
                "mohge_rmsnorm");
}

size_t mohge_norm_workspace_size(const mohge_norm_config* cfg) {
  return check_norm(cfg) ? 0 : norm_workspace_bytes(*cfg);
}

int mohge_rmsnorm_bwd(const mohge_norm_config* cfg, const void* dy, const void* h, const float* weight,
                      const float* rstd, const void* dsum, void* dx, float* dweight, void* workspace,
                      size_t workspace_bytes, void* stream) {
  int rc = check_norm(cfg);
  if (rc) return rc;
  NEED(dweight); NEED(workspace);
  if (cfg->T > 0) { NEED(dy); NEED(h); NEED(weight); NEED(rstd); OPT(dsum); NEED(dx); }
  if (workspace_bytes < norm_workspace_bytes(*cfg)) {
    set_error("rmsnorm_bwd workspace: %zu bytes given, %zu needed", workspace_bytes, norm_workspace_bytes(*cfg));
    return MOHGE_EWORKSPACE;
  }
  return hip_rc(launch_rmsnorm_bwd(*cfg, dy, h, weight, rstd, dsum, dx, dweight, workspace, (hipStream_t)stream),
                "mohge_rmsnorm_bwd");
}

int mohge_cache_append(const mohge_cache_config* cfg, int32_t n_tokens, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, const int32_t* tok_offsets, const int32_t* block_table,
                       const int32_t* seq_lens, void* k_pages, void* v_pages, float* k_scale, float* v_scale,
                       void* stream) {
  int rc = check_cache(cfg);
  if (rc) return rc;
  if (n_tokens < 0) { set_error("n_tokens = %d is negative", n_tokens); return MOHGE_EINVAL; }
  if (!tok_offsets && n_tokens != cfg->n_seqs) {
    set_error("n_tokens = %d without tok_offsets: one row for each of n_seqs = %d is taken", n_tokens, cfg->n_seqs);
    return MOHGE_EINVAL; }
  if (cfg->n_seqs == 0 && n_tokens) { set_error("n_tokens = %d without a sequence", n_tokens); return MOHGE_EINVAL; }
  const int64_t width = (int64_t)cfg->n_kv_heads * cfg->head_size;
  if (n_tokens * (width / 8) >= (int64_t)1 << 31) {
    set_error("n_tokens = %d: the rows have 2^34 elements or more", n_tokens); return MOHGE_EINVAL; }
  if (n_tokens == 0) return MOHGE_OK;
  NEED(k); NEED(v); OPT(tok_offsets);
  if ((rc = check_cache_pointers(cfg, block_table, seq_lens, k_pages, v_pages, k_scale, v_scale))) return rc;
  if ((rc = check_stride(k_stride, width, "k_stride"))) return rc;
  if ((rc = check_stride(v_stride, width, "v_stride"))) return rc;
  return hip_rc(launch_cache_append(*cfg, n_tokens, k, k_stride, v, v_stride, tok_offsets, block_table, seq_lens,
                                    k_pages, v_pages, k_scale, v_scale, (hipStream_t)stream),
                "mohge_cache_append");
}

size_t mohge_cache_workspace_size(const mohge_cache_config* cfg) {
  return check_cache(cfg) ? 0 : cache_workspace_bytes(*cfg);
}

int mohge_cache_attention(const mohge_cache_config* cfg, const void* q, int64_t q_stride, const int32_t* block_table,
                          const int32_t* seq_lens, const void* k_pages, const void* v_pages, const float* k_scale,
                          const float* v_scale, float scale, void* out, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream) {
  int rc = check_cache(cfg);
  if (rc) return rc;
  if (cfg->n_seqs == 0) return MOHGE_OK;
  NEED(q); NEED(out); OPT(lse); NEED(workspace);
  if ((rc = check_cache_pointers(cfg, block_table, seq_lens, k_pages, v_pages, k_scale, v_scale))) return rc;
  if ((rc = check_stride(q_stride, (int64_t)cfg->n_heads * cfg->head_size, "q_stride"))) return rc;
  if (workspace_bytes < cache_workspace_bytes(*cfg)) {
    set_error("cache_attention workspace: %zu bytes given, %zu needed", workspace_bytes, cache_workspace_bytes(*cfg));
    return MOHGE_EWORKSPACE;
  }
  return hip_rc(launch_cache_attention(*cfg, q, q_stride, block_table, seq_lens, k_pages, v_pages, k_scale, v_scale,
                                       scale, out, lse, workspace, (hipStream_t)stream),
                "mohge_cache_attention");
}

int mohge_proj_w4(const mohge_proj_config* cfg, const void* x, const float* x_scale, const void* codes,
                  const void* scales, const void* zeros, void* y, void* stream) {
  int rc = check_proj(cfg);
  if (rc) return rc;
  if (cfg->T == 0) return MOHGE_OK;
  NEED(x); NEED(codes); NEED(scales); OPT(zeros); NEED(y);
  if (cfg->x_dtype == MOHGE_E4M3) NEED(x_scale);
  else if (x_scale) { set_error("x_scale given for rows without scales"); return MOHGE_EINVAL; }
  return hip_rc(launch_proj_w4(*cfg, x, x_scale, codes, scales, zeros, y, (hipStream_t)stream), "mohge_proj_w4");
}

}  // extern "C"
