// C ABI of libearn: argument validation on the host, then kernel launches on the caller's stream.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <atomic>
#include <exception>
#include <vector>

#include "common.h"

namespace earn {

static thread_local char g_err[512] = "";

void set_error(const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
}

RopeTable make_rope_table(float base, int head_dim) {
  // every entry point asks for the table on every call, nearly always for the same model: keep the last one per thread
  // (64 calls of pow() cost about as much host time as a kernel launch)
  static thread_local RopeTable cached;
  static thread_local float cached_base = 0.f;
  static thread_local int cached_dim = 0;
  if (base > 0.f && base == cached_base && head_dim == cached_dim) return cached;
  RopeTable t;
  memset(&t, 0, sizeof(t));
  t.enabled = base > 0.f ? 1 : 0;
  if (!t.enabled) return t;
  const double two_pi = 6.283185307179586476925286766559;
  for (int e = 0; e < head_dim / 2 && e < kMaxHalfDim; ++e) {
    double turns = pow((double)base, -2.0 * (double)e / (double)head_dim) / two_pi;
    float hi = (float)turns;
    t.hi[e] = hi;
    t.lo[e] = (float)(turns - (double)hi);
  }
  cached = t; cached_base = base; cached_dim = head_dim;
  return t;
}

int launch_compact(int n_tensors, const void* const* src, void* const* dst, const int64_t* row_bytes,
                   const int32_t* cu_seqlens, int batch, int total_tokens, int h, int t, int32_t* idx_out,
                   int32_t* pos_out, int32_t* cu_out, hipStream_t stream);
int launch_prefill(const earn_attn_desc* desc, const void* q, const void* k, const void* v, const int32_t* cu_seqlens,
                   const int32_t* positions, int batch, int total_tokens, int max_seqlen, void* out, void* k_rot_out,
                   float* lse_out, void* workspace, size_t workspace_bytes, hipStream_t stream,
                   const PrefillLayers* layers);
size_t prefill_workspace_bytes(const earn_attn_desc* desc, int total_tokens, int have_k_rot_out);
int launch_decode(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new,
                  const int32_t* q_pos, const void* shared_k, const void* shared_v, const int32_t* shared_cu,
                  const int32_t* stream_to_seq, void* gen_k, void* gen_v, const int32_t* gen_len, int gen_cap,
                  int n_streams, int batch, int max_shared_len, int shared_total, void* out, void* workspace,
                  size_t workspace_bytes, hipStream_t stream, const DecodeLayers* layers, const int32_t* gen_src);
size_t beam_topk_workspace_bytes(int batch, int beams, int vocab);
int launch_beam_topk(const float* beam_scores, const float* logp, int batch, int beams, int vocab, int32_t* parent,
                     int32_t* token, float* score, void* workspace, hipStream_t stream);
int launch_beam_reorder(const int32_t* parent, const int32_t* src_in, int32_t* src_out, int n_streams, int gen_cap, int step,
                        hipStream_t stream);
int beam_topk_limits(int beams, int vocab, const char** why);
size_t decode_workspace_bytes(int dtype, int hq, int hkv, int d, int n_streams, int batch, int max_shared_len,
                              int gen_cap, int n_layers);
int launch_decode_static(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new,
                         const int32_t* q_pos, const void* shared_k, const void* shared_v, const int32_t* shared_cu,
                         const int32_t* stream_to_seq, void* gen_k, void* gen_v, const int32_t* gen_len, int gen_cap,
                         int n_streams, int batch, int max_shared_len, int shared_total, void* out, hipStream_t stream);
int launch_step_positions(const int32_t* cu, const int32_t* stream_to_seq, int n_streams, int batch, int step,
                          int32_t* q_pos, int32_t* gen_len, hipStream_t stream);
int launch_attn_stats(const earn_attn_desc* desc, const void* q_rows, const void* k_rot, const int32_t* cu_seqlens,
                      const int32_t* row_pos, int batch, int total_tokens, int rows_per_seq, float epsilon, int t_head,
                      int tail_back, float* stats_out, hipStream_t stream);
int launch_linear(const void* x, const void* w, int rows, int k, int n, int activation, void* out, void* workspace,
                  size_t workspace_bytes, hipStream_t stream);
size_t linear_workspace_bytes(long long rows, int k, int n);
int launch_qkv_rope_project(const earn_attn_desc* desc, const void* x, const void* w_qkv, int rows, int d_model,
                            const int32_t* cu_seqlens, const int32_t* positions, int batch, void* q_out, void* k_out,
                            void* v_out, void* workspace, size_t workspace_bytes, hipStream_t stream);
size_t attn_backward_workspace_bytes(int hq, int total_tokens);
int launch_attn_backward(const earn_attn_desc* desc, const void* q, const void* k, const void* v, const void* out,
                         const float* lse, const void* d_out, const int32_t* cu_seqlens, int batch, int total_tokens,
                         int max_seqlen, void* dq, void* dk, void* dv, void* workspace, hipStream_t stream);
int launch_cache_store(const earn_attn_desc* desc, const void* k, const void* v, const int32_t* cu, const int32_t* start, int batch,
                       int total, void* k_pages, void* v_pages, const int32_t* table, int max_pages, int n_pages, int page_size,
                       hipStream_t stream);
size_t decode_paged_workspace_bytes(const earn_attn_desc* desc, int n_streams, int max_len, bool weights, int forced);
int launch_decode_paged(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new, const int32_t* q_pos,
                        void* k_pages, void* v_pages, const int32_t* table, const int32_t* cache_len, int n_streams, int max_pages,
                        int n_pages, int page_size, int max_len, const float* w_in, float* w_out, int w_cap, void* out,
                        void* workspace, int forced, hipStream_t stream);
int launch_cache_evict(const earn_attn_desc* desc, void* k_pages, void* v_pages, const int32_t* table, const int32_t* cache_len,
                       int n_streams, int max_pages, int n_pages, int page_size, int max_len, const float* w_in, int w_cap, int budget,
                       int first, int last, const int32_t* new_table, int new_pages, int32_t* kept, int32_t* len_out, float* w_out,
                       int w_out_cap, hipStream_t stream);
int launch_sample(const void* logits, int dtype, int64_t row_stride, int rows, int vocab, const float* temperature,
                  const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform, int32_t* token,
                  float* logprob, int32_t* n_kept, hipStream_t stream);
int launch_rope_keys(const earn_attn_desc* desc, const void* k, void* k_rot, const int32_t* cu_seqlens,
                     const int32_t* positions, int batch, int total_tokens, hipStream_t stream);
int launch_prefill_rows_f32(const earn_attn_desc* desc, const void* q_rows, const void* k_rot, const void* v,
                            const int32_t* cu_seqlens, const int32_t* row_pos, int batch, int total_tokens,
                            int max_seqlen, int rows_per_seq, void* out_rows, hipStream_t stream);
size_t prefill_rows_workspace_bytes(int hq, int hkv, int d, int batch, int max_seqlen, int rows_per_seq);
int launch_prefill_rows(const earn_attn_desc* desc, const void* q_rows, const void* k_rot, const void* v,
                        const int32_t* cu_seqlens, const int32_t* row_pos, int batch, int total_tokens, int max_seqlen,
                        int rows_per_seq, void* out_rows, void* workspace, size_t workspace_bytes, hipStream_t stream);

static std::atomic<int> g_tuning[kTuneCount];
int tuning(Tuning t, int dflt) {
  const int v = g_tuning[t].load(std::memory_order_relaxed);
  return v > 0 ? v : dflt;
}

int make_head_map(const earn_attn_desc* d, HeadMap* m, const char* who) {
  memset(m, 0, sizeof(*m));
  if (!d->q_to_kv) return EARN_OK;
  const int hq = d->n_q_heads, hkv = d->n_kv_heads, gq = hq / hkv;
  if (hq > kMaxMappedHeads) { set_error("%s: an explicit q_to_kv map takes at most %d query heads", who, kMaxMappedHeads); return EARN_ERR_UNSUPPORTED; }
  int count[kMaxMappedHeads] = {0};
  bool identity = true;
  for (int a = 0; a < hq; ++a) {
    const int c = d->q_to_kv[a];
    if (c < 0 || c >= hkv) { set_error("%s: q_to_kv[%d] = %d outside [0, %d)", who, a, c, hkv); return EARN_ERR_INVALID_ARG; }
    if (count[c] >= gq) {
      set_error("%s: q_to_kv gives kv head %d more than Hq/Hkv = %d query heads (groups of unequal size are not supported)", who, c, gq);
      return EARN_ERR_UNSUPPORTED;
    }
    m->q_of_slot[c * gq + count[c]++] = (unsigned char)a;
    identity = identity && c == a / gq;
  }
  m->enabled = identity ? 0 : 1;
  return EARN_OK;
}

static int check_desc(const earn_attn_desc* d, const char* who) {
  if (!d) { set_error("%s: desc is NULL", who); return EARN_ERR_INVALID_ARG; }
  if (d->dtype != EARN_F32 && d->dtype != EARN_BF16) { set_error("%s: unknown dtype %d", who, d->dtype); return EARN_ERR_UNSUPPORTED; }
  if (d->n_q_heads <= 0 || d->n_kv_heads <= 0) { set_error("%s: head counts must be positive", who); return EARN_ERR_INVALID_ARG; }
  if (d->n_q_heads % d->n_kv_heads != 0) {
    set_error("%s: n_q_heads (%d) is not a multiple of n_kv_heads (%d)", who, d->n_q_heads, d->n_kv_heads);
    return d->q_to_kv ? EARN_ERR_UNSUPPORTED : EARN_ERR_INVALID_ARG;
  }
  if (d->head_dim != 64 && d->head_dim != 128) { set_error("%s: head_dim %d not in {64,128}", who, d->head_dim); return EARN_ERR_UNSUPPORTED; }
  HeadMap m;
  return make_head_map(d, &m, who);
}

// ---- debug validation of the preconditions that live in device memory ----
static std::atomic<int> g_validate{0};

// copies n int32 from device to host on the stream and waits for it
static int fetch_i32(const int32_t* dev, size_t n, std::vector<int32_t>& host, hipStream_t stream, const char* who) {
  host.resize(n);
  if (n == 0) return EARN_OK;
  if (hipMemcpyAsync(host.data(), dev, n * sizeof(int32_t), hipMemcpyDeviceToHost, stream) != hipSuccess ||
      hipStreamSynchronize(stream) != hipSuccess) {
    set_error("%s: validation could not read a device array", who);
    return EARN_ERR_HIP;
  }
  return EARN_OK;
}
// cu[0] == 0, non-decreasing, every length <= max_len, cu[batch] == total (total < 0: not checked)
static int validate_cu(const char* who, const char* name, const std::vector<int32_t>& cu, int batch, long long total,
                       int max_len) {
  if (cu[0] != 0) { set_error("%s: %s[0] = %d, must be 0", who, name, cu[0]); return EARN_ERR_INVALID_ARG; }
  for (int s = 0; s < batch; ++s) {
    if (cu[s + 1] < cu[s]) { set_error("%s: %s decreases at %d (%d -> %d)", who, name, s, cu[s], cu[s + 1]); return EARN_ERR_INVALID_ARG; }
    if (cu[s + 1] - cu[s] > max_len) {
      set_error("%s: sequence %d has %d rows, more than the bound %d passed by value", who, s, cu[s + 1] - cu[s], max_len);
      return EARN_ERR_INVALID_ARG;
    }
  }
  if (total >= 0 && cu[batch] != total) { set_error("%s: %s[batch] = %d, expected %lld", who, name, cu[batch], total); return EARN_ERR_INVALID_ARG; }
  return EARN_OK;
}
static int validate_positions(const char* who, const char* name, const std::vector<int32_t>& p) {
  for (size_t i = 0; i < p.size(); ++i)
    if (p[i] < 0 || p[i] >= (1 << 24)) { set_error("%s: %s[%zu] = %d outside [0, 2^24)", who, name, i, p[i]); return EARN_ERR_INVALID_ARG; }
  return EARN_OK;
}

static int validate_decode(const char* who, const int32_t* q_pos, const int32_t* shared_cu, const int32_t* stream_to_seq,
                           const int32_t* gen_len, int gen_cap, int n_streams, int batch, int max_shared_len,
                           int shared_total, hipStream_t stream) {
  std::vector<int32_t> cu, qp, gl, s2s;
  int rc;
  if ((rc = fetch_i32(shared_cu, (size_t)batch + 1, cu, stream, who)) != EARN_OK) return rc;
  if ((rc = validate_cu(who, "shared_cu", cu, batch, -1, max_shared_len)) != EARN_OK) return rc;
  if (cu[batch] > shared_total) {
    set_error("%s: shared_cu[batch] = %d, more than the %d rows of the shared tensors", who, cu[batch], shared_total);
    return EARN_ERR_INVALID_ARG;
  }
  if ((rc = fetch_i32(q_pos, (size_t)n_streams, qp, stream, who)) != EARN_OK) return rc;
  if ((rc = validate_positions(who, "q_pos", qp)) != EARN_OK) return rc;
  if ((rc = fetch_i32(gen_len, (size_t)n_streams, gl, stream, who)) != EARN_OK) return rc;
  for (int u = 0; u < n_streams; ++u)
    if (gl[u] < 0 || gl[u] >= gen_cap) { set_error("%s: gen_len[%d] = %d outside [0, gen_cap = %d)", who, u, gl[u], gen_cap); return EARN_ERR_INVALID_ARG; }
  if (stream_to_seq) {
    if ((rc = fetch_i32(stream_to_seq, (size_t)n_streams, s2s, stream, who)) != EARN_OK) return rc;
    std::vector<int32_t> per_seq((size_t)batch, 0);
    for (int u = 0; u < n_streams; ++u) {
      if (s2s[u] < 0 || s2s[u] >= batch) { set_error("%s: stream_to_seq[%d] = %d outside [0, batch = %d)", who, u, s2s[u], batch); return EARN_ERR_INVALID_ARG; }
      if (++per_seq[s2s[u]] > 1024) { set_error("%s: sequence %d holds more than 1024 streams", who, s2s[u]); return EARN_ERR_INVALID_ARG; }
    }
  }
  return EARN_OK;
}

// Tables and lengths of a call over pages: rows [0, rows[u]) of every stream lie in pages of the pool.
static int validate_table(const char* who, const char* name, const std::vector<int32_t>& table, int streams, int max_pages, int n_pages,
                          int page_size, const std::vector<long long>& rows) {
  for (int u = 0; u < streams; ++u) {
    if (rows[u] > (long long)max_pages * page_size) {
      set_error("%s: stream %d has %lld rows, more than the %d pages of %s hold", who, u, rows[u], max_pages, name);
      return EARN_ERR_INVALID_ARG;
    }
    for (long long i = 0; i * page_size < rows[u]; ++i) {
      const int page = table[(size_t)u * max_pages + i];
      if (page < 0 || page >= n_pages) {
        set_error("%s: %s[%d][%lld] = %d outside [0, n_pages = %d)", who, name, u, i, page, n_pages);
        return EARN_ERR_INVALID_ARG;
      }
    }
  }
  return EARN_OK;
}
// Pages [from[u], to[u]) of every stream are written: none of them is named twice, nor among the pages [0, from[u]) of a stream
// or the pages that `taken` counts.
static int validate_written(const char* who, const char* name, const std::vector<int32_t>& table, int streams, int max_pages,
                            const std::vector<long long>& from, const std::vector<long long>& to, std::vector<int32_t>& taken) {
  for (int u = 0; u < streams; ++u)
    for (long long i = 0; i < to[u]; ++i) ++taken[table[(size_t)u * max_pages + i]];
  for (int u = 0; u < streams; ++u)
    for (long long i = from[u]; i < to[u]; ++i)
      if (taken[table[(size_t)u * max_pages + i]] > 1) {
        set_error("%s: page %d (%s[%d][%lld]) is written to and named elsewhere too", who, table[(size_t)u * max_pages + i], name, u, i);
        return EARN_ERR_INVALID_ARG;
      }
  return EARN_OK;
}
static int validate_lengths(const char* who, const std::vector<int32_t>& len, int max_len) {
  for (size_t u = 0; u < len.size(); ++u)
    if (len[u] > max_len) { set_error("%s: cache_len[%zu] = %d, more than the bound %d passed by value", who, u, len[u], max_len); return EARN_ERR_INVALID_ARG; }
  return EARN_OK;
}

static int validate_store(const char* who, const int32_t* cu_seqlens, const int32_t* start, const int32_t* page_table, int batch, int total_tokens, int max_pages,
                          int n_pages, int page_size, void* stream) {
  int rc;
  std::vector<int32_t> cu, st((size_t)batch, 0), table;
  if ((rc = fetch_i32(cu_seqlens, (size_t)batch + 1, cu, (hipStream_t)stream, who)) != EARN_OK) return rc;
  if ((rc = validate_cu(who, "cu_seqlens", cu, batch, total_tokens, 0x7fffffff)) != EARN_OK) return rc;
  if (start && (rc = fetch_i32(start, (size_t)batch, st, (hipStream_t)stream, who)) != EARN_OK) return rc;
  if ((rc = fetch_i32(page_table, (size_t)batch * max_pages, table, (hipStream_t)stream, who)) != EARN_OK) return rc;
  std::vector<long long> rows((size_t)batch), from((size_t)batch), to((size_t)batch);
  for (int s = 0; s < batch; ++s) {
    if (st[s] < 0) { set_error("%s: start[%d] = %d is negative", who, s, st[s]); return EARN_ERR_INVALID_ARG; }
    const int n = cu[s + 1] - cu[s];
    rows[s] = n > 0 ? (long long)st[s] + n : 0;
    to[s] = (rows[s] + page_size - 1) / page_size;
    from[s] = n > 0 ? st[s] / page_size : to[s];
  }
  if ((rc = validate_table(who, "page_table", table, batch, max_pages, n_pages, page_size, rows)) != EARN_OK) return rc;
  std::vector<int32_t> taken((size_t)n_pages, 0);
  if ((rc = validate_written(who, "page_table", table, batch, max_pages, from, to, taken)) != EARN_OK) return rc;
  return EARN_OK;
}
static int validate_decode_paged(const char* who, const int32_t* q_pos, const int32_t* cache_len, const int32_t* page_table, int n_streams, int max_cache_len,
                                 int max_pages, int n_pages, int page_size, void* stream) {
  int rc;
  std::vector<int32_t> qp, len, table;
  if ((rc = fetch_i32(q_pos, (size_t)n_streams, qp, (hipStream_t)stream, who)) != EARN_OK) return rc;
  if ((rc = fetch_i32(cache_len, (size_t)n_streams, len, (hipStream_t)stream, who)) != EARN_OK) return rc;
  if ((rc = validate_lengths(who, len, max_cache_len)) != EARN_OK) return rc;
  std::vector<long long> rows((size_t)n_streams), from((size_t)n_streams), to((size_t)n_streams);
  for (int u = 0; u < n_streams; ++u) {
    if (len[u] < 0) qp[u] = 0;                   // an idle stream's position is not read
    rows[u] = len[u] < 0 ? 0 : (long long)len[u] + 1;
    to[u] = (rows[u] + page_size - 1) / page_size;
    from[u] = rows[u] > 0 ? to[u] - 1 : 0;
  }
  if ((rc = validate_positions(who, "q_pos", qp)) != EARN_OK) return rc;
  if ((rc = fetch_i32(page_table, (size_t)n_streams * max_pages, table, (hipStream_t)stream, who)) != EARN_OK) return rc;
  if ((rc = validate_table(who, "page_table", table, n_streams, max_pages, n_pages, page_size, rows)) != EARN_OK) return rc;
  std::vector<int32_t> taken((size_t)n_pages, 0);
  if ((rc = validate_written(who, "page_table", table, n_streams, max_pages, from, to, taken)) != EARN_OK) return rc;
  return EARN_OK;
}
static int validate_evict(const char* who, const int32_t* cache_len, const int32_t* page_table, const int32_t* new_table, int n_streams, int max_cache_len,
                          int budget, int max_pages, int new_max_pages, int n_pages, int page_size, void* stream) {
  int rc;
  std::vector<int32_t> len, table, fresh;
  if ((rc = fetch_i32(cache_len, (size_t)n_streams, len, (hipStream_t)stream, who)) != EARN_OK) return rc;
  if ((rc = validate_lengths(who, len, max_cache_len)) != EARN_OK) return rc;
  if ((rc = fetch_i32(page_table, (size_t)n_streams * max_pages, table, (hipStream_t)stream, who)) != EARN_OK) return rc;
  if ((rc = fetch_i32(new_table, (size_t)n_streams * new_max_pages, fresh, (hipStream_t)stream, who)) != EARN_OK) return rc;
  std::vector<long long> rows((size_t)n_streams), kept((size_t)n_streams), zero((size_t)n_streams, 0), to((size_t)n_streams);
  for (int u = 0; u < n_streams; ++u) {
    rows[u] = len[u] < 0 ? 0 : len[u];
    kept[u] = rows[u] < budget ? rows[u] : budget;
    to[u] = (kept[u] + page_size - 1) / page_size;
  }
  if ((rc = validate_table(who, "page_table", table, n_streams, max_pages, n_pages, page_size, rows)) != EARN_OK) return rc;
  if ((rc = validate_table(who, "new_table", fresh, n_streams, new_max_pages, n_pages, page_size, kept)) != EARN_OK) return rc;
  std::vector<int32_t> taken((size_t)n_pages, 0);
  for (int u = 0; u < n_streams; ++u)
    for (long long i = 0; i * page_size < rows[u]; ++i) taken[table[(size_t)u * max_pages + i]] = 1;
  if ((rc = validate_written(who, "new_table", fresh, n_streams, new_max_pages, zero, to, taken)) != EARN_OK) return rc;
  return EARN_OK;
}
// A check in a host memory that may not be enough for the tables: no exception leaves a C entry.
template <typename F>
static int guarded(const char* who, F check) {
  try {
    return check();
  } catch (const std::exception&) {
    set_error("%s: validation ran out of host memory", who);
    return EARN_ERR_HIP;
  }
}

}  // namespace earn

using namespace earn;

extern "C" {

const char* earn_last_error(void) { return g_err; }

const char* earn_version(void) { return "libearn 0.2 (gfx950)"; }

int earn_set_validation(int enabled) { return g_validate.exchange(enabled ? 1 : 0); }

int earn_set_tuning(const char* key, int32_t value) {
  static const char* const names[kTuneCount] = {"prefill_block_rows", "decode_mfma_min_len", "decode_mfma_short_wgs",
                                                "decode_mfma_wgs", "decode_vec_wgs", "decode_vec_waves", "compact_blocks", "linear_tile", "linear_splits",
                                                "paged_chunk"};
  g_err[0] = 0;
  for (int i = 0; key && i < kTuneCount; ++i)
    if (strcmp(key, names[i]) == 0) { g_tuning[i].store(value > 0 ? value : 0, std::memory_order_relaxed); return EARN_OK; }
  set_error("earn_set_tuning: unknown key '%s'", key ? key : "(null)");
  return EARN_ERR_INVALID_ARG;
}

size_t earn_prefill_workspace_bytes(const earn_attn_desc* desc, int32_t batch, int32_t total_tokens,
                                    int32_t max_seqlen, int32_t have_k_rot_out) {
  (void)batch; (void)max_seqlen;
  if (check_desc(desc, "earn_prefill_workspace_bytes") != EARN_OK || total_tokens < 0) return 0;
  return prefill_workspace_bytes(desc, total_tokens, have_k_rot_out);
}

static int prefill_entry(const char* who, const earn_attn_desc* desc, const void* q, const void* k, const void* v,
                         const int32_t* cu_seqlens, const int32_t* positions, int32_t batch, int32_t total_tokens,
                         int32_t max_seqlen, void* out, void* k_rot_out, float* lse_out, void* workspace,
                         size_t workspace_bytes, void* stream, const PrefillLayers* layers) {
  g_err[0] = 0;
  int rc = check_desc(desc, who);
  if (rc != EARN_OK) return rc;
  if (batch <= 0 || total_tokens < 0 || max_seqlen <= 0) {
    set_error("%s: batch (%d) and max_seqlen (%d) must be positive, total_tokens (%d) non-negative", who, batch, max_seqlen, total_tokens);
    return EARN_ERR_INVALID_ARG;
  }
  if (!cu_seqlens) { set_error("%s: cu_seqlens is NULL", who); return EARN_ERR_INVALID_ARG; }
  if (total_tokens == 0) return EARN_OK;
  if (!q || !k || !v || !out) { set_error("%s: q, k, v and out must not be NULL", who); return EARN_ERR_INVALID_ARG; }
  if (g_validate.load(std::memory_order_relaxed)) {
    std::vector<int32_t> cu, pos;
    if ((rc = fetch_i32(cu_seqlens, (size_t)batch + 1, cu, (hipStream_t)stream, who)) != EARN_OK) return rc;
    if ((rc = validate_cu(who, "cu_seqlens", cu, batch, total_tokens, max_seqlen)) != EARN_OK) return rc;
    if (positions) {
      if ((rc = fetch_i32(positions, (size_t)total_tokens, pos, (hipStream_t)stream, who)) != EARN_OK) return rc;
      if ((rc = validate_positions(who, "positions", pos)) != EARN_OK) return rc;
    }
  }
  if (max_seqlen > total_tokens) max_seqlen = total_tokens;
  return launch_prefill(desc, q, k, v, cu_seqlens, positions, batch, total_tokens, max_seqlen, out, k_rot_out, lse_out,
                        workspace, workspace_bytes, (hipStream_t)stream, layers);
}

int earn_prefill_attn(const earn_attn_desc* desc, const void* q, const void* k, const void* v,
                      const int32_t* cu_seqlens, const int32_t* positions, int32_t batch, int32_t total_tokens,
                      int32_t max_seqlen, void* out, void* k_rot_out, float* lse_out, void* workspace,
                      size_t workspace_bytes, void* stream) {
  return prefill_entry("earn_prefill_attn", desc, q, k, v, cu_seqlens, positions, batch, total_tokens, max_seqlen, out,
                       k_rot_out, lse_out, workspace, workspace_bytes, stream, nullptr);
}

static int check_layer_stride(const char* who, const char* name, int64_t stride, int n_layers, int align = 16) {
  if (n_layers > 1 && (stride <= 0 || stride % align != 0)) {
    set_error("%s: %s = %lld must be a positive multiple of %d bytes", who, name, (long long)stride, align);
    return EARN_ERR_INVALID_ARG;
  }
  return EARN_OK;
}

int earn_prefill_attn_layers(const earn_attn_desc* desc, int32_t n_layers, const void* q, int64_t q_layer_stride,
                             const void* k, const void* v, int64_t kv_layer_stride, const int32_t* cu_seqlens,
                             const int32_t* positions, int32_t batch, int32_t total_tokens, int32_t max_seqlen,
                             void* out, int64_t out_layer_stride, void* k_rot_out, int64_t k_rot_layer_stride,
                             float* lse_out, int64_t lse_layer_stride, void* workspace, size_t workspace_bytes,
                             void* stream) {
  const char* who = "earn_prefill_attn_layers";
  g_err[0] = 0;
  if (n_layers <= 0 || n_layers > 65535) { set_error("%s: n_layers (%d) outside [1, 65535]", who, n_layers); return EARN_ERR_INVALID_ARG; }
  if (!k_rot_out) { set_error("%s: k_rot_out is required (every layer keeps its rotated keys)", who); return EARN_ERR_INVALID_ARG; }
  int rc;
  if ((rc = check_layer_stride(who, "q_layer_stride", q_layer_stride, n_layers)) != EARN_OK ||
      (rc = check_layer_stride(who, "kv_layer_stride", kv_layer_stride, n_layers)) != EARN_OK ||
      (rc = check_layer_stride(who, "out_layer_stride", out_layer_stride, n_layers)) != EARN_OK ||
      (rc = check_layer_stride(who, "k_rot_layer_stride", k_rot_layer_stride, n_layers)) != EARN_OK ||
      (lse_out && (rc = check_layer_stride(who, "lse_layer_stride", lse_layer_stride, n_layers, 4)) != EARN_OK))
    return rc;
  const PrefillLayers layers = {n_layers, q_layer_stride, kv_layer_stride, out_layer_stride, k_rot_layer_stride, lse_layer_stride};
  return prefill_entry(who, desc, q, k, v, cu_seqlens, positions, batch, total_tokens, max_seqlen, out, k_rot_out, lse_out,
                       workspace, workspace_bytes, stream, &layers);
}

int earn_compact_registers(int32_t n_tensors, const void* const* src, void* const* dst, const int64_t* row_bytes,
                           const int32_t* cu_seqlens, int32_t batch, int32_t total_tokens, int32_t n_head_reg,
                           int32_t n_tail_reg, int32_t* idx_out, int32_t* pos_out, int32_t* cu_out, void* stream) {
  g_err[0] = 0;
  if (batch <= 0 || total_tokens < 0) { set_error("earn_compact_registers: batch must be positive, total_tokens non-negative"); return EARN_ERR_INVALID_ARG; }
  if (n_head_reg < 0 || n_tail_reg < 0 || n_head_reg + n_tail_reg == 0) {
    set_error("earn_compact_registers: register counts must be non-negative and not both zero (h=%d, t=%d)", n_head_reg, n_tail_reg);
    return EARN_ERR_INVALID_ARG;
  }
  if (n_tensors < 0 || n_tensors > EARN_MAX_COMPACT_TENSORS) {
    set_error("earn_compact_registers: n_tensors %d outside [0, %d]", n_tensors, EARN_MAX_COMPACT_TENSORS);
    return EARN_ERR_INVALID_ARG;
  }
  if (!cu_seqlens) { set_error("earn_compact_registers: cu_seqlens is NULL"); return EARN_ERR_INVALID_ARG; }
  if ((long long)batch * (n_head_reg + n_tail_reg) > 0x7fffffffLL) { set_error("earn_compact_registers: too many rows"); return EARN_ERR_INVALID_ARG; }
  if (n_tensors > 0 && (!src || !dst || !row_bytes)) { set_error("earn_compact_registers: src, dst and row_bytes must not be NULL"); return EARN_ERR_INVALID_ARG; }
  for (int i = 0; i < n_tensors; ++i) {
    if (!src[i] || !dst[i]) { set_error("earn_compact_registers: tensor %d has a NULL pointer", i); return EARN_ERR_INVALID_ARG; }
    if (((uintptr_t)src[i] | (uintptr_t)dst[i]) & 15) { set_error("earn_compact_registers: tensor %d is not 16-byte aligned", i); return EARN_ERR_INVALID_ARG; }
    if (row_bytes[i] <= 0 || row_bytes[i] % 16 != 0 || row_bytes[i] / 16 > 0x7fffffffLL) {
      set_error("earn_compact_registers: row_bytes[%d] = %lld is not a positive multiple of 16", i, (long long)row_bytes[i]);
      return EARN_ERR_INVALID_ARG;
    }
  }
  if (g_validate.load(std::memory_order_relaxed)) {
    const char* who = "earn_compact_registers";
    std::vector<int32_t> cu;
    int rc = fetch_i32(cu_seqlens, (size_t)batch + 1, cu, (hipStream_t)stream, who);
    if (rc != EARN_OK) return rc;
    if ((rc = validate_cu(who, "cu_seqlens", cu, batch, -1, 0x7fffffff)) != EARN_OK) return rc;
    for (int s = 0; s < batch; ++s)
      if (cu[s + 1] - cu[s] < n_head_reg + n_tail_reg) {
        set_error("%s: sequence %d has %d rows, fewer than h + t = %d", who, s, cu[s + 1] - cu[s], n_head_reg + n_tail_reg);
        return EARN_ERR_INVALID_ARG;
      }
  }
  return launch_compact(n_tensors, src, dst, row_bytes, cu_seqlens, batch, total_tokens, n_head_reg, n_tail_reg, idx_out,
                        pos_out, cu_out, (hipStream_t)stream);
}

int earn_decode_step_positions(const int32_t* cu_seqlens, const int32_t* stream_to_seq, int32_t n_streams,
                               int32_t batch, int32_t step, int32_t* q_pos, int32_t* gen_len, void* stream) {
  g_err[0] = 0;
  if (!cu_seqlens || n_streams <= 0 || batch <= 0 || step < 0) {
    set_error("earn_decode_step_positions: cu_seqlens must not be NULL, n_streams (%d) and batch (%d) positive, step (%d) non-negative", n_streams, batch, step);
    return EARN_ERR_INVALID_ARG;
  }
  if (!stream_to_seq && n_streams != batch) {
    set_error("earn_decode_step_positions: stream_to_seq is NULL but n_streams (%d) != batch (%d)", n_streams, batch);
    return EARN_ERR_INVALID_ARG;
  }
  if (!q_pos && !gen_len) return EARN_OK;
  return launch_step_positions(cu_seqlens, stream_to_seq, n_streams, batch, step, q_pos, gen_len, (hipStream_t)stream);
}

size_t earn_decode_workspace_bytes(const earn_attn_desc* desc, int32_t n_streams, int32_t batch,
                                   int32_t max_shared_len, int32_t gen_cap) {
  if (check_desc(desc, "earn_decode_workspace_bytes") != EARN_OK || n_streams <= 0 || batch <= 0 || max_shared_len < 0 || gen_cap <= 0) return 0;
  return decode_workspace_bytes(desc->dtype, desc->n_q_heads, desc->n_kv_heads, desc->head_dim, n_streams, batch,
                                max_shared_len, gen_cap, 1);
}

// the host-side checks earn_decode_attn and earn_decode_attn_static share
static int check_decode_args(const char* who, const earn_attn_desc* desc, const void* q, const void* k_new,
                             const void* v_new, const int32_t* q_pos, const void* shared_k, const void* shared_v,
                             const int32_t* shared_cu, const int32_t* stream_to_seq, void* gen_k, void* gen_v,
                             const int32_t* gen_len, int32_t gen_cap, int32_t n_streams, int32_t batch,
                             int32_t max_shared_len, int32_t shared_total, void* out, void* stream) {
  g_err[0] = 0;
  int rc = check_desc(desc, who);
  if (rc != EARN_OK) return rc;
  if (n_streams <= 0 || batch <= 0 || gen_cap <= 0 || max_shared_len < 0 || shared_total < 0) {
    set_error("%s: n_streams (%d), batch (%d), gen_cap (%d) must be positive, max_shared_len (%d) and shared_total (%d) non-negative",
              who, n_streams, batch, gen_cap, max_shared_len, shared_total);
    return EARN_ERR_INVALID_ARG;
  }
  if (!q || !k_new || !v_new || !q_pos || !shared_cu || !gen_k || !gen_v || !gen_len || !out) {
    set_error("%s: a required pointer is NULL", who);
    return EARN_ERR_INVALID_ARG;
  }
  if (max_shared_len > 0 && (!shared_k || !shared_v)) { set_error("%s: shared_k/shared_v are NULL but max_shared_len > 0", who); return EARN_ERR_INVALID_ARG; }
  if (!stream_to_seq && n_streams != batch) { set_error("%s: stream_to_seq is NULL but n_streams (%d) != batch (%d)", who, n_streams, batch); return EARN_ERR_INVALID_ARG; }
  if (g_validate.load(std::memory_order_relaxed) &&
      (rc = validate_decode(who, q_pos, shared_cu, stream_to_seq, gen_len, gen_cap, n_streams, batch, max_shared_len,
                            shared_total, (hipStream_t)stream)) != EARN_OK)
    return rc;
  return EARN_OK;
}

int earn_decode_attn_static(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new,
                            const int32_t* q_pos, const void* shared_k, const void* shared_v,
                            const int32_t* shared_cu, const int32_t* stream_to_seq, void* gen_k, void* gen_v,
                            const int32_t* gen_len, int32_t gen_cap, int32_t n_streams, int32_t batch,
                            int32_t max_shared_len, int32_t shared_total, void* out, void* stream) {
  const int rc = check_decode_args("earn_decode_attn_static", desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu,
                                   stream_to_seq, gen_k, gen_v, gen_len, gen_cap, n_streams, batch, max_shared_len, shared_total, out,
                                   stream);
  if (rc != EARN_OK) return rc;
  return launch_decode_static(desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu, stream_to_seq, gen_k, gen_v,
                              gen_len, gen_cap, n_streams, batch, max_shared_len, shared_total, out, (hipStream_t)stream);
}

int earn_decode_attn(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new,
                     const int32_t* q_pos, const void* shared_k, const void* shared_v, const int32_t* shared_cu,
                     const int32_t* stream_to_seq, void* gen_k, void* gen_v, const int32_t* gen_len, int32_t gen_cap,
                     int32_t n_streams, int32_t batch, int32_t max_shared_len, int32_t shared_total, void* out, void* workspace,
                     size_t workspace_bytes, void* stream) {
  const int rc = check_decode_args("earn_decode_attn", desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu,
                                   stream_to_seq, gen_k, gen_v, gen_len, gen_cap, n_streams, batch, max_shared_len, shared_total, out,
                                   stream);
  if (rc != EARN_OK) return rc;
  return launch_decode(desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu, stream_to_seq, gen_k, gen_v, gen_len,
                       gen_cap, n_streams, batch, max_shared_len, shared_total, out, workspace, workspace_bytes, (hipStream_t)stream,
                       nullptr, nullptr);
}

int earn_decode_attn_beams(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new,
                           const int32_t* q_pos, const void* shared_k, const void* shared_v, const int32_t* shared_cu,
                           const int32_t* stream_to_seq, void* gen_k, void* gen_v, const int32_t* gen_len,
                           const int32_t* gen_src, int32_t gen_cap, int32_t n_streams, int32_t batch,
                           int32_t max_shared_len, int32_t shared_total, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_decode_args("earn_decode_attn_beams", desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu,
                                   stream_to_seq, gen_k, gen_v, gen_len, gen_cap, n_streams, batch, max_shared_len, shared_total, out,
                                   stream);
  if (rc != EARN_OK) return rc;
  if (gen_src && g_validate.load(std::memory_order_relaxed)) {
    std::vector<int32_t> src;
    int rc2 = fetch_i32(gen_src, (size_t)n_streams * gen_cap, src, (hipStream_t)stream, "earn_decode_attn_beams");
    if (rc2 != EARN_OK) return rc2;
    for (size_t i = 0; i < src.size(); ++i)
      if (src[i] < 0 || src[i] >= n_streams) {
        set_error("earn_decode_attn_beams: gen_src[%zu] = %d outside [0, n_streams = %d)", i, src[i], n_streams);
        return EARN_ERR_INVALID_ARG;
      }
  }
  return launch_decode(desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu, stream_to_seq, gen_k, gen_v, gen_len,
                       gen_cap, n_streams, batch, max_shared_len, shared_total, out, workspace, workspace_bytes, (hipStream_t)stream,
                       nullptr, gen_src);
}

size_t earn_beam_topk_workspace_bytes(int32_t batch, int32_t beams, int32_t vocab) {
  const char* why;
  if (batch <= 0 || beams <= 0 || vocab <= 0 || !beam_topk_limits(beams, vocab, &why)) return 0;
  return beam_topk_workspace_bytes(batch, beams, vocab);
}

int earn_beam_topk(const float* beam_scores, const float* token_logprobs, int32_t batch, int32_t beams, int32_t vocab,
                   int32_t* parent_out, int32_t* token_out, float* score_out, void* workspace, size_t workspace_bytes,
                   void* stream) {
  g_err[0] = 0;
  if (!token_logprobs || !parent_out || !token_out || !score_out || batch <= 0 || beams <= 0 || vocab <= 0 || batch > 65535) {
    set_error("earn_beam_topk: NULL pointer or non-positive size (batch %d, beams %d, vocab %d)", batch, beams, vocab);
    return EARN_ERR_INVALID_ARG;
  }
  const char* why = "";
  if (!beam_topk_limits(beams, vocab, &why)) { set_error("earn_beam_topk: %s", why); return EARN_ERR_UNSUPPORTED; }
  const size_t need = beam_topk_workspace_bytes(batch, beams, vocab);
  if (need > workspace_bytes || (need > 0 && !workspace)) {
    set_error("earn_beam_topk: workspace too small (%zu bytes given, %zu needed)", workspace_bytes, need);
    return EARN_ERR_WORKSPACE_TOO_SMALL;
  }
  return launch_beam_topk(beam_scores, token_logprobs, batch, beams, vocab, parent_out, token_out, score_out, workspace,
                          (hipStream_t)stream);
}

int earn_beam_reorder(const int32_t* parent, const int32_t* gen_src_in, int32_t* gen_src_out, int32_t n_streams,
                      int32_t gen_cap, int32_t step, void* stream) {
  g_err[0] = 0;
  if (!parent || !gen_src_out || gen_src_out == gen_src_in || n_streams <= 0 || gen_cap <= 0 || step < 0 || step >= gen_cap) {
    set_error("earn_beam_reorder: NULL or aliased table, or sizes out of range (n_streams %d, gen_cap %d, step %d)", n_streams, gen_cap, step);
    return EARN_ERR_INVALID_ARG;
  }
  return launch_beam_reorder(parent, gen_src_in, gen_src_out, n_streams, gen_cap, step, (hipStream_t)stream);
}

size_t earn_decode_layers_workspace_bytes(const earn_attn_desc* desc, int32_t n_layers, int32_t n_streams, int32_t batch,
                                          int32_t max_shared_len, int32_t gen_cap) {
  if (check_desc(desc, "earn_decode_layers_workspace_bytes") != EARN_OK || n_layers <= 0 || n_layers > 65535 ||
      n_streams <= 0 || batch <= 0 || max_shared_len < 0 || gen_cap <= 0)
    return 0;
  return decode_workspace_bytes(desc->dtype, desc->n_q_heads, desc->n_kv_heads, desc->head_dim, n_streams, batch,
                                max_shared_len, gen_cap, n_layers);
}

int earn_decode_attn_layers(const earn_attn_desc* desc, int32_t n_layers, const void* q, int64_t q_layer_stride,
                            const void* k_new, const void* v_new, int64_t kv_new_layer_stride, const int32_t* q_pos,
                            const void* shared_k, const void* shared_v, int64_t shared_layer_stride,
                            const int32_t* shared_cu, const int32_t* stream_to_seq, void* gen_k, void* gen_v,
                            int64_t gen_layer_stride, const int32_t* gen_len, int32_t gen_cap, int32_t n_streams,
                            int32_t batch, int32_t max_shared_len, int32_t shared_total, void* out, int64_t out_layer_stride, void* workspace,
                            size_t workspace_bytes, void* stream) {
  const char* who = "earn_decode_attn_layers";
  int rc = check_decode_args(who, desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu, stream_to_seq, gen_k,
                             gen_v, gen_len, gen_cap, n_streams, batch, max_shared_len, shared_total, out, stream);
  if (rc != EARN_OK) return rc;
  if (n_layers <= 0 || n_layers > 65535) { set_error("%s: n_layers (%d) outside [1, 65535]", who, n_layers); return EARN_ERR_INVALID_ARG; }
  if ((rc = check_layer_stride(who, "q_layer_stride", q_layer_stride, n_layers)) != EARN_OK ||
      (rc = check_layer_stride(who, "kv_new_layer_stride", kv_new_layer_stride, n_layers)) != EARN_OK ||
      (max_shared_len > 0 && (rc = check_layer_stride(who, "shared_layer_stride", shared_layer_stride, n_layers)) != EARN_OK) ||
      (rc = check_layer_stride(who, "gen_layer_stride", gen_layer_stride, n_layers)) != EARN_OK ||
      (rc = check_layer_stride(who, "out_layer_stride", out_layer_stride, n_layers)) != EARN_OK)
    return rc;
  const DecodeLayers layers = {n_layers, q_layer_stride, kv_new_layer_stride, shared_layer_stride, gen_layer_stride, out_layer_stride};
  return launch_decode(desc, q, k_new, v_new, q_pos, shared_k, shared_v, shared_cu, stream_to_seq, gen_k, gen_v, gen_len,
                       gen_cap, n_streams, batch, max_shared_len, shared_total, out, workspace, workspace_bytes, (hipStream_t)stream,
                       &layers, nullptr);
}

size_t earn_prefill_register_rows_workspace_bytes(const earn_attn_desc* desc, int32_t batch, int32_t max_seqlen,
                                                  int32_t rows_per_seq) {
  if (check_desc(desc, "earn_prefill_register_rows_workspace_bytes") != EARN_OK || batch <= 0 || max_seqlen < 0 ||
      rows_per_seq <= 0)
    return 0;
  if (desc->dtype == EARN_F32) return 0;
  return prefill_rows_workspace_bytes(desc->n_q_heads, desc->n_kv_heads, desc->head_dim, batch, max_seqlen, rows_per_seq);
}

int earn_prefill_register_rows(const earn_attn_desc* desc, const void* q_rows, const void* k, const void* v,
                               const int32_t* cu_seqlens, const int32_t* row_pos, int32_t batch, int32_t total_tokens,
                               int32_t max_seqlen, int32_t rows_per_seq, void* out_rows, void* k_rot_out,
                               void* workspace, size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  int rc = check_desc(desc, "earn_prefill_register_rows");
  if (rc != EARN_OK) return rc;
  if (batch <= 0 || total_tokens <= 0 || max_seqlen <= 0 || rows_per_seq <= 0) {
    set_error("earn_prefill_register_rows: batch (%d), total_tokens (%d), max_seqlen (%d) and rows_per_seq (%d) must be positive", batch, total_tokens, max_seqlen, rows_per_seq);
    return EARN_ERR_INVALID_ARG;
  }
  if (rows_per_seq > max_seqlen) {
    set_error("earn_prefill_register_rows: rows_per_seq (%d) exceeds max_seqlen (%d)", rows_per_seq, max_seqlen);
    return EARN_ERR_INVALID_ARG;
  }
  if (!q_rows || !k || !v || !cu_seqlens || !row_pos || !out_rows || !k_rot_out) {
    set_error("earn_prefill_register_rows: a required pointer is NULL");
    return EARN_ERR_INVALID_ARG;
  }
  if (g_validate.load(std::memory_order_relaxed)) {
    const char* who = "earn_prefill_register_rows";
    std::vector<int32_t> cu, rp;
    if ((rc = fetch_i32(cu_seqlens, (size_t)batch + 1, cu, (hipStream_t)stream, who)) != EARN_OK) return rc;
    if ((rc = validate_cu(who, "cu_seqlens", cu, batch, total_tokens, max_seqlen)) != EARN_OK) return rc;
    if ((rc = fetch_i32(row_pos, (size_t)batch * rows_per_seq, rp, (hipStream_t)stream, who)) != EARN_OK) return rc;
    for (int s = 0; s < batch; ++s)
      for (int m = 0; m < rows_per_seq; ++m) {
        const int p = rp[(size_t)s * rows_per_seq + m], n = cu[s + 1] - cu[s];
        if (p < 0 || p >= n || (m > 0 && p <= rp[(size_t)s * rows_per_seq + m - 1])) {
          set_error("%s: row_pos[%d] = %d (row %d of sequence %d, %d tokens) is outside the sequence or not ascending", who, s * rows_per_seq + m, p, m, s, n);
          return EARN_ERR_INVALID_ARG;
        }
      }
  }
  if (desc->dtype == EARN_F32) {
    rc = launch_rope_keys(desc, k, k_rot_out, cu_seqlens, nullptr, batch, total_tokens, (hipStream_t)stream);
    if (rc != EARN_OK) return rc;
    return launch_prefill_rows_f32(desc, q_rows, k_rot_out, v, cu_seqlens, row_pos, batch, total_tokens, max_seqlen,
                                   rows_per_seq, out_rows, (hipStream_t)stream);
  }
  const size_t need = prefill_rows_workspace_bytes(desc->n_q_heads, desc->n_kv_heads, desc->head_dim, batch, max_seqlen, rows_per_seq);
  if (need > workspace_bytes || (need > 0 && !workspace)) {
    set_error("earn_prefill_register_rows: workspace too small (%zu bytes given, %zu needed)", workspace_bytes, need);
    return EARN_ERR_WORKSPACE_TOO_SMALL;
  }
  rc = launch_rope_keys(desc, k, k_rot_out, cu_seqlens, nullptr, batch, total_tokens, (hipStream_t)stream);
  if (rc != EARN_OK) return rc;
  return launch_prefill_rows(desc, q_rows, k_rot_out, v, cu_seqlens, row_pos, batch, total_tokens, max_seqlen, rows_per_seq,
                             out_rows, workspace, workspace_bytes, (hipStream_t)stream);
}

int earn_attn_stats(const earn_attn_desc* desc, const void* q_rows, const void* k_rot, const int32_t* cu_seqlens,
                    const int32_t* row_pos, int32_t batch, int32_t total_tokens, int32_t rows_per_seq, float epsilon,
                    int32_t t_head, int32_t tail_back, float* stats_out, void* stream) {
  g_err[0] = 0;
  int rc = check_desc(desc, "earn_attn_stats");
  if (rc != EARN_OK) return rc;
  if (batch <= 0 || total_tokens < 0 || rows_per_seq <= 0 || !(epsilon >= 0.f) || t_head < 0 || tail_back < 0 ||
      (long long)batch * rows_per_seq > 0x7fffffffLL || desc->n_q_heads > 65535) {
    set_error("earn_attn_stats: batch (%d) and rows_per_seq (%d) must be positive, epsilon, t_head (%d) and tail_back (%d) non-negative", batch, rows_per_seq, t_head, tail_back);
    return EARN_ERR_INVALID_ARG;
  }
  if (!q_rows || !k_rot || !cu_seqlens || !row_pos || !stats_out) {
    set_error("earn_attn_stats: a required pointer is NULL");
    return EARN_ERR_INVALID_ARG;
  }
  return launch_attn_stats(desc, q_rows, k_rot, cu_seqlens, row_pos, batch, total_tokens, rows_per_seq, epsilon, t_head,
                           tail_back, stats_out, (hipStream_t)stream);
}

int earn_qkv_rope_project(const earn_attn_desc* desc, const void* x, const void* w_qkv, int32_t rows, int32_t d_model,
                          const int32_t* cu_seqlens, const int32_t* positions, int32_t batch, void* q_out, void* k_out,
                          void* v_out, void* workspace, size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  int rc = check_desc(desc, "earn_qkv_rope_project");
  if (rc != EARN_OK) return rc;
  if (desc->dtype != EARN_BF16) { set_error("earn_qkv_rope_project: bf16 only"); return EARN_ERR_UNSUPPORTED; }
  if (!x || !w_qkv || !q_out || !k_out || !v_out || rows <= 0 || d_model <= 0) {
    set_error("earn_qkv_rope_project: NULL pointer or non-positive size (rows %d, d_model %d)", rows, d_model);
    return EARN_ERR_INVALID_ARG;
  }
  if (desc->rope_base > 0.f && !positions && (!cu_seqlens || batch <= 0)) {
    set_error("earn_qkv_rope_project: positions is NULL and no cu_seqlens / batch to derive them from");
    return EARN_ERR_INVALID_ARG;
  }
  return launch_qkv_rope_project(desc, x, w_qkv, rows, d_model, cu_seqlens, positions, batch, q_out, k_out, v_out,
                                 workspace, workspace_bytes, (hipStream_t)stream);
}

size_t earn_linear_workspace_bytes(int32_t rows, int32_t k, int32_t n) { return linear_workspace_bytes(rows, k, n); }

int earn_linear(const void* x, const void* w, int32_t rows, int32_t k, int32_t n, int32_t activation, void* out,
                void* workspace, size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  if (!x || !w || !out || rows <= 0 || k <= 0 || n <= 0 || activation < 0 || activation > 1) {
    set_error("earn_linear: NULL pointer, non-positive size or unknown activation %d", activation);
    return EARN_ERR_INVALID_ARG;
  }
  return launch_linear(x, w, rows, k, n, activation, out, workspace, workspace_bytes, (hipStream_t)stream);
}

size_t earn_attn_backward_workspace_bytes(const earn_attn_desc* desc, int32_t total_tokens) {
  if (check_desc(desc, "earn_attn_backward_workspace_bytes") != EARN_OK || total_tokens <= 0) return 0;
  return attn_backward_workspace_bytes(desc->n_q_heads, total_tokens);
}

int earn_attn_backward(const earn_attn_desc* desc, const void* q, const void* k, const void* v, const void* out,
                       const float* lse, const void* d_out, const int32_t* cu_seqlens, int32_t batch,
                       int32_t total_tokens, int32_t max_seqlen, void* dq, void* dk, void* dv, void* workspace,
                       size_t workspace_bytes, void* stream) {
  g_err[0] = 0;
  int rc = check_desc(desc, "earn_attn_backward");
  if (rc != EARN_OK) return rc;
  if (desc->rope_base > 0.f) {
    set_error("earn_attn_backward: takes rotated q and k and rotates nothing: set rope_base <= 0");
    return EARN_ERR_UNSUPPORTED;
  }
  if (!q || !k || !v || !out || !lse || !d_out || !cu_seqlens || !dq || !dk || !dv || batch <= 0 || total_tokens <= 0 ||
      max_seqlen <= 0) {
    set_error("earn_attn_backward: NULL pointer or non-positive size (batch %d, total_tokens %d, max_seqlen %d)", batch, total_tokens, max_seqlen);
    return EARN_ERR_INVALID_ARG;
  }
  const size_t need = attn_backward_workspace_bytes(desc->n_q_heads, total_tokens);
  if (need > workspace_bytes || !workspace) {
    set_error("earn_attn_backward: workspace too small (%zu bytes given, %zu needed)", workspace_bytes, need);
    return EARN_ERR_WORKSPACE_TOO_SMALL;
  }
  if (g_validate.load(std::memory_order_relaxed)) {
    std::vector<int32_t> cu;
    if ((rc = fetch_i32(cu_seqlens, (size_t)batch + 1, cu, (hipStream_t)stream, "earn_attn_backward")) != EARN_OK) return rc;
    if ((rc = validate_cu("earn_attn_backward", "cu_seqlens", cu, batch, total_tokens, max_seqlen)) != EARN_OK) return rc;
  }
  if (max_seqlen > total_tokens) max_seqlen = total_tokens;
  return launch_attn_backward(desc, q, k, v, out, lse, d_out, cu_seqlens, batch, total_tokens, max_seqlen, dq, dk, dv,
                              workspace, (hipStream_t)stream);
}

static int check_pages(const char* who, const void* k_pages, const void* v_pages, const int32_t* table, int32_t max_pages,
                       int32_t n_pages, int32_t page_size) {
  if (!k_pages || !v_pages || !table) { set_error("%s: k_pages, v_pages and page_table must not be NULL", who); return EARN_ERR_INVALID_ARG; }
  if (((uintptr_t)k_pages | (uintptr_t)v_pages) & 15) { set_error("%s: k_pages and v_pages must be 16-byte aligned", who); return EARN_ERR_INVALID_ARG; }
  if (max_pages <= 0 || n_pages <= 0 || page_size <= 0) {
    set_error("%s: max_pages (%d), n_pages (%d) and page_size (%d) must be positive", who, max_pages, n_pages, page_size);
    return EARN_ERR_INVALID_ARG;
  }
  return EARN_OK;
}
static int check_workspace(const char* who, size_t need, const void* workspace, size_t bytes) {
  if (need > bytes || (need > 0 && !workspace)) {
    set_error("%s: workspace too small (%zu bytes given, %zu needed)", who, bytes, need);
    return EARN_ERR_WORKSPACE_TOO_SMALL;
  }
  if (need > 0 && ((uintptr_t)workspace & 255)) { set_error("%s: the workspace must be 256-byte aligned", who); return EARN_ERR_INVALID_ARG; }
  return EARN_OK;
}

static bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  return (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

int earn_cache_store(const earn_attn_desc* desc, const void* k, const void* v, const int32_t* cu_seqlens, const int32_t* start,
                     int32_t batch, int32_t total_tokens, void* k_pages, void* v_pages, const int32_t* page_table,
                     int32_t max_pages, int32_t n_pages, int32_t page_size, void* stream) {
  const char* who = "earn_cache_store";
  g_err[0] = 0;
  int rc = check_desc(desc, who);
  if (rc != EARN_OK) return rc;
  if (batch <= 0 || total_tokens < 0) { set_error("%s: batch (%d) must be positive, total_tokens (%d) non-negative", who, batch, total_tokens); return EARN_ERR_INVALID_ARG; }
  if ((rc = check_pages(who, k_pages, v_pages, page_table, max_pages, n_pages, page_size)) != EARN_OK) return rc;
  if (!cu_seqlens) { set_error("%s: cu_seqlens is NULL", who); return EARN_ERR_INVALID_ARG; }
  if (total_tokens == 0) return EARN_OK;
  if (!k || !v) { set_error("%s: k and v must not be NULL", who); return EARN_ERR_INVALID_ARG; }
  if (((uintptr_t)k | (uintptr_t)v) & 15) { set_error("%s: k and v must be 16-byte aligned", who); return EARN_ERR_INVALID_ARG; }
  if (g_validate.load(std::memory_order_relaxed) && (rc = guarded(who, [&] { return validate_store(who, cu_seqlens, start, page_table, batch, total_tokens, max_pages, n_pages, page_size, stream); })) != EARN_OK) return rc;
  return launch_cache_store(desc, k, v, cu_seqlens, start, batch, total_tokens, k_pages, v_pages, page_table, max_pages, n_pages,
                            page_size, (hipStream_t)stream);
}

// what the kernels over pages take beyond the description's own checks; sizes of the grid
static int check_paged_desc(const earn_attn_desc* d, int32_t n_streams, const char* who) {
  const int rc = check_desc(d, who);
  if (rc != EARN_OK) return rc;
  if (d->n_q_heads / d->n_kv_heads > 128) { set_error("%s: more than 128 query heads per kv head", who); return EARN_ERR_UNSUPPORTED; }
  if (n_streams > 65535 || d->n_q_heads > 65535) { set_error("%s: more than 65535 streams or heads", who); return EARN_ERR_UNSUPPORTED; }
  return EARN_OK;
}

size_t earn_decode_paged_workspace_bytes(const earn_attn_desc* desc, int32_t n_streams, int32_t max_cache_len,
                                         int32_t have_weights) {
  if (check_paged_desc(desc, n_streams, "earn_decode_paged_workspace_bytes") != EARN_OK || n_streams <= 0 || max_cache_len < 0 ||
      max_cache_len > EARN_MAX_CACHE_LEN)
    return 0;
  return decode_paged_workspace_bytes(desc, n_streams, max_cache_len, have_weights != 0, tuning(kTunePagedChunk, 0));
}

int earn_decode_attn_paged(const earn_attn_desc* desc, const void* q, const void* k_new, const void* v_new,
                           const int32_t* q_pos, void* k_pages, void* v_pages, const int32_t* page_table,
                           const int32_t* cache_len, int32_t n_streams, int32_t max_pages, int32_t n_pages,
                           int32_t page_size, int32_t max_cache_len, const float* weights_in, float* weights_out,
                           int32_t weight_rows, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "earn_decode_attn_paged";
  g_err[0] = 0;
  int rc = check_paged_desc(desc, n_streams, who);
  if (rc != EARN_OK) return rc;
  if (n_streams <= 0 || max_cache_len < 0 || max_cache_len > EARN_MAX_CACHE_LEN) {
    set_error("%s: n_streams (%d) must be positive, max_cache_len (%d) in [0, %d]", who, n_streams, max_cache_len, EARN_MAX_CACHE_LEN);
    return EARN_ERR_INVALID_ARG;
  }
  if ((rc = check_pages(who, k_pages, v_pages, page_table, max_pages, n_pages, page_size)) != EARN_OK) return rc;
  if (!q || !k_new || !v_new || !q_pos || !cache_len || !out) { set_error("%s: a required pointer is NULL", who); return EARN_ERR_INVALID_ARG; }
  if (((uintptr_t)q | (uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)out) & 15) { set_error("%s: q, k_new, v_new and out must be 16-byte aligned", who); return EARN_ERR_INVALID_ARG; }
  if (weights_in && !weights_out) { set_error("%s: weights_in without weights_out", who); return EARN_ERR_INVALID_ARG; }
  if (weights_out && weight_rows <= 0) { set_error("%s: weight_rows (%d) must be positive", who, weight_rows); return EARN_ERR_INVALID_ARG; }
  const size_t w_bytes = weights_out ? (size_t)n_streams * desc->n_kv_heads * weight_rows * sizeof(float) : 0;
  if (weights_in && weights_in != weights_out && overlap(weights_in, w_bytes, weights_out, w_bytes)) {
    set_error("%s: weights_in and weights_out overlap without being the same", who);
    return EARN_ERR_INVALID_ARG;
  }
  const int forced = tuning(kTunePagedChunk, 0);   // read once: the size checked is that of the launch, whoever sets it meanwhile
  const size_t need = decode_paged_workspace_bytes(desc, n_streams, max_cache_len, weights_out != nullptr, forced);
  if ((rc = check_workspace(who, need, workspace, workspace_bytes)) != EARN_OK) return rc;
  if (g_validate.load(std::memory_order_relaxed) && (rc = guarded(who, [&] { return validate_decode_paged(who, q_pos, cache_len, page_table, n_streams, max_cache_len, max_pages, n_pages, page_size, stream); })) != EARN_OK) return rc;
  return launch_decode_paged(desc, q, k_new, v_new, q_pos, k_pages, v_pages, page_table, cache_len, n_streams, max_pages, n_pages,
                             page_size, max_cache_len, weights_in, weights_out, weight_rows, out, workspace, forced, (hipStream_t)stream);
}

size_t earn_cache_evict_workspace_bytes(const earn_attn_desc* desc, int32_t n_streams, int32_t max_cache_len, int32_t budget) {
  (void)desc; (void)n_streams; (void)max_cache_len; (void)budget;
  return 0;
}

int earn_cache_evict(const earn_attn_desc* desc, void* k_pages, void* v_pages, const int32_t* page_table,
                     const int32_t* cache_len, int32_t n_streams, int32_t max_pages, int32_t n_pages, int32_t page_size,
                     int32_t max_cache_len, const float* weights, int32_t weight_rows, int32_t budget, int32_t n_first,
                     int32_t n_last, const int32_t* new_table, int32_t new_max_pages, int32_t* kept_out, int32_t* len_out,
                     float* weights_out, int32_t weight_rows_out, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "earn_cache_evict";
  g_err[0] = 0;
  int rc = check_paged_desc(desc, n_streams, who);
  if (rc != EARN_OK) return rc;
  if (n_streams <= 0 || max_cache_len < 0 || max_cache_len > EARN_MAX_CACHE_LEN || budget <= 0 || budget > EARN_MAX_CACHE_LEN ||
      weight_rows <= 0) {
    set_error("%s: n_streams (%d), budget (%d) and weight_rows (%d) must be positive, max_cache_len (%d) and budget at most %d", who, n_streams, budget, weight_rows, max_cache_len, EARN_MAX_CACHE_LEN);
    return EARN_ERR_INVALID_ARG;
  }
  if (n_first < 0 || n_last < 0 || (long long)n_first + n_last > budget) {
    set_error("%s: n_first (%d) and n_last (%d) must be non-negative and together at most budget (%d)", who, n_first, n_last, budget);
    return EARN_ERR_INVALID_ARG;
  }
  if ((rc = check_pages(who, k_pages, v_pages, page_table, max_pages, n_pages, page_size)) != EARN_OK) return rc;
  if (!cache_len || !weights || !new_table || !kept_out || !len_out) { set_error("%s: a required pointer is NULL", who); return EARN_ERR_INVALID_ARG; }
  if (max_cache_len > weight_rows) { set_error("%s: max_cache_len (%d) exceeds weight_rows (%d)", who, max_cache_len, weight_rows); return EARN_ERR_INVALID_ARG; }
  if (new_max_pages <= 0 || (long long)new_max_pages * page_size < budget) {
    set_error("%s: %d new pages of %d rows do not hold budget = %d rows", who, new_max_pages, page_size, budget);
    return EARN_ERR_INVALID_ARG;
  }
  if (weights_out && weight_rows_out < budget) { set_error("%s: weight_rows_out (%d) is less than budget (%d)", who, weight_rows_out, budget); return EARN_ERR_INVALID_ARG; }
  const size_t w_row = (size_t)n_streams * desc->n_kv_heads * sizeof(float);
  if (weights_out && overlap(weights, w_row * weight_rows, weights_out, w_row * weight_rows_out)) {   // a sum would be overwritten before it is moved
    set_error("%s: weights_out overlaps weights", who);
    return EARN_ERR_INVALID_ARG;
  }
  if ((rc = check_workspace(who, earn_cache_evict_workspace_bytes(desc, n_streams, max_cache_len, budget), workspace, workspace_bytes)) != EARN_OK) return rc;
  if (g_validate.load(std::memory_order_relaxed) && (rc = guarded(who, [&] { return validate_evict(who, cache_len, page_table, new_table, n_streams, max_cache_len, budget, max_pages, new_max_pages, n_pages, page_size, stream); })) != EARN_OK) return rc;
  return launch_cache_evict(desc, k_pages, v_pages, page_table, cache_len, n_streams, max_pages, n_pages, page_size, max_cache_len,
                            weights, weight_rows, budget, n_first, n_last, new_table, new_max_pages, kept_out, len_out, weights_out,
                            weight_rows_out, (hipStream_t)stream);
}

size_t earn_sample_workspace_bytes(int32_t rows, int32_t vocab) {
  (void)rows; (void)vocab;
  return 0;
}

int earn_sample(const void* logits, int32_t dtype, int64_t row_stride, int32_t rows, int32_t vocab, const float* temperature,
                const int32_t* top_k, const float* top_p, const float* min_p, const float* uniform, int32_t* token_out,
                float* logprob_out, int32_t* n_kept_out, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "earn_sample";
  g_err[0] = 0;
  if (dtype != EARN_F32 && dtype != EARN_BF16) { set_error("%s: unknown dtype %d", who, dtype); return EARN_ERR_UNSUPPORTED; }
  if (rows < 0 || vocab <= 0 || row_stride < vocab) {
    set_error("%s: rows (%d) must be non-negative, vocab (%d) positive, row_stride (%lld) at least vocab", who, rows, vocab, (long long)row_stride);
    return EARN_ERR_INVALID_ARG;
  }
  if (vocab > 524288 || rows > (1 << 21)) { set_error("%s: vocab (%d) beyond 524288 or rows (%d) beyond 2^21", who, vocab, rows); return EARN_ERR_UNSUPPORTED; }
  if (rows == 0) return EARN_OK;
  if (!logits || !uniform || !token_out) { set_error("%s: logits, uniform and token_out must not be NULL", who); return EARN_ERR_INVALID_ARG; }
  if ((uintptr_t)logits & (dtype == EARN_F32 ? 3 : 1)) { set_error("%s: logits are not aligned to their type", who); return EARN_ERR_INVALID_ARG; }
  const int rc = check_workspace(who, earn_sample_workspace_bytes(rows, vocab), workspace, workspace_bytes);
  if (rc != EARN_OK) return rc;
  return launch_sample(logits, dtype, row_stride, rows, vocab, temperature, top_k, top_p, min_p, uniform, token_out, logprob_out,
                       n_kept_out, (hipStream_t)stream);
}

int64_t earn_cache_entries(int32_t n_layers, int32_t split_k, int64_t seq_len, int32_t n_registers, int64_t gen) {
  return (int64_t)split_k * seq_len + (int64_t)(n_layers - split_k) * n_registers + (int64_t)n_layers * gen;
}

}  // extern "C"
