// C ABI of libhifa4 (declared in include/hifa4.h): argument validation,
// workspace carving and kernel launches.
#include "../../include/hifa4.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdarg>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <mutex>
#include <string>

#include "hifa4_decode.h"
#include "hifa4_internal.h"
#include "hifa4_paged.h"

namespace {

thread_local std::string g_last_error;

hifa4_status fail(hifa4_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
hifa4_status fail(hifa4_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return st;
}

hifa4_status hip_fail(hipError_t e, const char* what) {
  return fail(HIFA4_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

struct Dims {
  long tokens;   // rows of the [T, H, D] view
  int S;         // max_seqlen
  int NB;        // ceil(S/64)
};

// Vector loads and stores of the kernels need these alignments (a pointer
// that may be NULL passes).
bool aligned(const void* ptr, uintptr_t a) { return ((uintptr_t)ptr % a) == 0; }

hifa4_status check_aligned16(std::initializer_list<const void*> ptrs) {
  for (const void* ptr : ptrs)
    if (!aligned(ptr, 16)) return fail(HIFA4_ERR_INVALID_ARGUMENT, "tensor pointer %p is not 16-byte aligned", ptr);
  return HIFA4_OK;
}

hifa4_status check_aligned4(std::initializer_list<const void*> ptrs) {
  for (const void* ptr : ptrs)
    if (!aligned(ptr, 4)) return fail(HIFA4_ERR_INVALID_ARGUMENT, "pointer %p is not 4-byte aligned", ptr);
  return HIFA4_OK;
}

hifa4_status check_problem(const hifa4_problem* p, Dims* d) {
  if (!p) return fail(HIFA4_ERR_INVALID_ARGUMENT, "problem is NULL");
  if (p->batch <= 0 || p->num_heads_q <= 0 || p->num_heads_kv <= 0 || p->max_seqlen < 0)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "batch, head counts must be > 0 and max_seqlen >= 0");
  if (p->num_heads_q % p->num_heads_kv != 0)
    return fail(HIFA4_ERR_UNSUPPORTED, "num_heads_q (%d) must be a multiple of num_heads_kv (%d)", p->num_heads_q,
                p->num_heads_kv);
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256)
    return fail(HIFA4_ERR_UNSUPPORTED, "head_dim %d not in {64, 128, 256}", p->head_dim);
  if (p->causal != 1) return fail(HIFA4_ERR_UNSUPPORTED, "only causal prefill (causal = 1) is supported");
  if (p->cu_seqlens && p->total_tokens < 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "total_tokens < 0");
  d->S = p->max_seqlen;
  d->NB = (p->max_seqlen + 63) / 64;
  d->tokens = p->cu_seqlens ? (long)p->total_tokens : (long)p->batch * p->max_seqlen;
  if (d->tokens > (1L << 31) / std::max(1, p->num_heads_q))
    return fail(HIFA4_ERR_UNSUPPORTED, "problem too large for 32-bit row indexing");
  return HIFA4_OK;
}

}  // namespace

extern "C" {

const char* hifa4_last_error(void) { return g_last_error.c_str(); }

size_t hifa4_workspace_bytes(const hifa4_problem* p, const hifa4_fwd_options* opt) {
  Dims d;
  if (check_problem(p, &d) != HIFA4_OK) return 0;
  const bool fp16 = opt && (opt->operands == HIFA4_OPERANDS_FP16 || opt->operands == HIFA4_OPERANDS_P_ONLY);
  const bool qmean = opt && opt->q_mean != 0;
  const size_t chunk = fp16 ? hifa4::chunk_layout_fp16(p->head_dim).bytes
                            : hifa4::chunk_layout_hif4(p->head_dim / 64, qmean).bytes;
  return chunk * (size_t)p->batch * p->num_heads_kv * std::max(1, d.NB);
}

size_t hifa4_calibrate_workspace_bytes(const hifa4_problem* p, int32_t n_calib) {
  if (!p || n_calib <= 0 || p->num_heads_kv <= 0 || p->head_dim <= 0) return 0;
  return hifa4::round_up256((size_t)n_calib * 2 * p->num_heads_kv * p->head_dim * 4) + 32768 * 8;
}

hifa4_status hifa4_quantize_qk(const hifa4_problem* p, const void* q, const void* k, const float* s, void* q_codes,
                               void* q_meta, void* k_codes, void* k_meta, void* stream) {
  Dims d;
  hifa4_status st = check_problem(p, &d);
  if (st != HIFA4_OK) return st;
  const bool q_none = !q && !q_codes && !q_meta;
  if ((!q_none && (!q || !q_codes || !q_meta)) || !k || !k_codes || !k_meta)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if ((st = check_aligned16({q, k, s, q_codes, k_codes})) != HIFA4_OK) return st;
  if ((st = check_aligned4({q_meta, k_meta, p->cu_seqlens})) != HIFA4_OK) return st;
  hipStream_t hs = (hipStream_t)stream;
  using hifa4::half_t;
  hipError_t e = hipSuccess;
  if (!q_none) {
    e = hifa4::launch_quant_rows((const half_t*)q, s, (uint8_t*)q_codes, (uint32_t*)q_meta, d.tokens,
                                 p->num_heads_q, p->num_heads_kv, p->head_dim, false, hs);
    if (e != hipSuccess) return hip_fail(e, "quantize Q");
  }
  e = hifa4::launch_quant_rows((const half_t*)k, s, (uint8_t*)k_codes, (uint32_t*)k_meta, d.tokens, p->num_heads_kv,
                               p->num_heads_kv, p->head_dim, true, hs);
  if (e != hipSuccess) return hip_fail(e, "quantize K");
  return HIFA4_OK;
}

hifa4_status hifa4_quantize_v(const hifa4_problem* p, const void* v, void* v_codes, void* v_meta, void* stream) {
  Dims d;
  hifa4_status st = check_problem(p, &d);
  if (st != HIFA4_OK) return st;
  if (!v || !v_codes || !v_meta) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if ((st = check_aligned16({v, v_codes})) != HIFA4_OK) return st;
  if ((st = check_aligned4({v_meta, p->cu_seqlens})) != HIFA4_OK) return st;
  hipError_t e = hifa4::launch_quant_v((const hifa4::half_t*)v, p->cu_seqlens, (uint8_t*)v_codes, (uint32_t*)v_meta,
                                       p->batch, d.S, d.NB, p->num_heads_kv, p->head_dim, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "quantize V");
  return HIFA4_OK;
}

hifa4_status hifa4_attention_fwd(const hifa4_problem* p, const hifa4_fwd_options* opt, const void* q, const void* k,
                                 const void* v, const float* s, void* o, float* lse, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  Dims d;
  hifa4_status st = check_problem(p, &d);
  if (st != HIFA4_OK) return st;
  if (!opt) return fail(HIFA4_ERR_INVALID_ARGUMENT, "options is NULL");
  if (opt->norm != HIFA4_NORM_PREORDER && opt->norm != HIFA4_NORM_INCONSISTENT)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "unknown norm %d", opt->norm);
  if (opt->operands != HIFA4_OPERANDS_HIF4 && opt->operands != HIFA4_OPERANDS_FP16 &&
      opt->operands != HIFA4_OPERANDS_P_ONLY)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "unknown operands %d", opt->operands);
  if (!q || !k || !v || !o || !lse) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if ((opt->debug_p_codes == nullptr) != (opt->debug_p_meta == nullptr))
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "debug_p_codes and debug_p_meta must both be set or both be NULL");
  if ((st = check_aligned16({q, k, v, o, s, workspace, opt->debug_p_codes})) != HIFA4_OK) return st;
  if ((st = check_aligned4({lse, p->cu_seqlens, opt->debug_p_meta})) != HIFA4_OK) return st;
  if (opt->debug_head_count < 0 || opt->debug_token_count < 0 || opt->debug_head_begin < 0 ||
      opt->debug_token_begin < 0 || (!opt->debug_head_count && opt->debug_head_begin) ||
      (!opt->debug_token_count && opt->debug_token_begin) ||
      (long)opt->debug_head_begin + opt->debug_head_count > p->num_heads_q ||
      (long)opt->debug_token_begin + opt->debug_token_count > (long)d.tokens)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "debug window outside the problem");
  // FP16 and P-only keep Q, K and V in fp16 (fp16 chunk layout, no smoothing)
  const bool fp16 = opt->operands != HIFA4_OPERANDS_HIF4;
  if (fp16 && opt->q_mean)
    return fail(HIFA4_ERR_UNSUPPORTED, "q_mean applies to HIF4 operands only");
  const bool qmean = opt->q_mean != 0;
  const float* sm = (!fp16 && opt->smooth_qk) ? s : nullptr;
  if (!fp16 && opt->smooth_qk && !s) return fail(HIFA4_ERR_INVALID_ARGUMENT, "smooth_qk set but s is NULL");
  if (d.tokens == 0 || d.S == 0) return HIFA4_OK;
  const size_t need = hifa4_workspace_bytes(p, opt);
  if (!workspace || workspace_bytes < need)
    return fail(HIFA4_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", workspace_bytes, need);
  hipStream_t hs = (hipStream_t)stream;
  hipEvent_t* ev = (hipEvent_t*)opt->timing_events;
  hipError_t e = hipSuccess;
  if (ev && (e = hipEventRecord(ev[0], hs)) != hipSuccess) return hip_fail(e, "timing event");
  e = hifa4::launch_prep_kv((const hifa4::half_t*)k, (const hifa4::half_t*)v, sm, p->cu_seqlens, (uint8_t*)workspace,
                            p->batch, d.S, d.NB, p->num_heads_kv, p->head_dim, fp16, qmean, hs);
  if (e != hipSuccess) return hip_fail(e, "K/V pre-pass");
  if (ev && (e = hipEventRecord(ev[1], hs)) != hipSuccess) return hip_fail(e, "timing event");
  hifa4::AttnArgs a;
  a.q = (const hifa4::half_t*)q;
  a.s = sm;
  a.cu = p->cu_seqlens;
  a.ws = (const uint8_t*)workspace;
  a.o = (hifa4::half_t*)o;
  a.lse = lse;
  const bool dump = opt->operands != HIFA4_OPERANDS_FP16;
  a.dbg_codes = dump ? (uint8_t*)opt->debug_p_codes : nullptr;
  a.dbg_meta = dump ? (uint32_t*)opt->debug_p_meta : nullptr;
  a.dbg_h0 = opt->debug_head_count ? opt->debug_head_begin : 0;
  a.dbg_nh = opt->debug_head_count ? opt->debug_head_count : p->num_heads_q;
  a.dbg_t0 = opt->debug_token_count ? opt->debug_token_begin : 0;
  a.dbg_nt = opt->debug_token_count ? opt->debug_token_count : (int)d.tokens;
  a.batch = p->batch;
  a.S = d.S;
  a.NB = d.NB;
  a.hq = p->num_heads_q;
  a.hkv = p->num_heads_kv;
  a.D = p->head_dim;
  a.total_tokens = (int)d.tokens;
  a.c = (float)(1.4426950408889634 / std::sqrt((double)p->head_dim));
  e = hifa4::launch_attention(a, opt->norm, opt->operands, qmean, hs);
  if (e != hipSuccess) return hip_fail(e, "attention kernel");
  if (ev && (e = hipEventRecord(ev[2], hs)) != hipSuccess) return hip_fail(e, "timing event");
  return HIFA4_OK;
}

size_t hifa4_decode_workspace_bytes(const hifa4_problem* p) {
  Dims d;
  if (check_problem(p, &d) != HIFA4_OK) return 0;
  return hifa4::decode_workspace_bytes(p->batch, p->num_heads_q, p->num_heads_kv, p->head_dim, std::max(1, d.NB));
}

hifa4_status hifa4_decode_fwd(const hifa4_problem* p, const hifa4_fwd_options* opt, const void* q,
                              const void* k_codes, const void* k_meta, const void* v_codes, const void* v_meta,
                              const float* s, void* o, float* lse, void* workspace, size_t workspace_bytes,
                              void* stream) {
  Dims d;
  hifa4_status st = check_problem(p, &d);
  if (st != HIFA4_OK) return st;
  if (!opt) return fail(HIFA4_ERR_INVALID_ARGUMENT, "options is NULL");
  if (opt->norm != HIFA4_NORM_PREORDER && opt->norm != HIFA4_NORM_INCONSISTENT)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "unknown norm %d", opt->norm);
  if (opt->operands != HIFA4_OPERANDS_HIF4)
    return fail(HIFA4_ERR_UNSUPPORTED, "decode reads a HIF4 cache: operands must be HIFA4_OPERANDS_HIF4");
  if (opt->q_mean) return fail(HIFA4_ERR_UNSUPPORTED, "q_mean is not supported by decode (the cache has no key sums)");
  if (p->num_heads_q / p->num_heads_kv > 8)
    return fail(HIFA4_ERR_UNSUPPORTED, "decode supports at most 8 query heads per kv head (got %d)",
                p->num_heads_q / p->num_heads_kv);
  if (!q || !k_codes || !k_meta || !v_codes || !v_meta || !o || !lse)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if ((opt->debug_p_codes == nullptr) != (opt->debug_p_meta == nullptr))
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "debug_p_codes and debug_p_meta must both be set or both be NULL");
  if ((st = check_aligned16({q, k_codes, v_codes, o, s, workspace, opt->debug_p_codes})) != HIFA4_OK) return st;
  if ((st = check_aligned4({k_meta, v_meta, lse, p->cu_seqlens, opt->debug_p_meta})) != HIFA4_OK) return st;
  if (opt->smooth_qk && !s) return fail(HIFA4_ERR_INVALID_ARGUMENT, "smooth_qk set but s is NULL");
  if (d.tokens == 0 || d.S == 0) return HIFA4_OK;
  const size_t need = hifa4_decode_workspace_bytes(p);
  if (!workspace || workspace_bytes < need)
    return fail(HIFA4_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", workspace_bytes, need);
  hipStream_t hs = (hipStream_t)stream;
  hipEvent_t* ev = (hipEvent_t*)opt->timing_events;
  hipError_t e = hipSuccess;
  if (ev && (e = hipEventRecord(ev[0], hs)) != hipSuccess) return hip_fail(e, "timing event");
  hifa4::DecodeLaunch dl;
  dl.q = (const hifa4::half_t*)q;
  dl.s = opt->smooth_qk ? s : nullptr;
  dl.cu = p->cu_seqlens;
  dl.kc = (const uint8_t*)k_codes;
  dl.km = (const uint32_t*)k_meta;
  dl.vc = (const uint8_t*)v_codes;
  dl.vm = (const uint32_t*)v_meta;
  dl.o = (hifa4::half_t*)o;
  dl.lse = lse;
  dl.dbg_codes = (uint8_t*)opt->debug_p_codes;
  dl.dbg_meta = (uint32_t*)opt->debug_p_meta;
  dl.ws = (uint8_t*)workspace;
  dl.ev = ev;
  dl.batch = p->batch;
  dl.S = d.S;
  dl.NB = d.NB;
  dl.hq = p->num_heads_q;
  dl.hkv = p->num_heads_kv;
  dl.D = p->head_dim;
  dl.norm = opt->norm;
  dl.tokens = d.tokens;
  dl.test_no_publish = opt->test_decode_no_publish == 2 ? 2 : opt->test_decode_no_publish ? 1 : 0;
  dl.c = (float)(1.4426950408889634 / std::sqrt((double)p->head_dim));
  e = hifa4::launch_decode(dl, hs);
  if (e != hipSuccess) return hip_fail(e, "decode kernels");
  if (ev && (e = hipEventRecord(ev[2], hs)) != hipSuccess) return hip_fail(e, "timing event");
  return HIFA4_OK;
}

// ---------------------------------------------------------------------------
// The paged cache.
namespace {

hifa4_status check_paged_shape(int32_t heads_kv, int32_t D, int32_t operands) {
  if (heads_kv <= 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "num_heads_kv must be > 0");
  if (D != 64 && D != 128 && D != 256) return fail(HIFA4_ERR_UNSUPPORTED, "head_dim %d not in {64, 128, 256}", D);
  if (operands != HIFA4_OPERANDS_HIF4 && operands != HIFA4_OPERANDS_FP16)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "pages hold HIF4 or FP16 operands, not %d", operands);
  return HIFA4_OK;
}

// `touches`: the entry point reads or writes pages (else only sizes are asked for)
hifa4_status check_paged(const hifa4_paged_cache* c, bool touches, hifa4::PagedCache* out) {
  if (!c) return fail(HIFA4_ERR_INVALID_ARGUMENT, "cache is NULL");
  hifa4_status st = check_paged_shape(c->num_heads_kv, c->head_dim, c->operands);
  if (st != HIFA4_OK) return st;
  if (c->batch <= 0 || c->num_pages <= 0 || c->max_pages <= 0)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "batch, num_pages and max_pages must be > 0");
  if (c->max_pages >= (1 << 25) || (int64_t)c->batch * c->max_pages >= (1LL << 30))
    return fail(HIFA4_ERR_UNSUPPORTED, "a table of %d x %d pages is too large", c->batch, c->max_pages);
  if (touches) {
    if (!c->pool || !c->block_table || !c->seq_lens) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null cache pointer");
    if ((st = check_aligned16({c->pool, c->v_tail})) != HIFA4_OK) return st;
    if ((st = check_aligned4({c->block_table, c->seq_lens})) != HIFA4_OK) return st;
  }
  out->pool = (uint8_t*)c->pool;
  out->table = c->block_table;
  out->lens = c->seq_lens;
  out->tail = (hifa4::half_t*)c->v_tail;
  out->batch = c->batch;
  out->hkv = c->num_heads_kv;
  out->D = c->head_dim;
  out->num_pages = c->num_pages;
  out->max_pages = c->max_pages;
  out->fp16 = c->operands == HIFA4_OPERANDS_FP16;
  return HIFA4_OK;
}

hifa4_status check_query_heads(int32_t hq, int32_t batch, int32_t hkv) {
  if (hq <= 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "num_heads_q must be > 0");
  if (hq % hkv) return fail(HIFA4_ERR_UNSUPPORTED, "num_heads_q (%d) must be a multiple of num_heads_kv (%d)", hq, hkv);
  if ((int64_t)batch * hq >= (1LL << 24))
    return fail(HIFA4_ERR_UNSUPPORTED, "problem too large for 32-bit row indexing");
  return HIFA4_OK;
}

// workgroups of `threads` threads of a launch over (sequence, page, head)
hifa4_status check_page_grid(const hifa4_paged_cache* c, int32_t tokens, int threads, const char* bound) {
  const int64_t blocks = ((int64_t)tokens + 62) / 64 + 1;
  if ((int64_t)c->batch * c->num_heads_kv >= (1LL << 31) ||
      (size_t)(blocks * c->batch * c->num_heads_kv) >= hifa4::max_grid(threads))
    return fail(HIFA4_ERR_UNSUPPORTED, "too many pages for one launch (%s of %d tokens for each of %d sequences)", bound,
                tokens, c->batch);
  return HIFA4_OK;
}
hifa4_status check_decode_grid(const hifa4::PagedCache& c, int32_t hq, bool weights) {
  if (!hifa4::paged_decode_fits(c, hq, weights))
    return fail(HIFA4_ERR_UNSUPPORTED, "%d x %d pages%s are too many for one launch", c.batch, c.max_pages,
                weights ? " with page weights" : "");
  return HIFA4_OK;
}

}  // namespace

size_t hifa4_paged_page_bytes(int32_t num_heads_kv, int32_t head_dim, int32_t operands) {
  if (check_paged_shape(num_heads_kv, head_dim, operands) != HIFA4_OK) return 0;
  return (size_t)num_heads_kv * hifa4::paged_record_bytes(head_dim, operands == HIFA4_OPERANDS_FP16);
}

hifa4_status hifa4_paged_append(const hifa4_paged_cache* c, int32_t total_new, int32_t max_new, const int32_t* cu_new,
                                const void* k, const void* v, const float* s, void* stream) {
  hifa4::PagedAppend a;
  hifa4_status st = check_paged(c, true, &a.c);
  if (st != HIFA4_OK) return st;
  if (total_new < 0 || max_new < 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "total_new and max_new must be >= 0");
  if (!cu_new && total_new != c->batch)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "without cu_new there is one new token per sequence (%d), not %d in all",
                c->batch, total_new);
  if (total_new == 0 || max_new == 0) return HIFA4_OK;
  if (!k || !v) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if (!a.c.fp16 && !c->v_tail) return fail(HIFA4_ERR_INVALID_ARGUMENT, "HIF4 pages need v_tail");
  if ((st = check_aligned16({k, v, s})) != HIFA4_OK) return st;
  if ((st = check_aligned4({cu_new})) != HIFA4_OK) return st;
  a.max_new = cu_new ? std::min(max_new, total_new) : 1;
  if ((st = check_page_grid(c, a.max_new, hifa4::paged_append_threads(c->head_dim, a.c.fp16), "max_new")) != HIFA4_OK) return st;
  a.k = (const hifa4::half_t*)k;
  a.v = (const hifa4::half_t*)v;
  a.s = s;
  a.cu = cu_new;
  a.total = total_new;
  const hipError_t e = hifa4::launch_paged_append(a, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "paged append");
  return HIFA4_OK;
}

hifa4_status hifa4_paged_gather(const hifa4_paged_cache* c, int32_t total_tokens, int32_t max_tokens,
                                const int32_t* cu_tokens, const int32_t* starts, void* k, void* v, void* stream) {
  hifa4::PagedGather a;
  hifa4_status st = check_paged(c, true, &a.c);
  if (st != HIFA4_OK) return st;
  if (total_tokens < 0 || max_tokens < 0)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "total_tokens and max_tokens must be >= 0");
  if (!cu_tokens) return fail(HIFA4_ERR_INVALID_ARGUMENT, "cu_tokens is NULL");
  if (total_tokens == 0 || max_tokens == 0) return HIFA4_OK;
  if (!k || !v) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if ((st = check_aligned16({k, v})) != HIFA4_OK) return st;
  if ((st = check_aligned4({cu_tokens, starts})) != HIFA4_OK) return st;
  a.max_tokens = std::min(max_tokens, total_tokens);
  if ((st = check_page_grid(c, a.max_tokens, 256, "max_tokens")) != HIFA4_OK) return st;
  a.cu = cu_tokens;
  a.starts = starts;
  a.k = (hifa4::half_t*)k;
  a.v = (hifa4::half_t*)v;
  a.total = total_tokens;
  const hipError_t e = hifa4::launch_paged_gather(a, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "paged gather");
  return HIFA4_OK;
}

size_t hifa4_paged_decode_workspace_bytes(const hifa4_paged_cache* c, int32_t num_heads_q, int32_t page_weights) {
  hifa4::PagedCache pc;
  if (check_paged(c, false, &pc) != HIFA4_OK || check_query_heads(num_heads_q, c->batch, c->num_heads_kv) != HIFA4_OK ||
      check_decode_grid(pc, num_heads_q, page_weights != 0) != HIFA4_OK)
    return 0;
  return hifa4::paged_decode_workspace(pc, num_heads_q, page_weights != 0);
}

hifa4_status hifa4_paged_decode_fwd(const hifa4_paged_cache* c, int32_t num_heads_q, const void* q, const float* s,
                                    void* o, float* lse, const float* page_weights, float* weights_out, float decay,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  hifa4::PagedDecode a;
  hifa4_status st = check_paged(c, true, &a.c);
  if (st != HIFA4_OK) return st;
  if ((st = check_query_heads(num_heads_q, c->batch, c->num_heads_kv)) != HIFA4_OK) return st;
  if ((st = check_decode_grid(a.c, num_heads_q, page_weights != nullptr)) != HIFA4_OK) return st;
  if (!q || !o || !lse) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if ((page_weights == nullptr) != (weights_out == nullptr))
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "page_weights and weights_out must both be set or both be NULL");
  if (page_weights && !std::isfinite(decay)) return fail(HIFA4_ERR_INVALID_ARGUMENT, "decay must be finite");
  if ((st = check_aligned16({q, s, o, workspace})) != HIFA4_OK) return st;
  if ((st = check_aligned4({lse, page_weights, weights_out})) != HIFA4_OK) return st;
  const size_t need = hifa4::paged_decode_workspace(a.c, num_heads_q, page_weights != nullptr);
  if (!workspace || workspace_bytes < need)
    return fail(HIFA4_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", workspace_bytes, need);
  a.hq = num_heads_q;
  a.q = (const hifa4::half_t*)q;
  a.s = s;
  a.o = (hifa4::half_t*)o;
  a.lse = lse;
  a.w_in = page_weights;
  a.w_out = weights_out;
  a.decay = decay;
  a.scale = (float)(1.4426950408889634 / std::sqrt((double)c->head_dim));
  a.ws = (uint8_t*)workspace;
  const hipError_t e = hifa4::launch_paged_decode(a, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "paged decode kernels");
  return HIFA4_OK;
}

hifa4_status hifa4_paged_evict(int32_t batch, int32_t max_pages, const int32_t* block_table, const int32_t* seq_lens,
                               const float* page_weights, int32_t budget, int32_t first, int32_t last,
                               int32_t* out_table, int32_t* out_lens, float* out_weights, int32_t* freed,
                               int32_t* num_freed, void* stream) {
  if (batch <= 0 || max_pages <= 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "batch and max_pages must be > 0");
  if (max_pages >= (1 << 25) || (int64_t)batch * max_pages >= (1LL << 30) || batch >= (1 << 22))
    return fail(HIFA4_ERR_UNSUPPORTED, "a table of %d x %d pages is too large", batch, max_pages);
  if (first < 0 || last < 1 || (int64_t)first + last > budget)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "needs first >= 0, last >= 1 and first + last <= budget (%d, %d, %d)", first,
                last, budget);
  if (!block_table || !seq_lens || !page_weights || !out_table || !out_lens || !out_weights || !freed || !num_freed)
    return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  const hifa4_status st = check_aligned4(
      {block_table, seq_lens, page_weights, out_table, out_lens, out_weights, freed, num_freed});
  if (st != HIFA4_OK) return st;
  hifa4::PagedEvict a;
  a.batch = batch;
  a.max_pages = max_pages;
  a.budget = budget;
  a.first = first;
  a.last = last;
  a.table = block_table;
  a.lens = seq_lens;
  a.w = page_weights;
  a.out_table = out_table;
  a.out_lens = out_lens;
  a.out_w = out_weights;
  a.freed = freed;
  a.num_freed = num_freed;
  const hipError_t e = hifa4::launch_paged_evict(a, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "paged evict");
  return HIFA4_OK;
}

hifa4_status hifa4_selftest_exp2(const void* x, void* y, int64_t n, void* stream) {
  if (n < 0 || (n > 0 && (!x || !y))) return fail(HIFA4_ERR_INVALID_ARGUMENT, "bad self-test arguments");
  hipError_t e = hifa4::launch_selftest_exp2((const hifa4::half_t*)x, (hifa4::half_t*)y, (long)n, (hipStream_t)stream);
  if (e != hipSuccess) return hip_fail(e, "exp2 self-test");
  return HIFA4_OK;
}

hifa4_status hifa4_calibrate_smooth_qk(const hifa4_problem* p, int32_t n_calib, const void* q_calib,
                                       const void* k_calib, float alpha, float* s_out, hifa4_calib_report* report,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  if (!p) return fail(HIFA4_ERR_INVALID_ARGUMENT, "problem is NULL");
  if (n_calib <= 0 || p->max_seqlen <= 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "n_calib and max_seqlen must be > 0");
  if (p->num_heads_q <= 0 || p->num_heads_kv <= 0 || p->num_heads_q % p->num_heads_kv)
    return fail(HIFA4_ERR_UNSUPPORTED, "num_heads_q must be a positive multiple of num_heads_kv");
  if (p->head_dim != 64 && p->head_dim != 128 && p->head_dim != 256)
    return fail(HIFA4_ERR_UNSUPPORTED, "head_dim %d not in {64, 128, 256}", p->head_dim);
  if (!q_calib || !k_calib || !s_out) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  hifa4_status st = check_aligned16({q_calib, k_calib, workspace});
  if (st == HIFA4_OK) st = check_aligned4({s_out});
  if (st != HIFA4_OK) return st;
  if (!std::isfinite(alpha) || alpha >= 1.0f) return fail(HIFA4_ERR_INVALID_ARGUMENT, "alpha must be finite and < 1");
  const size_t need = hifa4_calibrate_workspace_bytes(p, n_calib);
  if (!workspace || workspace_bytes < need)
    return fail(HIFA4_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", workspace_bytes, need);
  const int hkv = p->num_heads_kv, D = p->head_dim, S = p->max_seqlen;
  const size_t n_stats = (size_t)n_calib * 2 * hkv * D;
  uint32_t* stats = (uint32_t*)workspace;
  unsigned long long* hist = (unsigned long long*)((uint8_t*)workspace + hifa4::round_up256(n_stats * 4));
  hipStream_t hs = (hipStream_t)stream;
  hipError_t e = hifa4::launch_calib((const hifa4::half_t*)q_calib, (const hifa4::half_t*)k_calib, n_calib, S,
                                     p->num_heads_q, hkv, D, alpha, stats, hist, s_out, hs);
  if (e != hipSuccess) return hip_fail(e, "calibration kernels");
  hifa4::CalibGate gate;
  e = hipMemcpyAsync(&gate, hist, sizeof gate, hipMemcpyDeviceToHost, hs);
  if (e == hipSuccess) e = hipStreamSynchronize(hs);
  if (e != hipSuccess) return hip_fail(e, "calibration copy-back");
  if (report) {
    report->rho_k = gate.rho;
    report->t_kq = gate.t_kq;
    report->branch = gate.branch;
    report->alpha_used = (float)gate.alpha;
  }
  return HIFA4_OK;
}

hifa4_status hifa4_calibrate_smooth_qk_layers(const hifa4_problem* p, int32_t n_layers, int32_t n_calib,
                                              const void* q_calib, const void* k_calib, float alpha, float* s_out,
                                              hifa4_calib_report* reports, void* workspace, size_t workspace_bytes,
                                              void* stream) {
  if (!p) return fail(HIFA4_ERR_INVALID_ARGUMENT, "problem is NULL");
  if (n_layers <= 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "n_layers must be > 0");
  if (!q_calib || !k_calib || !s_out) return fail(HIFA4_ERR_INVALID_ARGUMENT, "null tensor pointer");
  if (n_calib <= 0 || p->max_seqlen <= 0) return fail(HIFA4_ERR_INVALID_ARGUMENT, "n_calib and max_seqlen must be > 0");
  const size_t q_layer = (size_t)n_calib * p->max_seqlen * p->num_heads_q * p->head_dim;
  const size_t k_layer = (size_t)n_calib * p->max_seqlen * p->num_heads_kv * p->head_dim;
  const size_t s_layer = (size_t)p->num_heads_kv * p->head_dim;
  for (int32_t l = 0; l < n_layers; ++l) {
    const hifa4_status st = hifa4_calibrate_smooth_qk(
        p, n_calib, (const uint16_t*)q_calib + l * q_layer, (const uint16_t*)k_calib + l * k_layer, alpha,
        s_out + l * s_layer, reports ? reports + l : nullptr, workspace, workspace_bytes, stream);
    if (st != HIFA4_OK) {
      const std::string msg = g_last_error;
      return fail(st, "layer %d: %s", l, msg.c_str());
    }
  }
  return HIFA4_OK;
}

}  // extern "C"

// ---------------------------------------------------------------------------
// hifa4_attention_fwd_noalloc: the forward with its K/V pre-pass workspace in
// a file-scope device array (one copy per GPU, held until the process ends),
// for callers that cannot allocate.  In host code `scratch` names a host-side
// stand-in, never the device memory: the device address comes from
// hipGetSymbolAddress, once per device with that device current, and only
// that address is passed to kernels.
static __device__ __align__(256) uint8_t scratch[HIFA4_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

hifa4_status scratch_pointer(void** out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  if (dev < 0 || dev >= kMaxDevices) return fail(HIFA4_ERR_UNSUPPORTED, "device index %d above %d", dev, kMaxDevices - 1);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void* ptr = nullptr;
    e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return hip_fail(e, "hipGetSymbolAddress(scratch)");
    if (!ptr) return fail(HIFA4_ERR_HIP, "hipGetSymbolAddress(scratch) returned NULL");
    g_scratch_ptr[dev] = ptr;
  }
  *out = g_scratch_ptr[dev];
  return HIFA4_OK;
}

}  // namespace

hifa4_status hifa4_attention_fwd_noalloc(const hifa4_problem* p, const hifa4_fwd_options* opt, const void* q,
                                         const void* k, const void* v, const float* s, void* o, float* lse,
                                         void* stream) {
  Dims d;
  hifa4_status st = check_problem(p, &d);
  if (st != HIFA4_OK) return st;
  if (!opt) return fail(HIFA4_ERR_INVALID_ARGUMENT, "options is NULL");
  const size_t need = hifa4_workspace_bytes(p, opt);
  if (need > (size_t)HIFA4_NOALLOC_SCRATCH_BYTES)
    return fail(HIFA4_ERR_WORKSPACE,
                "problem needs %zu bytes of scratch; hifa4_attention_fwd_noalloc holds at most %zu "
                "(use hifa4_attention_fwd with a caller workspace)",
                need, (size_t)HIFA4_NOALLOC_SCRATCH_BYTES);
  void* ws = nullptr;
  if ((st = scratch_pointer(&ws)) != HIFA4_OK) return st;
  return hifa4_attention_fwd(p, opt, q, k, v, s, o, lse, ws, (size_t)HIFA4_NOALLOC_SCRATCH_BYTES, stream);
}
