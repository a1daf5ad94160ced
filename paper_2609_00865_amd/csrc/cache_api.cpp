// C ABI of the cache, its attention and the rotary positions with several
// axes: argument validation and dispatch.  As in api.cpp, validation is
// complete before anything is enqueued.
#include <cmath>
#include <sstream>

#include "mv_cache_dev.h"

namespace mv {

hipError_t launch_rope_axes(const mv_rope_axes_spec& spec, int n, int H, int d, const void* x,
                            int64_t xs, const int32_t* pos, int direction, void* out, int64_t os,
                            hipStream_t stream);
hipError_t launch_cache_write(const CacheDev& a, int layer, int n, const int32_t* slot,
                              const void* k, int64_t ks, const void* v, int64_t vs,
                              const mv_rope_axes_spec* spec, const int32_t* pos,
                              hipStream_t stream);
hipError_t launch_cache_reset(const CacheDev& a, hipStream_t stream);
hipError_t launch_cache_count(const CacheDev& a, hipStream_t stream);
hipError_t launch_cache_clear_counts(const CacheDev& a, hipStream_t stream);
hipError_t launch_cache_reserve(const CacheDev& a, int n, const int32_t* ids, const int32_t* ptr,
                                int n_new, int32_t* slot, int32_t* pos, hipStream_t stream);
size_t cache_move_ws_bytes(const mv_cache_shape& s, int n);
hipError_t launch_cache_move(const mv_cache_shape& shape, const CacheDev& a, int n,
                             const int32_t* src, const int32_t* dst, const int32_t* span_ptr,
                             const mv_span* spans, int n_spans, bool share, void* ws,
                             hipStream_t stream);
hipError_t launch_cache_free(const CacheDev& a, int n, const int32_t* ids, hipStream_t stream);
size_t tree_attn_ws_bytes(const mv_cache_shape& c, const mv_tree_attn_shape& s);
bool tree_attn_fits(const mv_cache_shape& c, const mv_tree_attn_shape& s);
hipError_t launch_tree_attn(const mv_cache_shape& cs, const CacheDev& cd, int layer,
                            const mv_tree_attn_shape& s, float scale, const int32_t* ids,
                            const int32_t* ptr, const uint32_t* tree, const void* q, void* o,
                            float* lse, void* ws, hipStream_t stream);
hipError_t launch_tree_mask(int B, int N, const int32_t* ptr, const int32_t* parent, int words,
                            uint32_t* tree, int32_t* depth, hipStream_t stream);

}  // namespace mv

namespace {

mv_status fail(mv_status s, const std::string& msg) {
  mv::set_error(msg);
  return s;
}

mv_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return MV_OK;
  return fail(MV_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

mv_status check_ptrs(std::initializer_list<const void*> ps) {
  for (const void* p : ps) {
    if (p == nullptr) return fail(MV_ERR_INVALID_ARG, "null device pointer");
    if (reinterpret_cast<uintptr_t>(p) & 15)
      return fail(MV_ERR_INVALID_ARG, "device pointer not 16-byte aligned");
  }
  return MV_OK;
}

// Index arrays: present, and aligned as their words are.
mv_status check_words(std::initializer_list<const void*> ps) {
  for (const void* p : ps) {
    if (p == nullptr) return fail(MV_ERR_INVALID_ARG, "null index array");
    if (reinterpret_cast<uintptr_t>(p) & 3)
      return fail(MV_ERR_INVALID_ARG, "index array not 4-byte aligned");
  }
  return MV_OK;
}

mv_status check_rope(const mv_rope_axes_spec* s, int head_dim) {
  if (s->rotary_dim < 2 || s->rotary_dim % 2 != 0 || s->rotary_dim > head_dim ||
      s->rotary_dim > 2 * MV_ROPE_MAX_PAIRS)
    return fail(MV_ERR_SHAPE, "rotary_dim must be even and in [2, head_dim]");
  if (s->n_axes < 1 || s->n_axes > MV_ROPE_MAX_AXES)
    return fail(MV_ERR_SHAPE, "n_axes must be in [1, 8]");
  if (!(s->theta > 0.f) || !std::isfinite(s->theta))
    return fail(MV_ERR_INVALID_ARG, "theta must be positive and finite");
  for (int i = 0; i < s->rotary_dim / 2; ++i)
    if (s->axis[i] >= s->n_axes) return fail(MV_ERR_SHAPE, "axis of a pair >= n_axes");
  return MV_OK;
}

mv_status check_stride(int64_t stride, int64_t row, const char* what) {
  if (stride < row || stride % 8 != 0)
    return fail(MV_ERR_SHAPE, std::string(what) +
                                  " must be a multiple of 8 and at least one token's elements");
  return MV_OK;
}

mv_status check_cache_shape(const mv_cache_shape* s) {
  if (s == nullptr) return fail(MV_ERR_INVALID_ARG, "null cache shape");
  if (s->n_layers <= 0 || s->n_pages <= 0 || s->n_heads_kv <= 0 || s->n_seqs <= 0 ||
      s->max_pages <= 0)
    return fail(MV_ERR_SHAPE, "every size of the cache must be positive");
  if (s->page_size != 16 && s->page_size != 32 && s->page_size != 64 && s->page_size != 128 &&
      s->page_size != 256)
    return fail(MV_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256");
  if (s->head_dim != 64 && s->head_dim != 128)
    return fail(MV_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (s->n_seqs > MV_CACHE_MAX_SEQS)
    return fail(MV_ERR_UNSUPPORTED, "more sequences than MV_CACHE_MAX_SEQS");
  if (int64_t(s->n_pages) * s->page_size >= (int64_t(1) << 31) ||
      int64_t(s->max_pages) * s->page_size >= (int64_t(1) << 31) ||
      int64_t(s->n_seqs) * s->max_pages >= (int64_t(1) << 30))
    return fail(MV_ERR_UNSUPPORTED, "rows of the pool or of a sequence must stay below 2^31, "
                                    "entries of the page table below 2^30");
  if (int64_t(s->n_heads_kv) * s->page_size * s->head_dim >= (int64_t(1) << 30))
    return fail(MV_ERR_UNSUPPORTED, "a page of more than 2^30 elements");
  return MV_OK;
}

mv_status check_cache(const mv_cache_shape* s, const mv_cache* c, mv::CacheDev* d) {
  if (mv_status st = check_cache_shape(s); st != MV_OK) return st;
  if (c == nullptr) return fail(MV_ERR_INVALID_ARG, "null cache");
  if (mv_status st = check_ptrs({c->k, c->v, c->page_table, c->seq_len, c->page_refs, c->ctl});
      st != MV_OK)
    return st;
  d->k = static_cast<mv::u16*>(c->k);
  d->v = static_cast<mv::u16*>(c->v);
  d->table = c->page_table;
  d->len = c->seq_len;
  d->refs = c->page_refs;
  d->ctl = c->ctl;
  d->n_layers = s->n_layers;
  d->n_pages = s->n_pages;
  d->n_seqs = s->n_seqs;
  d->max_pages = s->max_pages;
  d->Hkv = s->n_heads_kv;
  d->D = s->head_dim;
  d->psl = __builtin_ctz(unsigned(s->page_size));
  return MV_OK;
}

mv_status check_entries(int32_t n) {
  if (n < 0) return fail(MV_ERR_SHAPE, "a negative number of entries");
  if (n > MV_CACHE_MAX_SEQS) return fail(MV_ERR_UNSUPPORTED, "more entries than MV_CACHE_MAX_SEQS");
  return MV_OK;
}

mv_status check_tree_shape(const mv_cache_shape* c, const mv_tree_attn_shape* s) {
  if (mv_status st = check_cache_shape(c); st != MV_OK) return st;
  if (s == nullptr) return fail(MV_ERR_INVALID_ARG, "null shape");
  if (mv_status st = check_entries(s->n_batch); st != MV_OK) return st;
  if (s->n_rows < 0 || s->tree_words < 0 || s->max_len < 0)
    return fail(MV_ERR_SHAPE, "n_rows, tree_words and max_len must be >= 0");
  if (s->n_heads_q <= 0 || s->n_heads_q % c->n_heads_kv != 0)
    return fail(MV_ERR_SHAPE, "n_heads_q must be a positive multiple of n_heads_kv");
  if (!std::isfinite(s->softmax_scale)) return fail(MV_ERR_INVALID_ARG, "softmax_scale not finite");
  if (int64_t(s->n_rows) * s->n_heads_q >= (int64_t(1) << 30) || !mv::tree_attn_fits(*c, *s))
    return fail(MV_ERR_UNSUPPORTED, "too many rows in one call");
  return MV_OK;
}

mv_status check_space(const char* what, size_t have, size_t need) {
  if (have >= need) return MV_OK;
  std::ostringstream os;
  os << what << " workspace has " << have << " bytes, needs " << need;
  return fail(MV_ERR_WORKSPACE, os.str());
}

}  // namespace

extern "C" {

mv_status mv_rope_axes(const mv_rope_axes_spec* spec, int32_t n_tokens, int32_t n_heads,
                       int32_t head_dim, const void* x, int64_t x_stride, const int32_t* pos,
                       int32_t direction, void* out, int64_t out_stride, hipStream_t stream) {
  if (spec == nullptr) return fail(MV_ERR_INVALID_ARG, "null rotary spec");
  if (n_tokens < 0 || n_heads <= 0 || head_dim <= 0)
    return fail(MV_ERR_SHAPE, "n_tokens >= 0, n_heads > 0, head_dim > 0 required");
  if (head_dim % 8 != 0 || head_dim > 256)
    return fail(MV_ERR_UNSUPPORTED, "head_dim must be a multiple of 8, at most 256");
  if (mv_status st = check_rope(spec, head_dim); st != MV_OK) return st;
  if (direction != 1 && direction != -1)
    return fail(MV_ERR_INVALID_ARG, "direction must be +1 or -1");
  const int64_t row = int64_t(n_heads) * head_dim;
  if (mv_status st = check_stride(x_stride, row, "x_stride"); st != MV_OK) return st;
  if (mv_status st = check_stride(out_stride, row, "out_stride"); st != MV_OK) return st;
  if (row >= (int64_t(1) << 30)) return fail(MV_ERR_UNSUPPORTED, "a token of 2^30 elements");
  if (n_tokens == 0) return MV_OK;
  if (mv_status st = check_ptrs({x, out}); st != MV_OK) return st;
  if (mv_status st = check_words({pos}); st != MV_OK) return st;
  if (x == out && x_stride != out_stride)
    return fail(MV_ERR_INVALID_ARG, "in place, both strides must be equal");
  return hip_status(mv::launch_rope_axes(*spec, n_tokens, n_heads, head_dim, x, x_stride, pos,
                                         direction, out, out_stride, stream),
                    "rotary launch");
}

mv_status mv_cache_reset(const mv_cache_shape* s, const mv_cache* c, hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(s, c, &d); st != MV_OK) return st;
  return hip_status(mv::launch_cache_reset(d, stream), "cache reset launch");
}

mv_status mv_cache_status(const mv_cache_shape* s, const mv_cache* c, mv_cache_counts* host_out,
                          hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(s, c, &d); st != MV_OK) return st;
  if (host_out == nullptr) return fail(MV_ERR_INVALID_ARG, "null host_out");
  int32_t w[4] = {0, 0, 0, 0};
  if (hipError_t e = mv::launch_cache_count(d, stream); e != hipSuccess)
    return hip_status(e, "cache count launch");
  if (hipError_t e = hipMemcpyAsync(w, c->ctl, sizeof w, hipMemcpyDeviceToHost, stream);
      e != hipSuccess)
    return hip_status(e, "cache status copy");
  if (hipError_t e = mv::launch_cache_clear_counts(d, stream); e != hipSuccess)
    return hip_status(e, "cache status launch");
  if (hipError_t e = hipStreamSynchronize(stream); e != hipSuccess)
    return hip_status(e, "cache status wait");
  host_out->refused_pages = w[1];
  host_out->refused_entries = w[2];
  host_out->free_pages = w[3];
  return MV_OK;
}

mv_status mv_cache_reserve(const mv_cache_shape* s, const mv_cache* c, int32_t n,
                           const int32_t* seq_ids, const int32_t* new_ptr, int32_t n_new,
                           int32_t* slot, int32_t* pos, hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(s, c, &d); st != MV_OK) return st;
  if (mv_status st = check_entries(n); st != MV_OK) return st;
  if (n_new < 0) return fail(MV_ERR_SHAPE, "n_new must be >= 0");
  if (n == 0 && n_new == 0) return MV_OK;
  if (n > 0)
    if (mv_status st = check_words({seq_ids, new_ptr}); st != MV_OK) return st;
  if (n_new > 0)
    if (mv_status st = check_words({slot}); st != MV_OK) return st;
  if (pos != nullptr)
    if (mv_status st = check_words({pos}); st != MV_OK) return st;
  return hip_status(mv::launch_cache_reserve(d, n, seq_ids, new_ptr, n_new, slot, pos, stream),
                    "cache reserve launch");
}

mv_status mv_cache_write(const mv_cache_shape* s, const mv_cache* c, int32_t layer, int32_t n_rows,
                         const int32_t* slot, const void* k, int64_t k_stride, const void* v,
                         int64_t v_stride, const mv_rope_axes_spec* rope, const int32_t* pos,
                         hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(s, c, &d); st != MV_OK) return st;
  if (layer < 0 || layer >= s->n_layers) return fail(MV_ERR_SHAPE, "layer outside the cache");
  if (n_rows < 0) return fail(MV_ERR_SHAPE, "n_rows must be >= 0");
  const int64_t row = int64_t(s->n_heads_kv) * s->head_dim;
  if (mv_status st = check_stride(k_stride, row, "k_stride"); st != MV_OK) return st;
  if (mv_status st = check_stride(v_stride, row, "v_stride"); st != MV_OK) return st;
  if (rope != nullptr)
    if (mv_status st = check_rope(rope, s->head_dim); st != MV_OK) return st;
  if (n_rows == 0) return MV_OK;
  if (mv_status st = check_ptrs({k, v}); st != MV_OK) return st;
  if (mv_status st = check_words({slot}); st != MV_OK) return st;
  if (rope != nullptr)
    if (mv_status st = check_words({pos}); st != MV_OK) return st;
  return hip_status(mv::launch_cache_write(d, layer, n_rows, slot, k, k_stride, v, v_stride, rope,
                                           pos, stream),
                    "cache write launch");
}

size_t mv_cache_compact_workspace_bytes(const mv_cache_shape* s, int32_t n) {
  if (check_cache_shape(s) != MV_OK || check_entries(n) != MV_OK) return 0;
  return mv::cache_move_ws_bytes(*s, n);
}

mv_status mv_cache_fork(const mv_cache_shape* s, const mv_cache* c, int32_t n, const int32_t* src,
                        const int32_t* dst, int32_t share, void* ws, size_t ws_bytes,
                        hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(s, c, &d); st != MV_OK) return st;
  if (mv_status st = check_entries(n); st != MV_OK) return st;
  if (n == 0) return MV_OK;
  if (mv_status st = check_words({src, dst}); st != MV_OK) return st;
  if (mv_status st = check_ptrs({ws}); st != MV_OK) return st;
  if (mv_status st = check_space("cache", ws_bytes, mv::cache_move_ws_bytes(*s, n)); st != MV_OK)
    return st;
  return hip_status(mv::launch_cache_move(*s, d, n, src, dst, nullptr, nullptr, 0, share != 0, ws,
                                          stream),
                    "cache fork launch");
}

mv_status mv_cache_compact(const mv_cache_shape* s, const mv_cache* c, int32_t n,
                           const int32_t* src, const int32_t* dst, const int32_t* span_ptr,
                           const mv_span* spans, int32_t n_spans, void* ws, size_t ws_bytes,
                           hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(s, c, &d); st != MV_OK) return st;
  if (mv_status st = check_entries(n); st != MV_OK) return st;
  if (n_spans < 0) return fail(MV_ERR_SHAPE, "n_spans must be >= 0");
  if (n == 0) return MV_OK;
  if (mv_status st = check_words({src, dst, span_ptr}); st != MV_OK) return st;
  if (n_spans > 0)
    if (mv_status st = check_words({spans}); st != MV_OK) return st;
  if (mv_status st = check_ptrs({ws}); st != MV_OK) return st;
  if (mv_status st = check_space("cache", ws_bytes, mv::cache_move_ws_bytes(*s, n)); st != MV_OK)
    return st;
  return hip_status(mv::launch_cache_move(*s, d, n, src, dst, span_ptr, spans, n_spans, true, ws,
                                          stream),
                    "cache compact launch");
}

mv_status mv_cache_free(const mv_cache_shape* s, const mv_cache* c, int32_t n,
                        const int32_t* seq_ids, hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(s, c, &d); st != MV_OK) return st;
  if (mv_status st = check_entries(n); st != MV_OK) return st;
  if (n == 0) return MV_OK;
  if (mv_status st = check_words({seq_ids}); st != MV_OK) return st;
  return hip_status(mv::launch_cache_free(d, n, seq_ids, stream), "cache free launch");
}

size_t mv_tree_attn_workspace_bytes(const mv_cache_shape* c, const mv_tree_attn_shape* s) {
  if (check_tree_shape(c, s) != MV_OK) return 0;
  return mv::tree_attn_ws_bytes(*c, *s);
}

mv_status mv_tree_attn(const mv_cache_shape* cs, const mv_cache* c, int32_t layer,
                       const mv_tree_attn_shape* s, const int32_t* seq_ids,
                       const int32_t* row_ptr, const uint32_t* tree, const void* q, void* o,
                       float* lse, void* ws, size_t ws_bytes, hipStream_t stream) {
  mv::CacheDev d;
  if (mv_status st = check_cache(cs, c, &d); st != MV_OK) return st;
  if (mv_status st = check_tree_shape(cs, s); st != MV_OK) return st;
  if (layer < 0 || layer >= cs->n_layers) return fail(MV_ERR_SHAPE, "layer outside the cache");
  if (s->n_batch == 0 || s->n_rows == 0) return MV_OK;
  if (mv_status st = check_words({seq_ids, row_ptr, lse}); st != MV_OK) return st;
  if (tree != nullptr) {
    if (mv_status st = check_words({tree}); st != MV_OK) return st;
    if (s->tree_words == 0) return fail(MV_ERR_SHAPE, "a tree of no words");
  }
  if (mv_status st = check_ptrs({q, o, ws}); st != MV_OK) return st;
  if (mv_status st = check_space("tree attention", ws_bytes, mv::tree_attn_ws_bytes(*cs, *s));
      st != MV_OK)
    return st;
  const float scale =
      s->softmax_scale > 0.f ? s->softmax_scale : 1.f / std::sqrt(float(cs->head_dim));
  return hip_status(mv::launch_tree_attn(*cs, d, layer, *s, scale, seq_ids, row_ptr, tree, q, o,
                                         lse, ws, stream),
                    "tree attention launch");
}

mv_status mv_tree_mask(int32_t n_batch, int32_t n_rows, const int32_t* row_ptr,
                       const int32_t* parent, int32_t words, uint32_t* tree, int32_t* depth,
                       hipStream_t stream) {
  if (mv_status st = check_entries(n_batch); st != MV_OK) return st;
  if (n_rows < 0 || words <= 0 || words > (1 << 20))
    return fail(MV_ERR_SHAPE, "n_rows >= 0 and 0 < words <= 2^20 required");
  if (n_batch == 0 || n_rows == 0) return MV_OK;
  if (mv_status st = check_words({row_ptr, parent, tree}); st != MV_OK) return st;
  if (depth != nullptr)
    if (mv_status st = check_words({depth}); st != MV_OK) return st;
  return hip_status(mv::launch_tree_mask(n_batch, n_rows, row_ptr, parent, words, tree, depth,
                                         stream),
                    "tree mask launch");
}

}  // extern "C"
