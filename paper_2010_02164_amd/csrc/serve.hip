// C entry points of the serving operators: the checks of their arguments on
// the host, before anything is enqueued.
#include <math.h>
#include <stdio.h>

#include <initializer_list>

#include "serve.h"

using namespace sb;

namespace {

sb_status refuse(sb_status s, const char *call, const char *why) {
  char text[200];
  snprintf(text, sizeof text, "%s: %s", call, why);
  set_call_error(text);
  return s;
}

sb_status launched(hipError_t e, const char *call) {
  return e == hipSuccess ? SB_OK : refuse(SB_E_HIP, call, hipGetErrorString(e));
}

// Compute units of the current device, asked for once per device.
hipError_t compute_units(int &n) {
  static int known[64];   // 0: not asked yet (threads that ask at once write the same)
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 64 && __atomic_load_n(&known[dev], __ATOMIC_RELAXED) > 0) {
    n = __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
    return hipSuccess;
  }
  const hipError_t e2 = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev);
  if (e2 == hipSuccess && dev < 64) __atomic_store_n(&known[dev], n, __ATOMIC_RELAXED);
  return e2;
}

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// 16-byte loads of rows: strides that keep every row's address a multiple. One
// that has a single place is never stepped along, and may be anything.
struct Stride {
  int64_t step, places;
};
bool strides_fit(std::initializer_list<Stride> all) {
  for (const Stride &s : all)
    if (s.places > 1 && (s.step < 0 || s.step % 8)) return false;
  return true;
}

#define REFUSE_IF(cond, status, why) \
  if (cond) return refuse(status, call, why)

sb_status check_attention(const sb_attention_args *a, const char *call, bool pointers) {
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a), SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "dtype is not SB_BF16 or SB_F16");
  REFUSE_IF(a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256, SB_E_UNSUPPORTED, "head_dim is not 64, 128 or 256");
  REFUSE_IF(a->n_tokens < 0 || a->n_requests < 1, SB_E_INVALID_ARG, "n_tokens < 0 or n_requests < 1");
  REFUSE_IF(a->kv_heads < 1 || a->kv_heads > 1024 || a->q_heads < 1 || a->q_heads > 1024 || a->q_heads % a->kv_heads,
            SB_E_INVALID_ARG, "q_heads is not a multiple of kv_heads, or outside 1 .. 1024");
  REFUSE_IF(a->n_pages < 1 || a->page_size < 1 || a->page_size > 4096 || a->max_pages < 1, SB_E_INVALID_ARG,
            "n_pages, max_pages < 1 or page_size outside 1 .. 4096");
  REFUSE_IF((int64_t)a->n_pages * a->page_size > INT32_MAX || (int64_t)a->max_pages * a->page_size > INT32_MAX,
            SB_E_UNSUPPORTED, "n_pages or max_pages times page_size is not below 2^31");
  // The kernels look a few tiles of keys behind a request's last one, in 32 bits.
  REFUSE_IF((int64_t)a->max_pages * a->page_size > SB_ATTENTION_MAX_KEYS, SB_E_UNSUPPORTED,
            "max_pages times page_size is above SB_ATTENTION_MAX_KEYS");
  REFUSE_IF((int64_t)a->n_tokens * a->q_heads > INT32_MAX, SB_E_UNSUPPORTED, "n_tokens times q_heads is not below 2^31");
  REFUSE_IF(a->window < 0 || a->sinks < 0 || a->max_q < 0 || a->max_kv < 0, SB_E_INVALID_ARG,
            "window, sinks, max_q or max_kv < 0");
  REFUSE_IF(!isfinite((float)(a->scale * 1.4426950408889634)), SB_E_INVALID_ARG, "scale, in powers of two, is not finite");
  REFUSE_IF(a->table_stride < a->max_pages, SB_E_INVALID_ARG, "table_stride < max_pages");
  REFUSE_IF(!strides_fit({{a->q_token, a->n_tokens}, {a->q_head, a->q_heads}, {a->out_token, a->n_tokens}, {a->out_head, a->q_heads},
                          {a->kc_page, a->n_pages}, {a->kc_slot, a->page_size}, {a->kc_head, a->kv_heads}, {a->vc_page, a->n_pages},
                          {a->vc_slot, a->page_size}, {a->vc_head, a->kv_heads}}),
            SB_E_UNSUPPORTED, "a stride is negative or no multiple of 8");
  if (!pointers) return SB_OK;
  REFUSE_IF(!a->table || !a->lens || !a->q_start || !a->k_cache || !a->v_cache || (a->n_tokens && (!a->q || !a->out)),
            SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->q, 16) || !aligned(a->k_cache, 16) || !aligned(a->v_cache, 16) || !aligned(a->out, 16) ||
                !aligned(a->table, 4) || !aligned(a->lens, 4) || !aligned(a->q_start, 4),
            SB_E_UNSUPPORTED, "q, out or the caches are not 16-byte aligned");
  return SB_OK;
}

sb_status check_shared(const sb_shared_args *x, const char *call, bool pointers) {
  REFUSE_IF(!x, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(x->struct_bytes != (int64_t)sizeof(*x) || x->reserved, SB_E_INVALID_ARG, "struct_bytes is not this library's");
  const sb_status st = check_attention(&x->own, call, pointers);
  if (st != SB_OK) return st;
  const sb_attention_args *a = &x->own;
  REFUSE_IF(a->window || a->sinks, SB_E_INVALID_ARG, "window or sinks is not 0");
  REFUSE_IF(x->n_groups < 1 || x->prefix_pages < 1 || x->max_prefix < 0, SB_E_INVALID_ARG, "n_groups, prefix_pages < 1 or max_prefix < 0");
  REFUSE_IF((int64_t)x->prefix_pages * a->page_size > SB_ATTENTION_MAX_KEYS, SB_E_UNSUPPORTED,
            "prefix_pages times page_size is above SB_ATTENTION_MAX_KEYS");
  REFUSE_IF(x->prefix_stride < x->prefix_pages, SB_E_INVALID_ARG, "prefix_stride < prefix_pages");
  REFUSE_IF((int64_t)a->n_tokens * a->q_heads / 8 + ((int64_t)x->n_groups + a->n_requests) * a->kv_heads > (1 << 23), SB_E_UNSUPPORTED,
            "n_tokens times q_heads / 8 and groups and requests times kv_heads are more than 2^23");
  if (!pointers) return SB_OK;
  REFUSE_IF(!x->prefix_table || !x->prefix_lens || !x->group_start, SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(x->prefix_table, 4) || !aligned(x->prefix_lens, 4) || !aligned(x->group_start, 4), SB_E_INVALID_ARG,
            "an array is not aligned to its type");
  return SB_OK;
}

sb_status check_select(const sb_select_args *a, const char *call) {
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a) || a->reserved, SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "dtype is not SB_BF16 or SB_F16");
  REFUSE_IF(a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256, SB_E_UNSUPPORTED, "head_dim is not 64, 128 or 256");
  REFUSE_IF(a->n_tokens < 0 || a->n_requests < 1, SB_E_INVALID_ARG, "n_tokens < 0 or n_requests < 1");
  REFUSE_IF(a->kv_heads < 1 || a->kv_heads > 1024 || a->q_heads < 1 || a->q_heads > 1024 || a->q_heads % a->kv_heads,
            SB_E_INVALID_ARG, "q_heads is not a multiple of kv_heads, or outside 1 .. 1024");
  REFUSE_IF(a->n_pages < 1 || a->page_size < 1 || a->page_size > 4096 || a->max_pages < 1, SB_E_INVALID_ARG,
            "n_pages, max_pages < 1 or page_size outside 1 .. 4096");
  REFUSE_IF(a->top < 0 || a->first < 0 || a->last < 1 || a->max_kv < 0, SB_E_INVALID_ARG, "top, first or max_kv < 0, or last < 1");
  REFUSE_IF(((int64_t)a->top + a->first + a->last) * a->page_size > SB_ATTENTION_MAX_KEYS ||
                (int64_t)a->max_pages * a->page_size > SB_ATTENTION_MAX_KEYS || (int64_t)a->n_pages * a->page_size > INT32_MAX,
            SB_E_UNSUPPORTED, "pages (of the cache, a table's row, or selected) times page_size are above SB_ATTENTION_MAX_KEYS");
  REFUSE_IF(a->table_stride < a->max_pages, SB_E_INVALID_ARG, "table_stride < max_pages");
  REFUSE_IF(!strides_fit({{a->q_token, a->n_tokens}, {a->q_head, a->q_heads}}), SB_E_UNSUPPORTED, "a stride is negative or no multiple of 8");
  return SB_OK;
}

sb_status check_selected(const sb_selected_args *a, const char *call) {
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a) || a->reserved, SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "dtype is not SB_BF16 or SB_F16");
  REFUSE_IF(a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256, SB_E_UNSUPPORTED, "head_dim is not 64, 128 or 256");
  REFUSE_IF(a->n_tokens < 0, SB_E_INVALID_ARG, "n_tokens < 0");
  REFUSE_IF(a->kv_heads < 1 || a->kv_heads > 1024 || a->q_heads < 1 || a->q_heads > 1024 || a->q_heads % a->kv_heads,
            SB_E_INVALID_ARG, "q_heads is not a multiple of kv_heads, or outside 1 .. 1024");
  REFUSE_IF(a->n_pages < 1 || a->page_size < 1 || a->page_size > 4096 || a->width < 1, SB_E_INVALID_ARG,
            "n_pages, width < 1 or page_size outside 1 .. 4096");
  REFUSE_IF((int64_t)a->n_pages * a->page_size > INT32_MAX || (int64_t)a->width * a->page_size > SB_ATTENTION_MAX_KEYS, SB_E_UNSUPPORTED,
            "n_pages times page_size is not below 2^31, or width times page_size above SB_ATTENTION_MAX_KEYS");
  REFUSE_IF((int64_t)a->n_tokens * a->q_heads > (1 << 23), SB_E_UNSUPPORTED, "n_tokens times q_heads is above 2^23");
  REFUSE_IF(!isfinite((float)(a->scale * 1.4426950408889634)), SB_E_INVALID_ARG, "scale, in powers of two, is not finite");
  REFUSE_IF(!strides_fit({{a->q_token, a->n_tokens}, {a->q_head, a->q_heads}, {a->out_token, a->n_tokens}, {a->out_head, a->q_heads},
                          {a->kc_page, a->n_pages}, {a->kc_slot, a->page_size}, {a->kc_head, a->kv_heads}, {a->vc_page, a->n_pages},
                          {a->vc_slot, a->page_size}, {a->vc_head, a->kv_heads}}),
            SB_E_UNSUPPORTED, "a stride is negative or no multiple of 8");
  return SB_OK;
}

sb_status check_sample(const sb_sample_args *a, const char *call) {
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a) || a->reserved, SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_F32 && a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "unknown dtype");
  REFUSE_IF(a->rows < 0 || a->vocab < 1, SB_E_INVALID_ARG, "rows < 0 or vocab < 1");
  REFUSE_IF(a->vocab > SB_SAMPLE_MAX_VOCAB, SB_E_UNSUPPORTED, "vocab above SB_SAMPLE_MAX_VOCAB");
  REFUSE_IF(a->row_stride < 0 || (a->rows > 1 && a->row_stride < a->vocab), SB_E_INVALID_ARG, "row_stride < vocab");
  return SB_OK;
}

sb_status check_linear(const sb_linear_args *a, const char *call) {
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a), SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_F32 && a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "unknown dtype");
  REFUSE_IF(a->rows < 0 || a->channels < 1 || a->depth < 1, SB_E_INVALID_ARG, "rows < 0, channels < 1 or depth < 1");
  REFUSE_IF(a->rows > SB_LINEAR_MAX_ROWS || a->channels > SB_LINEAR_MAX_ROWS || a->depth > SB_LINEAR_MAX_DEPTH, SB_E_UNSUPPORTED,
            "rows or channels above SB_LINEAR_MAX_ROWS, or depth above SB_LINEAR_MAX_DEPTH");
  REFUSE_IF(a->depth % 16, SB_E_UNSUPPORTED, "depth is no multiple of 16");
  REFUSE_IF((a->rows > 1 && (a->x_row < a->depth || a->out_row < a->channels)) || (a->channels > 1 && a->w_row < a->depth),
            SB_E_INVALID_ARG, "rows of x, w or out overlap");
  REFUSE_IF((a->rows > 1 && a->x_row % 16) || (a->channels > 1 && a->w_row % 16), SB_E_UNSUPPORTED, "a row stride is no multiple of 16");
  return SB_OK;
}

}  // namespace

extern "C" {

sb_status sb_plan_pages(const sb_plan_args *a, void *stream) {
  const char *call = "sb_plan_pages";
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a) || a->reserved, SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->n_requests < 1, SB_E_INVALID_ARG, "n_requests < 1");
  REFUSE_IF(a->n_requests > SB_PLAN_MAX_REQUESTS, SB_E_UNSUPPORTED, "more than SB_PLAN_MAX_REQUESTS requests");
  REFUSE_IF(a->n_pages < 1 || a->page_size < 1 || a->page_size > 4096 || a->max_pages < 1 || a->token_cap < 0,
            SB_E_INVALID_ARG, "n_pages, max_pages < 1, token_cap < 0 or page_size outside 1 .. 4096");
  REFUSE_IF((int64_t)a->n_pages * a->page_size > INT32_MAX || (int64_t)a->max_pages * a->page_size > INT32_MAX,
            SB_E_UNSUPPORTED, "n_pages or max_pages times page_size is not below 2^31");
  REFUSE_IF(a->table_stride < a->max_pages, SB_E_INVALID_ARG, "table_stride < max_pages");
  REFUSE_IF(!a->lens || !a->add || !a->n_free || !a->free_list || !a->table || !a->lens_out || !a->n_free_out || !a->q_start ||
                !a->granted || (a->token_cap && (!a->slots || !a->positions)),
            SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->lens, 4) || !aligned(a->add, 4) || !aligned(a->n_free, 4) || !aligned(a->free_list, 4) ||
                !aligned(a->table, 4) || !aligned(a->lens_out, 4) || !aligned(a->n_free_out, 4) || !aligned(a->q_start, 4) ||
                !aligned(a->granted, 4) || !aligned(a->slots, 8) || !aligned(a->positions, 4),
            SB_E_INVALID_ARG, "an array is not aligned to its type");
  return launched(launch_plan(*a, static_cast<hipStream_t>(stream)), call);
}

sb_status sb_rope_append(const sb_rope_args *a, void *stream) {
  const char *call = "sb_rope_append";
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a), SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "dtype is not SB_BF16 or SB_F16");
  REFUSE_IF(a->layout != SB_ROPE_HALF && a->layout != SB_ROPE_INTERLEAVED, SB_E_INVALID_ARG, "unknown layout");
  REFUSE_IF(a->n_tokens < 0, SB_E_INVALID_ARG, "n_tokens < 0");
  REFUSE_IF(a->kv_heads < 1 || a->kv_heads > 1024 || a->q_heads < 1 || a->q_heads > 1024, SB_E_INVALID_ARG,
            "q_heads or kv_heads outside 1 .. 1024");
  REFUSE_IF(a->head_dim < 8 || a->head_dim > 512 || a->head_dim % 8, SB_E_UNSUPPORTED, "head_dim is no multiple of 8 up to 512");
  REFUSE_IF(a->n_pairs < 0 || 2 * (int64_t)a->n_pairs > a->head_dim, SB_E_INVALID_ARG, "2 n_pairs is not within the head");
  REFUSE_IF(a->n_pairs % (a->layout == SB_ROPE_HALF ? 8 : 4), SB_E_UNSUPPORTED,
            "n_pairs is no multiple of 8 (half) or 4 (interleaved)");
  REFUSE_IF(a->n_pages < 1 || a->page_size < 1 || a->page_size > 4096, SB_E_INVALID_ARG, "n_pages < 1 or page_size outside 1 .. 4096");
  REFUSE_IF((int64_t)a->n_pages * a->page_size > INT32_MAX, SB_E_UNSUPPORTED, "n_pages times page_size is not below 2^31");
  REFUSE_IF(!isfinite(a->mscale), SB_E_INVALID_ARG, "mscale is not finite");
  REFUSE_IF(!strides_fit({{a->q_token, a->n_tokens}, {a->q_head, a->q_heads}, {a->k_token, a->n_tokens}, {a->k_head, a->kv_heads},
                          {a->v_token, a->n_tokens}, {a->v_head, a->kv_heads}, {a->out_token, a->n_tokens}, {a->out_head, a->q_heads},
                          {a->kc_page, a->n_pages}, {a->kc_slot, a->page_size}, {a->kc_head, a->kv_heads}, {a->vc_page, a->n_pages},
                          {a->vc_slot, a->page_size}, {a->vc_head, a->kv_heads}}),
            SB_E_UNSUPPORTED, "a stride is negative or no multiple of 8");
  if (a->n_tokens == 0) return SB_OK;
  REFUSE_IF(!a->q || !a->k || !a->v || !a->q_out || !a->k_cache || !a->v_cache || !a->positions || !a->slots ||
                (a->n_pairs && !a->inv_freq),
            SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->q_out, 16) || !aligned(a->k_cache, 16) ||
                !aligned(a->v_cache, 16) || !aligned(a->positions, 4) || !aligned(a->slots, 8) || !aligned(a->inv_freq, 8),
            SB_E_UNSUPPORTED, "q, k, v, q_out or the caches are not 16-byte aligned");
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) return launched(e, call);
  return launched(launch_rope(*a, n_cu, static_cast<hipStream_t>(stream)), call);
}

int64_t sb_attention_workspace(const sb_attention_args *a) {
  if (check_attention(a, "sb_attention_workspace", false) != SB_OK) return -1;
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) {
    launched(e, "sb_attention_workspace");
    return -1;
  }
  return attention_workspace(*a, n_cu);
}

sb_status sb_paged_attention(const sb_attention_args *a, void *workspace, size_t bytes, void *stream) {
  const char *call = "sb_paged_attention";
  const sb_status st = check_attention(a, call, true);
  if (st != SB_OK) return st;
  if (a->n_tokens == 0) return SB_OK;
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) return launched(e, call);
  const int64_t need = attention_workspace(*a, n_cu);
  REFUSE_IF(need && (!workspace || !aligned(workspace, 256) || bytes < (size_t)need), SB_E_WORKSPACE,
            "workspace missing, misaligned or smaller than sb_attention_workspace");
  return launched(launch_paged_attention(*a, n_cu, workspace, static_cast<hipStream_t>(stream)), call);
}

int64_t sb_shared_workspace(const sb_shared_args *a) {
  const char *call = "sb_shared_workspace";
  if (check_shared(a, call, false) != SB_OK) return -1;
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) {
    launched(e, call);
    return -1;
  }
  return shared_workspace(*a, n_cu);
}

sb_status sb_shared_attention(const sb_shared_args *a, void *workspace, size_t bytes, void *stream) {
  const char *call = "sb_shared_attention";
  const sb_status st = check_shared(a, call, true);
  if (st != SB_OK) return st;
  if (a->own.n_tokens == 0) return SB_OK;
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) return launched(e, call);
  REFUSE_IF(!workspace || !aligned(workspace, 256) || bytes < (size_t)shared_workspace(*a, n_cu), SB_E_WORKSPACE,
            "workspace missing, misaligned or smaller than sb_shared_workspace");
  return launched(launch_shared_attention(*a, n_cu, workspace, static_cast<hipStream_t>(stream)), call);
}

sb_status sb_page_bounds(const sb_bounds_args *a, void *stream) {
  const char *call = "sb_page_bounds";
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a), SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "dtype is not SB_BF16 or SB_F16");
  REFUSE_IF(a->head_dim != 64 && a->head_dim != 128 && a->head_dim != 256, SB_E_UNSUPPORTED, "head_dim is not 64, 128 or 256");
  REFUSE_IF(a->n_requests < 1 || a->kv_heads < 1 || a->kv_heads > 1024 || a->max_q < 0, SB_E_INVALID_ARG,
            "n_requests < 1, kv_heads outside 1 .. 1024 or max_q < 0");
  REFUSE_IF(a->n_requests > (1 << 23), SB_E_UNSUPPORTED, "more than 2^23 requests");
  REFUSE_IF(a->n_pages < 1 || a->page_size < 1 || a->page_size > 4096 || a->max_pages < 1, SB_E_INVALID_ARG,
            "n_pages, max_pages < 1 or page_size outside 1 .. 4096");
  REFUSE_IF((int64_t)a->n_pages * a->page_size > INT32_MAX || (int64_t)a->max_pages * a->page_size > INT32_MAX, SB_E_UNSUPPORTED,
            "n_pages or max_pages times page_size is not below 2^31");
  REFUSE_IF(a->table_stride < a->max_pages, SB_E_INVALID_ARG, "table_stride < max_pages");
  REFUSE_IF(!strides_fit({{a->kc_page, a->n_pages}, {a->kc_slot, a->page_size}, {a->kc_head, a->kv_heads}}), SB_E_UNSUPPORTED,
            "a stride is negative or no multiple of 8");
  REFUSE_IF(!a->k_cache || !a->table || !a->lens || !a->q_start || !a->bounds, SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->table, 4) || !aligned(a->lens, 4) || !aligned(a->q_start, 4), SB_E_INVALID_ARG, "an array is not aligned to its type");
  REFUSE_IF(!aligned(a->k_cache, 16) || !aligned(a->bounds, 16), SB_E_UNSUPPORTED, "k_cache or bounds is not 16-byte aligned");
  return launched(launch_bounds(*a, static_cast<hipStream_t>(stream)), call);
}

int64_t sb_select_workspace(const sb_select_args *a) {
  return check_select(a, "sb_select_workspace") == SB_OK ? (a->n_tokens ? select_workspace(*a) : 0) : -1;
}

sb_status sb_select_pages(const sb_select_args *a, void *workspace, size_t bytes, void *stream) {
  const char *call = "sb_select_pages";
  const sb_status st = check_select(a, call);
  if (st != SB_OK) return st;
  if (a->n_tokens == 0) return SB_OK;
  REFUSE_IF(!a->q || !a->bounds || !a->table || !a->lens || !a->q_start || !a->pages || !a->kept, SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->table, 4) || !aligned(a->lens, 4) || !aligned(a->q_start, 4) || !aligned(a->pages, 4) || !aligned(a->kept, 4),
            SB_E_INVALID_ARG, "an array is not aligned to its type");
  REFUSE_IF(!aligned(a->q, 16) || !aligned(a->bounds, 16), SB_E_UNSUPPORTED, "q or bounds is not 16-byte aligned");
  REFUSE_IF(!workspace || !aligned(workspace, 256) || bytes < (size_t)select_workspace(*a), SB_E_WORKSPACE,
            "workspace missing, misaligned or smaller than sb_select_workspace");
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) return launched(e, call);
  return launched(launch_select(*a, n_cu, workspace, static_cast<hipStream_t>(stream)), call);
}

int64_t sb_selected_workspace(const sb_selected_args *a) {
  const char *call = "sb_selected_workspace";
  if (check_selected(a, call) != SB_OK) return -1;
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) {
    launched(e, call);
    return -1;
  }
  return selected_workspace(*a, n_cu);
}

sb_status sb_selected_attention(const sb_selected_args *a, void *workspace, size_t bytes, void *stream) {
  const char *call = "sb_selected_attention";
  const sb_status st = check_selected(a, call);
  if (st != SB_OK) return st;
  if (a->n_tokens == 0) return SB_OK;
  REFUSE_IF(!a->q || !a->k_cache || !a->v_cache || !a->pages || !a->kept || !a->out, SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->pages, 4) || !aligned(a->kept, 4), SB_E_INVALID_ARG, "an array is not aligned to its type");
  REFUSE_IF(!aligned(a->q, 16) || !aligned(a->k_cache, 16) || !aligned(a->v_cache, 16) || !aligned(a->out, 16), SB_E_UNSUPPORTED,
            "q, out or the caches are not 16-byte aligned");
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) return launched(e, call);
  const int64_t need = selected_workspace(*a, n_cu);
  REFUSE_IF(need && (!workspace || !aligned(workspace, 256) || bytes < (size_t)need), SB_E_WORKSPACE,
            "workspace missing, misaligned or smaller than sb_selected_workspace");
  return launched(launch_selected_attention(*a, n_cu, workspace, static_cast<hipStream_t>(stream)), call);
}

int64_t sb_sample_workspace(const sb_sample_args *a) {
  return check_sample(a, "sb_sample_workspace") == SB_OK ? sample_workspace(*a) : -1;
}

sb_status sb_sample_tokens(const sb_sample_args *a, void *workspace, size_t bytes, void *stream) {
  const char *call = "sb_sample_tokens";
  const sb_status st = check_sample(a, call);
  if (st != SB_OK) return st;
  if (a->rows == 0) return SB_OK;
  REFUSE_IF(!a->logits || !a->u || !a->tokens, SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->logits, a->dtype == SB_F32 ? 4 : 2) || !aligned(a->u, 4) || !aligned(a->temperature, 4) ||
                !aligned(a->top_k, 4) || !aligned(a->top_p, 4) || !aligned(a->min_p, 4) || !aligned(a->tokens, 4) ||
                !aligned(a->logprobs, 4),
            SB_E_INVALID_ARG, "an array is not aligned to its type");
  const int64_t need = sample_workspace(*a);
  REFUSE_IF(workspace && need && (!aligned(workspace, 256) || bytes < (size_t)need), SB_E_WORKSPACE,
            "workspace misaligned or smaller than sb_sample_workspace");
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) return launched(e, call);
  return launched(launch_sample(*a, need ? workspace : nullptr, n_cu, static_cast<hipStream_t>(stream)), call);
}

sb_status sb_quantize_rows(const sb_quantize_args *a, void *stream) {
  const char *call = "sb_quantize_rows";
  REFUSE_IF(!a, SB_E_INVALID_ARG, "no arguments");
  REFUSE_IF(a->struct_bytes != (int64_t)sizeof(*a) || a->reserved, SB_E_INVALID_ARG, "struct_bytes is not this library's");
  REFUSE_IF(a->dtype != SB_F32 && a->dtype != SB_BF16 && a->dtype != SB_F16, SB_E_UNSUPPORTED, "unknown dtype");
  REFUSE_IF(a->rows < 0 || a->cols < 1, SB_E_INVALID_ARG, "rows < 0 or cols < 1");
  REFUSE_IF(a->rows > SB_LINEAR_MAX_ROWS || a->cols > SB_LINEAR_MAX_DEPTH, SB_E_UNSUPPORTED,
            "rows above SB_LINEAR_MAX_ROWS or cols above SB_LINEAR_MAX_DEPTH");
  REFUSE_IF(a->rows > 1 && a->x_row < 0, SB_E_INVALID_ARG, "x_row < 0");
  REFUSE_IF(a->rows > 1 && a->codes_row < (a->cols + 15) / 16 * 16, SB_E_INVALID_ARG, "codes_row < cols rounded up to 16");
  REFUSE_IF(a->rows > 1 && a->codes_row % 16, SB_E_UNSUPPORTED, "codes_row is no multiple of 16");
  if (a->rows == 0) return SB_OK;
  REFUSE_IF(!a->x || !a->codes || !a->scales, SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->x, a->dtype == SB_F32 ? 4 : 2) || !aligned(a->scales, 4), SB_E_INVALID_ARG, "an array is not aligned to its type");
  REFUSE_IF(!aligned(a->codes, 16), SB_E_UNSUPPORTED, "codes are not 16-byte aligned");
  return launched(launch_quantize(*a, static_cast<hipStream_t>(stream)), call);
}

int64_t sb_linear_workspace(const sb_linear_args *a) {
  const char *call = "sb_linear_workspace";
  if (check_linear(a, call) != SB_OK) return -1;
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) {
    launched(e, call);
    return -1;
  }
  return linear_workspace(*a, n_cu);
}

sb_status sb_quantized_linear(const sb_linear_args *a, void *workspace, size_t bytes, void *stream) {
  const char *call = "sb_quantized_linear";
  const sb_status st = check_linear(a, call);
  if (st != SB_OK) return st;
  if (a->rows == 0) return SB_OK;
  REFUSE_IF(!a->x || !a->w || !a->x_scale || !a->w_scale || !a->out, SB_E_INVALID_ARG, "a pointer is missing");
  REFUSE_IF(!aligned(a->x_scale, 4) || !aligned(a->w_scale, 4) || !aligned(a->bias, 4) || !aligned(a->out, a->dtype == SB_F32 ? 4 : 2),
            SB_E_INVALID_ARG, "an array is not aligned to its type");
  REFUSE_IF(!aligned(a->x, 16) || !aligned(a->w, 16), SB_E_UNSUPPORTED, "x or w is not 16-byte aligned");
  int n_cu = 0;
  const hipError_t e = compute_units(n_cu);
  if (e != hipSuccess) return launched(e, call);
  const int64_t need = linear_workspace(*a, n_cu);
  REFUSE_IF(need && (!workspace || !aligned(workspace, 256) || bytes < (size_t)need), SB_E_WORKSPACE,
            "workspace missing, misaligned or smaller than sb_linear_workspace");
  return launched(launch_linear(*a, n_cu, workspace, static_cast<hipStream_t>(stream)), call);
}

}  // extern "C"
