// C ABI of the paged cache: argument validation and kernel sequencing.  Host code only.
#include <math.h>
#include <string.h>

#include "paged.h"
#include "rotary.h"
#include "strided.h"

namespace dash {

// Validates p and fills a (sizes, strides).  rows: the call uses q, o and n_rows; fresh: k_new and v_new; four: a cache in 4 bits.
static int paged_args(const dash_paged_params* p, PagedArgs* a, bool rows, bool fresh, bool four = false) {
  if (!p) return DASH_EINVAL;
  if (p->batch < 1 || p->h_q < 1 || p->h_kv < 1 || p->n_pages < 1 || p->max_pages < 1 || p->page_size < 1 || p->head_dim < 1) return DASH_EINVAL;
  if (p->h_q % p->h_kv != 0 || (p->causal != 0 && p->causal != 1) || p->reserved != 0) return DASH_EINVAL;
  if (p->dtype != DASH_F32 && p->dtype != DASH_BF16) return DASH_EINVAL;
  if ((rows || fresh) && p->n_rows < 1) return DASH_EINVAL;
  if (!isfinite(p->scale)) return DASH_EINVAL;
  // 16 bytes of the packed rows, and of the pages; bytes of their elements, or of two codes
  const int vec = p->dtype == DASH_BF16 ? 8 : 4, page_vec = four ? 16 : vec, es = 16 / page_vec, d = p->head_dim, held = four ? d / 2 : d;
  const auto bad = [](const int64_t* s, int k, int vec) {
    for (int i = 0; i < k; i++)
      if (s[i] < 0 || s[i] % vec != 0) return true;
    return false;
  };
  if (bad(p->k_stride, 3, page_vec) || bad(p->v_stride, 3, page_vec) || p->k_stride[2] < held || p->v_stride[2] < held) return DASH_EINVAL;
  if (rows && (bad(p->q_stride, 2, vec) || bad(p->o_stride, 2, vec))) return DASH_EINVAL;
  if (fresh && (bad(p->k_new_stride, 2, vec) || bad(p->v_new_stride, 2, vec))) return DASH_EINVAL;
  if (d != 64 && d != 128) return DASH_EUNSUPPORTED;
  // offsets between the 16 rows of a tile are 32-bit numbers
  if (rows && (p->q_stride[0] > (1 << 25) || p->q_stride[1] > (1 << 25) || p->o_stride[0] > (1 << 25) || p->o_stride[1] > (1 << 25))) return DASH_EUNSUPPORTED;
  const int g = p->h_q / p->h_kv;
  if (g != 1 && g != 2 && g != 4 && g != 8 && g != 16) return DASH_EUNSUPPORTED;
  int log = 4;
  while (log < 10 && (1 << log) < p->page_size) log++;
  if ((1 << log) != p->page_size) return DASH_EUNSUPPORTED;
  if ((int64_t)p->max_pages * p->page_size > (1 << 24)) return DASH_EUNSUPPORTED;
  // offsets inside a page and the grids are 32-bit numbers
  const int64_t lim = (int64_t)1 << 31, span = p->page_size - 1;
  if (p->k_stride[2] >= lim / es / p->page_size || p->v_stride[2] >= lim / es / p->page_size ||
      (span * p->k_stride[2] + held) * es >= lim || (span * p->v_stride[2] + held) * es >= lim) return DASH_EUNSUPPORTED;
  if ((int64_t)p->batch * p->h_kv > (1 << 20) || (rows && (int64_t)p->n_rows * p->h_q > (1 << 28)) || p->n_rows > (1 << 28)) return DASH_EUNSUPPORTED;
  memset(a, 0, sizeof(*a));
  a->batch = p->batch; a->h_q = p->h_q; a->h_kv = p->h_kv; a->g = g;
  a->page_log = log; a->n_pages = p->n_pages; a->max_pages = p->max_pages; a->cap = p->max_pages * p->page_size;
  a->n_rows = p->n_rows; a->causal = p->causal;
  a->q_t = p->q_stride[0]; a->q_h = p->q_stride[1]; a->o_t = p->o_stride[0]; a->o_h = p->o_stride[1];
  a->kn_t = p->k_new_stride[0]; a->kn_h = p->k_new_stride[1]; a->vn_t = p->v_new_stride[0]; a->vn_h = p->v_new_stride[1];
  a->kp_p = p->k_stride[0]; a->kp_h = p->k_stride[1]; a->kp_t = p->k_stride[2];
  a->vp_p = p->v_stride[0]; a->vp_h = p->v_stride[1]; a->vp_t = p->v_stride[2];
  a->c1 = (float)((p->scale > 0.f ? (double)p->scale : 1.0 / sqrt((double)d)) * 1.4426950408889634);
  return DASH_OK;
}

static bool misaligned(const void* x) { return ((uintptr_t)x & 15) != 0; }
// Whether packed rows of heads that a call writes share elements among themselves.
static bool rows_repeat(const dash_paged_params* p, const PagedArgs& a, const void* o) {
  return strided_repeats({o, 2, {a.o_t, a.o_h}, {a.n_rows, a.h_q}}, p->head_dim);
}
// The turned queries of a call that appends: each in a place of its own, q's or apart from q, and apart from the new keys and values.
static bool queries_meet(const dash_paged_params* p, const PagedArgs& a) {
  if (!a.q) return false;
  const int es = p->dtype == DASH_BF16 ? 2 : 4;
  const auto rows = [&](const void* at, int64_t t, int64_t h, int heads) { return Strided{at, 2, {t, h}, {a.n_rows, heads}}; };
  const Strided out = rows(a.o, a.o_t, a.o_h, p->h_q);
  const auto meets = [&](const Strided& x) { return strided_meet(x, out, p->head_dim, es); };
  return rows_repeat(p, a, a.o) || (a.q == a.o ? a.q_t != a.o_t || a.q_h != a.o_h : meets(rows(a.q, a.q_t, a.q_h, p->h_q))) ||
         meets(rows(a.k_new, a.kn_t, a.kn_h, p->h_kv)) || meets(rows(a.v_new, a.vn_t, a.vn_h, p->h_kv));
}
static int check_scratch(size_t need, const void* ws, size_t bytes) {
  return (!ws || ((uintptr_t)ws & 255) != 0 || bytes < need) ? DASH_EWORKSPACE : DASH_OK;
}

}  // namespace dash

using namespace dash;

extern "C" {

int dash_paged_workspace_bytes(const dash_paged_params* p, size_t* out_bytes) {
  if (!out_bytes) return DASH_EINVAL;
  PagedArgs a;
  if (const int rc = paged_args(p, &a, true, false); rc != DASH_OK) return rc;
  const size_t x = paged_attend_ws(a, p->dtype, p->head_dim), y = paged_weigh_ws(a, p->dtype, p->head_dim);
  *out_bytes = x > y ? x : y;
  return DASH_OK;
}

int dash_paged_evict_workspace_bytes(const dash_paged_params* p, size_t* out_bytes) {
  if (!out_bytes) return DASH_EINVAL;
  PagedArgs a;
  if (const int rc = paged_args(p, &a, false, false); rc != DASH_OK) return rc;
  *out_bytes = paged_evict_ws(a);
  return DASH_OK;
}

int dash_paged_append(const dash_paged_params* p, const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                      const int32_t* row_start, const int32_t* lens, const int32_t* table, float* weights, int32_t* pos,
                      const int32_t* seen, void* stream) {
  PagedArgs a;
  if (const int rc = paged_args(p, &a, false, true); rc != DASH_OK) return rc;
  if (!k_new || !v_new || !k_pages || !v_pages || !row_start || !lens || !table) return DASH_EINVAL;
  if (misaligned(k_new) || misaligned(v_new) || misaligned(k_pages) || misaligned(v_pages)) return DASH_EINVAL;
  a.k_new = k_new; a.v_new = v_new; a.k = k_pages; a.v = v_pages;
  a.row_start = row_start; a.lens = lens; a.table = table; a.weights = weights; a.pos = pos; a.seen = seen;
  return launch_paged_append(a, p->dtype == DASH_BF16 ? 2 : 4, p->head_dim, (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

int dash_paged_attend(const dash_paged_params* p, const void* q, const void* k_pages, const void* v_pages,
                      const int32_t* row_start, const int32_t* lens, const int32_t* table, void* o, float* lse,
                      void* workspace, size_t workspace_bytes, void* stream) {
  PagedArgs a;
  if (const int rc = paged_args(p, &a, true, false); rc != DASH_OK) return rc;
  if (!q || !k_pages || !v_pages || !row_start || !lens || !table || !o) return DASH_EINVAL;
  if (misaligned(q) || misaligned(k_pages) || misaligned(v_pages) || misaligned(o)) return DASH_EINVAL;
  if (!paged_attend_fits(a, p->dtype)) return DASH_EUNSUPPORTED;
  if (rows_repeat(p, a, o)) return DASH_EINVAL;
  if (const int rc = check_scratch(paged_attend_ws(a, p->dtype, p->head_dim), workspace, workspace_bytes); rc != DASH_OK) return rc;
  a.q = q; a.k = (void*)k_pages; a.v = (void*)v_pages; a.o = o; a.lse = lse;
  a.row_start = row_start; a.lens = lens; a.table = table;
  return launch_paged_attend(a, p->dtype, p->head_dim, (char*)workspace, (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

int dash_paged_weigh(const dash_paged_params* p, const void* q, const void* k_pages, const int32_t* row_start,
                     const int32_t* lens, const int32_t* table, const float* lse, int32_t last, float* weights,
                     void* workspace, size_t workspace_bytes, void* stream) {
  PagedArgs a;
  if (const int rc = paged_args(p, &a, true, false); rc != DASH_OK) return rc;
  if (!q || !k_pages || !row_start || !lens || !table || !lse || !weights || last < 0) return DASH_EINVAL;
  if (misaligned(q) || misaligned(k_pages)) return DASH_EINVAL;
  if (const int rc = check_scratch(paged_weigh_ws(a, p->dtype, p->head_dim), workspace, workspace_bytes); rc != DASH_OK) return rc;
  a.q = q; a.k = (void*)k_pages; a.lse_in = lse; a.last = last; a.weights = weights;
  a.row_start = row_start; a.lens = lens; a.table = table;
  return launch_paged_weigh(a, p->dtype, p->head_dim, (char*)workspace, (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

int dash_paged_evict(const dash_paged_params* p, void* k_pages, void* v_pages, int32_t* lens, const int32_t* seen,
                     const int32_t* table, float* weights, int32_t* pos, int32_t budget, int32_t sinks, int32_t recent,
                     int32_t* src, void* workspace, size_t workspace_bytes, void* stream) {
  PagedArgs a;
  if (const int rc = paged_args(p, &a, false, false); rc != DASH_OK) return rc;
  if (!k_pages || !v_pages || !lens || !seen || !table || !weights || !pos) return DASH_EINVAL;
  if (misaligned(k_pages) || misaligned(v_pages)) return DASH_EINVAL;
  if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget) return DASH_EINVAL;
  if (const int rc = check_scratch(paged_evict_ws(a), workspace, workspace_bytes); rc != DASH_OK) return rc;
  a.k = k_pages; a.v = v_pages; a.lens = lens; a.seen = seen; a.table = table; a.weights = weights; a.pos = pos;
  return launch_paged_evict(a, p->dtype == DASH_BF16 ? 2 : 4, p->head_dim, lens, budget, sinks, recent, src, (char*)workspace,
                            (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

int dash_paged_append_rotary(const dash_paged_params* p, const dash_rotary* r, const void* q, void* q_out,
                             const void* k_new, const void* v_new, void* k_pages, void* v_pages, const int32_t* row_start,
                             const int32_t* lens, const int32_t* table, float* weights, int32_t* pos, const int32_t* seen, void* stream) {
  PagedArgs a;
  RotaryArgs turn;
  if (const int rc = paged_args(p, &a, q != nullptr, true); rc != DASH_OK) return rc;
  if (const int rc = rotary_args(r, p->head_dim, &turn); rc != DASH_OK) return rc;
  if (!q != !q_out || !k_new || !v_new || !k_pages || !v_pages || !row_start || !lens || !table) return DASH_EINVAL;
  if (misaligned(q) || misaligned(q_out) || misaligned(k_new) || misaligned(v_new) || misaligned(k_pages) || misaligned(v_pages)) return DASH_EINVAL;
  a.q = q; a.o = q_out; a.k_new = k_new; a.v_new = v_new; a.k = k_pages; a.v = v_pages;
  if (queries_meet(p, a)) return DASH_EINVAL;
  a.row_start = row_start; a.lens = lens; a.table = table; a.weights = weights; a.pos = pos; a.seen = seen;
  return launch_paged_append_rotary(a, turn, p->dtype == DASH_BF16 ? 2 : 4, p->head_dim, (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

int dash_paged4_workspace_bytes(const dash_paged_params* p, size_t* out_bytes) {
  if (!out_bytes) return DASH_EINVAL;
  PagedArgs a;
  if (const int rc = paged_args(p, &a, true, false, true); rc != DASH_OK) return rc;
  *out_bytes = paged4_attend_ws(a, p->dtype, p->head_dim);
  return DASH_OK;
}

int dash_paged4_append(const dash_paged_params* p, const dash_rotary* r, const void* q, void* q_out, const void* k_new,
                       const void* v_new, void* k_codes, void* k_scales, void* v_codes, void* v_scales, const int32_t* row_start,
                       const int32_t* lens, const int32_t* table, const int32_t* seen, void* stream) {
  PagedArgs a;
  RotaryArgs turn;
  if (const int rc = paged_args(p, &a, q != nullptr, true, true); rc != DASH_OK) return rc;
  if (r)
    if (const int rc = rotary_args(r, p->head_dim, &turn); rc != DASH_OK) return rc;
  if (!q != !q_out || (q && !r) || !k_new || !v_new || !k_codes || !k_scales || !v_codes || !v_scales || !row_start || !lens || !table) return DASH_EINVAL;
  if (misaligned(q) || misaligned(q_out) || misaligned(k_new) || misaligned(v_new) || misaligned(k_codes) || misaligned(v_codes) ||
      misaligned(k_scales) || misaligned(v_scales)) return DASH_EINVAL;
  a.q = q; a.o = q_out; a.k_new = k_new; a.v_new = v_new; a.k = k_codes; a.v = v_codes; a.k_sc = (const uint8_t*)k_scales; a.v_sc = (const uint8_t*)v_scales;
  if (queries_meet(p, a)) return DASH_EINVAL;
  a.row_start = row_start; a.lens = lens; a.table = table; a.seen = seen;
  return launch_paged4_append(a, r ? &turn : nullptr, p->dtype == DASH_BF16 ? 2 : 4, p->head_dim, (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

int dash_paged4_attend(const dash_paged_params* p, const void* q, const void* k_codes, const void* k_scales, const void* v_codes,
                       const void* v_scales, const int32_t* row_start, const int32_t* lens, const int32_t* table, void* o, float* lse,
                       void* workspace, size_t workspace_bytes, void* stream) {
  PagedArgs a;
  if (const int rc = paged_args(p, &a, true, false, true); rc != DASH_OK) return rc;
  if (!q || !k_codes || !k_scales || !v_codes || !v_scales || !row_start || !lens || !table || !o) return DASH_EINVAL;
  if (misaligned(q) || misaligned(k_codes) || misaligned(v_codes) || misaligned(k_scales) || misaligned(v_scales) || misaligned(o)) return DASH_EINVAL;
  if (!paged4_attend_fits(a, p->dtype)) return DASH_EUNSUPPORTED;
  if (rows_repeat(p, a, o)) return DASH_EINVAL;
  if (const int rc = check_scratch(paged4_attend_ws(a, p->dtype, p->head_dim), workspace, workspace_bytes); rc != DASH_OK) return rc;
  a.q = q; a.k = (void*)k_codes; a.v = (void*)v_codes; a.k_sc = (const uint8_t*)k_scales; a.v_sc = (const uint8_t*)v_scales; a.o = o; a.lse = lse;
  a.row_start = row_start; a.lens = lens; a.table = table;
  return launch_paged4_attend(a, p->dtype, p->head_dim, (char*)workspace, (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

int dash_paged4_unpack(const dash_paged_params* p, const void* k_codes, const void* k_scales, const void* v_codes,
                       const void* v_scales, void* k_pages, void* v_pages, void* stream) {
  PagedArgs a;
  if (const int rc = paged_args(p, &a, false, false, true); rc != DASH_OK) return rc;
  if (!k_codes || !k_scales || !v_codes || !v_scales || !k_pages || !v_pages) return DASH_EINVAL;
  if ((int64_t)p->n_pages * p->h_kv > 1 << 30) return DASH_EUNSUPPORTED;   // heads of pages are counted in 32 bits
  if (misaligned(k_codes) || misaligned(v_codes) || misaligned(k_scales) || misaligned(v_scales) || misaligned(k_pages) || misaligned(v_pages)) return DASH_EINVAL;
  a.k = (void*)k_codes; a.v = (void*)v_codes; a.k_sc = (const uint8_t*)k_scales; a.v_sc = (const uint8_t*)v_scales;
  return launch_paged4_unpack(a, k_pages, v_pages, p->dtype == DASH_BF16 ? 2 : 4, p->head_dim, (hipStream_t)stream) == hipSuccess ? DASH_OK : DASH_ELAUNCH;
}

}  // extern "C"
