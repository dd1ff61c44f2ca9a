// C-ABI front end of the rotary positions and the paged cache: argument checks (host only, before any launch) and dispatch.
#include "../../include/attn.h"
#include "attn_paged.h"

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>

static_assert(sizeof(attn_rotary_spec) == 24 && sizeof(attn_rotary_tensor) == 72 && sizeof(attn_rotary_params) == 72 && sizeof(attn_paged_params) == 176 &&
                  sizeof(attn_paged_copy_params) == 64,
              "the parameter blocks' layout is part of the ABI");
static_assert(sizeof(attn_norm_spec) == 24 && sizeof(attn_norm_grad) == 112, "the parameter blocks' layout is part of the ABI");

namespace {

bool head_dim_ok(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }
bool dtype_ok(int t) { return t == ATTN_FP16 || t == ATTN_BF16; }
bool aligned(const void* q, uintptr_t a) { return ((uintptr_t)q & (a - 1)) == 0; }
int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

// One axis of a tensor: stride and size.
struct Axis { int64_t stride, size; };
// Rows of d elements start on 16-byte boundaries, and no offset inside the tensor leaves 50 bits.
bool rows_ok(std::initializer_list<Axis> axes) {
  for (const Axis& a : axes)
    if (a.stride < 0 || a.stride % 8 != 0 || (a.size > 1 && a.stride > ((int64_t)1 << 50) / a.size)) return false;
  return true;
}
// No two rows of a tensor that is written share an element: the axes of more than one entry, by growing stride, nest.
bool rows_apart(int d, Axis a, Axis b, Axis c = {0, 1}, Axis e = {0, 1}) {
  Axis ax[4] = {a, b, c, e};
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 4; ++j)
      if (ax[j].stride < ax[i].stride) { const Axis t = ax[i]; ax[i] = ax[j]; ax[j] = t; }
  int64_t extent = d;
  for (const Axis& x : ax) {
    if (x.size == 1) continue;
    if (x.stride < extent) return false;
    extent = x.stride * x.size;
  }
  return true;
}

int check_rotary(const attn_rotary_spec& r, int d, int inverse, attn::RotaryArgs* out) {
  if (r.rotary_dim < 2 || r.rotary_dim > d || r.rotary_dim % 2 != 0) return ATTN_ERR_ROTARY;
  if (r.frequencies == nullptr || !aligned(r.frequencies, 8) || !std::isfinite(r.magnitude)) return ATTN_ERR_ROTARY;
  *out = {r.frequencies, r.rotary_dim, r.interleaved != 0, inverse != 0, r.magnitude};
  return ATTN_OK;
}

// a rotation that may be left out
int check_rotary_or_none(const attn_rotary_spec& r, int d, int inverse, attn::RotaryArgs* out) {
  if (r.frequencies != nullptr || r.rotary_dim != 0) return check_rotary(r, d, inverse, out);
  *out = {nullptr, 0, 0, 0, 1.f};
  return ATTN_OK;
}

int check_norm(const attn_norm_spec* n, bool with_k, attn::NormArgs* out) {
  if (n == nullptr) return ATTN_ERR_NULL;
  if (n->q_weight == nullptr || (with_k && n->k_weight == nullptr)) return ATTN_ERR_NORM;
  const uintptr_t size = n->weights_fp32 ? 4 : 2;
  if (!aligned(n->q_weight, size) || (with_k && !aligned(n->k_weight, size))) return ATTN_ERR_NORM;
  if (!std::isnormal(n->eps) || !(n->eps > 0.f)) return ATTN_ERR_NORM;
  *out = {{n->q_weight, with_k ? n->k_weight : nullptr}, n->weights_fp32 != 0, n->eps};
  return ATTN_OK;
}

bool page_size_ok(int n) { return n >= 16 && n <= 4096 && (n & (n - 1)) == 0; }

// The caches' shape and strides.
int check_caches(int pages, int Hk, int page_size, int d, int64_t sp, int64_t sh, int64_t sn) {
  if (pages <= 0 || Hk <= 0 || Hk > (1 << 16)) return ATTN_ERR_SHAPE;
  if (!page_size_ok(page_size)) return ATTN_ERR_PAGES;
  // a page, and the step from one page to the next, are less than 4 GiB (tile copies address rows by 32-bit byte offsets)
  if ((int64_t)Hk * page_size * d > (int64_t)1 << 33) return ATTN_ERR_SHAPE;   // (a copy counts a page's 16-byte pieces in 32 bits)
  if (sn > ((int64_t)1 << 23) || sn * page_size >= (int64_t)1 << 31 || sp >= (int64_t)1 << 31) return ATTN_ERR_SHAPE;
  const Axis p = {sp, pages}, h = {sh, Hk}, n = {sn, page_size};
  return rows_ok({p, h, n}) && rows_apart(d, p, h, n) ? ATTN_OK : ATTN_ERR_SHAPE;
}

int check_batch(const attn_paged_params* p, attn::PagedBatch* out) {
  if (p == nullptr) return ATTN_ERR_NULL;
  if (!dtype_ok(p->dtype)) return ATTN_ERR_DTYPE;
  if (!head_dim_ok(p->d)) return ATTN_ERR_HEADDIM;
  if (p->B <= 0 || p->T <= 0 || p->Hq <= 0 || p->Hk <= 0 || p->Hq % p->Hk != 0 || p->table_width <= 0) return ATTN_ERR_SHAPE;
  if (p->B > (1 << 20) || p->T > (1 << 28) || p->Hq > (1 << 16) || (int64_t)p->T * p->Hq > (int64_t)1 << 30) return ATTN_ERR_SHAPE;
  const int st = check_caches(p->pages, p->Hk, p->page_size, p->d, p->page_stride, p->head_stride, p->row_stride);
  if (st != ATTN_OK) return st;
  if ((int64_t)p->table_width * p->page_size > (int64_t)1 << 30) return ATTN_ERR_SHAPE;
  if (p->table_stride < 0 || (p->B > 1 && p->table_stride > ((int64_t)1 << 50) / p->B)) return ATTN_ERR_SHAPE;
  if (p->query_starts == nullptr && p->T < p->B) return ATTN_ERR_SHAPE;
  attn::PagedBatch& b = *out;
  std::memset(&b, 0, sizeof(b));
  b.table = p->block_table;
  b.lengths = p->lengths;
  b.starts = p->query_starts;
  b.table_stride = p->table_stride;
  b.B = p->B; b.T = p->T; b.Hq = p->Hq; b.Hk = p->Hk;
  b.pages = p->pages; b.page_log2 = log2_of(p->page_size); b.width = p->table_width;
  b.capacity = p->table_width << b.page_log2;
  b.sp = p->page_stride; b.sh = p->head_stride; b.sn = p->row_stride;
  b.page_bytes = (uint32_t)(2 * p->page_stride); b.row_bytes = (uint32_t)(2 * p->row_stride); b.page_mask = (uint32_t)p->page_size - 1;
  return ATTN_OK;
}
int check_batch_pointers(const attn::PagedBatch& b) {
  if (b.table == nullptr || b.lengths == nullptr) return ATTN_ERR_NULL;
  return aligned(b.table, 4) && aligned(b.lengths, 4) && aligned(b.starts, 4) ? ATTN_OK : ATTN_ERR_SHAPE;
}

// The line that the work is laid out on (attn_paged_line.h), at its longest (320: what an item costs beside its keys, at most); false: too long for its arithmetic.
bool lay_out(const attn_paged_params* p, const attn::PagedShape& shape, attn::PagedCall* out) {
  attn::PagedCall& c = *out;
  c.slots = shape.slots;
  const double rows = (double)p->T * c.G, blocks = rows / shape.rows + p->B;
  if (p->Hk * (blocks * c.G * ((double)c.b.capacity + 320) + rows * (blocks + 1)) > 0x1p50) return false;
  // (a sequence of r rows has at most r / BR + 1 blocks, and the sum over these of BR (t + 1) is at most (r + BR) (r / BR + 2) / 2: not above 2^51)
  c.longest_line = p->Hk * (blocks * c.G * ((double)c.b.capacity + 320) + 0.5 * (rows + (double)p->B * shape.rows) * (rows / shape.rows + 2)) + 1;
  return true;
}

// What attn_paged_fwd takes from the params beside the pointers.
int check_paged(const attn_paged_params* p, attn::PagedCall* out, attn::PagedShape* shape) {
  attn::PagedCall& c = *out;
  std::memset(&c, 0, sizeof(c));
  const int st = check_batch(p, &c.b);
  if (st != ATTN_OK) return st;
  if (!std::isfinite(p->softmax_scale) || !(p->softmax_scale > 0.0f)) return ATTN_ERR_SCALE;
  const Axis qt = {p->q_stride_t, p->T}, qh = {p->q_stride_h, p->Hq}, ot = {p->o_stride_t, p->T}, oh = {p->o_stride_h, p->Hq};
  if (!rows_ok({qt, qh, ot, oh}) || !rows_apart(p->d, ot, oh)) return ATTN_ERR_SHAPE;
  c.qt = qt.stride; c.qh = qh.stride; c.ot = ot.stride; c.oh = oh.stride;
  c.G = p->Hq / p->Hk;
  c.g_shift = 31 + (c.G > 1 ? log2_of(c.G - 1) + 1 : 0);
  c.g_factor = (uint32_t)((((uint64_t)1 << c.g_shift) + c.G - 1) / c.G);
  c.d = p->d;
  c.causal = p->causal != 0;
  c.scale_log2 = (float)((double)p->softmax_scale * 1.4426950408889634);
  *shape = attn::paged_shape((int64_t)p->T * c.G, p->B, p->Hk, p->d);
  return lay_out(p, *shape, &c) ? ATTN_OK : ATTN_ERR_SHAPE;
}

int check_rotary_sizes(const attn_rotary_params* p, int32_t n_tensors) {
  if (!dtype_ok(p->dtype)) return ATTN_ERR_DTYPE;
  if (!head_dim_ok(p->d)) return ATTN_ERR_HEADDIM;
  if (p->B <= 0 || p->N <= 0 || (int64_t)p->B * p->N > (int64_t)1 << 28 || n_tensors < 1 || n_tensors > 2) return ATTN_ERR_SHAPE;
  if (p->positions != nullptr && (!aligned(p->positions, 4) || p->position_stride_b < 0 || p->position_stride_b > ((int64_t)1 << 50) / p->B)) return ATTN_ERR_SHAPE;
  return ATTN_OK;
}
// Sizes, type, positions and tensors of a rotation (of a norm too: without a rotation if there is none).
int check_rotary_call(const attn_rotary_params* p, const attn_rotary_tensor* tensors, int32_t n_tensors, bool or_none, attn::RotaryCall* out) {
  if (p == nullptr || tensors == nullptr) return ATTN_ERR_NULL;
  int st = check_rotary_sizes(p, n_tensors);
  if (st != ATTN_OK) return st;
  attn::RotaryCall& c = *out;
  std::memset(&c, 0, sizeof(c));
  st = or_none ? check_rotary_or_none(p->rotary, p->d, p->inverse, &c.rot) : check_rotary(p->rotary, p->d, p->inverse, &c.rot);
  if (st != ATTN_OK) return st;
  for (int i = 0; i < n_tensors; ++i) {
    const attn_rotary_tensor& t = tensors[i];
    if (t.H <= 0 || t.H > (1 << 16)) return ATTN_ERR_SHAPE;
    const Axis xb = {t.x_stride_b, p->B}, xh = {t.x_stride_h, t.H}, xn = {t.x_stride_n, p->N};
    const Axis yb = {t.y_stride_b, p->B}, yh = {t.y_stride_h, t.H}, yn = {t.y_stride_n, p->N};
    if (!rows_ok({xb, xh, xn, yb, yh, yn}) || !rows_apart(p->d, yb, yh, yn)) return ATTN_ERR_SHAPE;
    if (t.x == nullptr || t.y == nullptr) return ATTN_ERR_NULL;
    if (!aligned(t.x, 16) || !aligned(t.y, 16)) return ATTN_ERR_SHAPE;
    if (t.x == t.y && (xb.stride != yb.stride || xh.stride != yh.stride || xn.stride != yn.stride)) return ATTN_ERR_SHAPE;
    c.t[i] = {t.x, t.y, t.H, xb.stride, xh.stride, xn.stride, yb.stride, yh.stride, yn.stride};
  }
  // (what one tensor's threads write, the other's must not read or write)
  if (n_tensors == 2 && (tensors[0].y == tensors[1].y || tensors[0].y == tensors[1].x || tensors[1].y == tensors[0].x)) return ATTN_ERR_SHAPE;
  c.n_tensors = n_tensors;
  c.B = p->B; c.N = p->N; c.d = p->d;
  c.positions = p->positions;
  c.position_sb = p->position_stride_b;
  return ATTN_OK;
}

}  // namespace

extern "C" {

int attn_rotary(const attn_rotary_params* p, const attn_rotary_tensor* tensors, int32_t n_tensors) {
  attn::RotaryCall c;
  const int st = check_rotary_call(p, tensors, n_tensors, false, &c);
  if (st != ATTN_OK) return st;
  return attn::launch_rotary(c, p->dtype, (hipStream_t)p->stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

int attn_norm_rotary(const attn_rotary_params* p, const attn_norm_spec* norm, const attn_rotary_tensor* tensors, int32_t n_tensors) {
  attn::NormCall c;
  int st = check_rotary_call(p, tensors, n_tensors, true, &c.rotary);
  if (st != ATTN_OK) return st;
  if (p->inverse != 0) return ATTN_ERR_ROTARY;
  st = check_norm(norm, n_tensors == 2, &c.norm);
  if (st != ATTN_OK) return st;
  return attn::launch_norm_rotary(c, p->dtype, (hipStream_t)p->stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

size_t attn_norm_rotary_bwd_workspace_bytes(int32_t d) { return head_dim_ok(d) ? attn::norm_workspace_bytes(d) : 0; }

int attn_norm_rotary_bwd(const attn_rotary_params* p, const attn_norm_spec* norm, const attn_norm_grad* tensors, int32_t n_tensors, void* workspace,
                         size_t workspace_bytes) {
  if (p == nullptr || tensors == nullptr) return ATTN_ERR_NULL;
  int st = check_rotary_sizes(p, n_tensors);
  if (st != ATTN_OK) return st;
  attn::NormBwdCall c;
  std::memset(&c, 0, sizeof(c));
  st = check_rotary_or_none(p->rotary, p->d, 1, &c.rot);
  if (st != ATTN_OK) return st;
  if (p->inverse != 0) return ATTN_ERR_ROTARY;
  st = check_norm(norm, n_tensors == 2, &c.norm);
  if (st != ATTN_OK) return st;
  for (int i = 0; i < n_tensors; ++i) {
    const attn_norm_grad& t = tensors[i];
    if (t.H <= 0 || t.H > (1 << 16)) return ATTN_ERR_SHAPE;
    const Axis xb = {t.x_stride_b, p->B}, xh = {t.x_stride_h, t.H}, xn = {t.x_stride_n, p->N};
    const Axis gb = {t.dy_stride_b, p->B}, gh = {t.dy_stride_h, t.H}, gn = {t.dy_stride_n, p->N};
    const Axis yb = {t.dx_stride_b, p->B}, yh = {t.dx_stride_h, t.H}, yn = {t.dx_stride_n, p->N};
    if (!rows_ok({xb, xh, xn, gb, gh, gn, yb, yh, yn}) || !rows_apart(p->d, yb, yh, yn)) return ATTN_ERR_SHAPE;
    if (t.x == nullptr || t.dy == nullptr || t.dx == nullptr) return ATTN_ERR_NULL;
    if (!aligned(t.x, 16) || !aligned(t.dy, 16) || !aligned(t.dx, 16)) return ATTN_ERR_SHAPE;
    if (!aligned(t.dw, c.norm.w_fp32 ? 4 : 2)) return ATTN_ERR_NORM;
    c.t[i] = {t.x, t.dy, t.dx, t.dw, t.H, xb.stride, xh.stride, xn.stride, gb.stride, gh.stride, gn.stride, yb.stride, yh.stride, yn.stride};
  }
  // (what one thread writes, no other must read or write)
  for (int i = 0; i < n_tensors; ++i)
    for (int j = 0; j < n_tensors; ++j)
      if (c.t[i].dx == c.t[j].x || c.t[i].dx == c.t[j].dy || (i != j && (c.t[i].dx == c.t[j].dx || (c.t[i].dw != nullptr && c.t[i].dw == c.t[j].dw)))) return ATTN_ERR_SHAPE;
  if ((c.t[0].dw != nullptr || c.t[1].dw != nullptr) &&
      (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < attn::norm_workspace_bytes(p->d)))
    return ATTN_ERR_WORKSPACE;
  c.n_tensors = n_tensors;
  c.B = p->B; c.N = p->N; c.d = p->d;
  c.positions = p->positions;
  c.position_sb = p->position_stride_b;
  c.partial = (float*)workspace;
  return attn::launch_norm_rotary_bwd(c, p->dtype, (hipStream_t)p->stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

static int check_append(const attn_paged_params* p, const attn_rotary_spec* rotary, bool normed, const void* K, const void* V, void* k_cache, void* v_cache, const void* Q,
                        void* Qout, attn::AppendCall* out) {
  attn::AppendCall& c = *out;
  std::memset(&c, 0, sizeof(c));
  int st = check_batch(p, &c.b);
  if (st != ATTN_OK) return st;
  if (rotary != nullptr) {
    st = check_rotary(*rotary, p->d, 0, &c.rot);
    if (st != ATTN_OK) return st;
  } else if (Q != nullptr && !normed) {
    return ATTN_ERR_ROTARY;
  }
  const Axis kt = {p->k_stride_t, p->T}, kh = {p->k_stride_h, p->Hk}, vt = {p->v_stride_t, p->T}, vh = {p->v_stride_h, p->Hk};
  if (!rows_ok({kt, kh, vt, vh})) return ATTN_ERR_SHAPE;
  st = check_batch_pointers(c.b);
  if (st != ATTN_OK) return st;
  if (!K || !V || !k_cache || !v_cache || (Q == nullptr) != (Qout == nullptr)) return ATTN_ERR_NULL;
  for (const void* q : {K, V, (const void*)k_cache, (const void*)v_cache, Q, (const void*)Qout})
    if (!aligned(q, 16)) return ATTN_ERR_SHAPE;
  if (Q != nullptr) {
    const Axis qt = {p->q_stride_t, p->T}, qh = {p->q_stride_h, p->Hq}, ot = {p->o_stride_t, p->T}, oh = {p->o_stride_h, p->Hq};
    if (!rows_ok({qt, qh, ot, oh}) || !rows_apart(p->d, ot, oh)) return ATTN_ERR_SHAPE;
    if (Q == Qout && (qt.stride != ot.stride || qh.stride != oh.stride)) return ATTN_ERR_SHAPE;
    c.qt = qt.stride; c.qh = qh.stride; c.ot = ot.stride; c.oh = oh.stride;
  }
  // (what two groups of threads would write, or one write and the other read)
  if (k_cache == v_cache || (Q != nullptr && (Qout == K || Qout == V || Qout == k_cache || Qout == v_cache))) return ATTN_ERR_SHAPE;
  c.d = p->d;
  c.K = K; c.V = V; c.Q = Q; c.Kc = k_cache; c.Vc = v_cache; c.Qo = Qout;
  c.kt = kt.stride; c.kh = kh.stride; c.vt = vt.stride; c.vh = vh.stride;
  return ATTN_OK;
}

int attn_paged_append(const attn_paged_params* p, const attn_rotary_spec* rotary, const void* K, const void* V, void* k_cache, void* v_cache, const void* Q,
                      void* Qout) {
  attn::AppendCall c;
  const int st = check_append(p, rotary, false, K, V, k_cache, v_cache, Q, Qout, &c);
  if (st != ATTN_OK) return st;
  return attn::launch_append(c, p->dtype, (hipStream_t)p->stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

int attn_paged_norm_append(const attn_paged_params* p, const attn_rotary_spec* rotary, const attn_norm_spec* norm, const void* K, const void* V, void* k_cache,
                           void* v_cache, const void* Q, void* Qout) {
  attn::AppendCall c;
  int st = check_append(p, rotary, true, K, V, k_cache, v_cache, Q, Qout, &c);
  if (st != ATTN_OK) return st;
  if (rotary == nullptr) c.rot.magnitude = 1.f;
  attn::NormArgs n;
  if (norm != nullptr && Q == nullptr) {   // (only K's weights are used then)
    attn_norm_spec k_only = *norm;
    k_only.q_weight = norm->k_weight;
    st = check_norm(&k_only, true, &n);
  } else {
    st = check_norm(norm, true, &n);
  }
  if (st != ATTN_OK) return st;
  return attn::launch_norm_append(c, n, p->dtype, (hipStream_t)p->stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

size_t attn_paged_workspace_bytes(const attn_paged_params* p) {
  attn::PagedCall c;
  attn::PagedShape shape;
  return check_paged(p, &c, &shape) == ATTN_OK ? attn::paged_workspace_bytes(p->d) : 0;
}

// window 0: none
static int paged_fwd(const attn_paged_params* p, int32_t window, int32_t sinks, const void* Q, const void* k_cache, const void* v_cache, void* O, float* LSE, void* workspace,
                     size_t workspace_bytes) {
  attn::PagedCall c;
  attn::PagedShape shape;
  int st = check_paged(p, &c, &shape);
  if (st != ATTN_OK) return st;
  c.window = window;
  c.sinks = sinks;
  st = check_batch_pointers(c.b);
  if (st != ATTN_OK) return st;
  if (!Q || !k_cache || !v_cache || !O || !LSE) return ATTN_ERR_NULL;
  for (const void* q : {Q, k_cache, v_cache, (const void*)O})
    if (!aligned(q, 16)) return ATTN_ERR_SHAPE;
  if (!aligned(LSE, 4)) return ATTN_ERR_SHAPE;
  if (workspace == nullptr || !aligned(workspace, 256) || workspace_bytes < attn::paged_workspace_bytes(p->d)) return ATTN_ERR_WORKSPACE;
  c.Q = Q; c.K = k_cache; c.V = v_cache; c.O = O; c.LSE = LSE;
  c.part = (float*)workspace;
  if (attn::paged_few(c)) return attn::launch_paged_few(c, p->dtype, (hipStream_t)p->stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
  if (window > 0 && attn::paged_window_apart(*p, shape, window, sinks)) {
    const attn::PagedShape few = {32, attn::paged_one_slots(p->d)};
    attn::PagedCall single = c;
    if (lay_out(p, few, &single)) {   // (one after the other, in the same workspace)
      c.only = 1;
      single.only = 2;
      int e = attn::launch_paged_rows(c, p->dtype, (hipStream_t)p->stream);
      if (e == 0) e = attn::launch_paged_one(single, p->dtype, (hipStream_t)p->stream);
      return e == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
    }
  }
  const int e = shape.rows == 32 ? attn::launch_paged_one(c, p->dtype, (hipStream_t)p->stream) : attn::launch_paged_rows(c, p->dtype, (hipStream_t)p->stream);
  return e == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

int attn_paged_fwd(const attn_paged_params* p, const void* Q, const void* k_cache, const void* v_cache, void* O, float* LSE, void* workspace,
                   size_t workspace_bytes) {
  return paged_fwd(p, 0, 0, Q, k_cache, v_cache, O, LSE, workspace, workspace_bytes);
}

int attn_paged_window_fwd(const attn_paged_params* p, int32_t window, int32_t sinks, const void* Q, const void* k_cache, const void* v_cache, void* O, float* LSE,
                          void* workspace, size_t workspace_bytes) {
  if (p == nullptr) return ATTN_ERR_NULL;
  if (p->causal == 0 || window < 1 || sinks < 0) return ATTN_ERR_WINDOW;
  // (a cache holds no more than 2^30 positions of a sequence)
  return paged_fwd(p, window, sinks < (1 << 30) ? sinks : 1 << 30, Q, k_cache, v_cache, O, LSE, workspace, workspace_bytes);
}

int attn_paged_copy(const attn_paged_copy_params* p, void* k_cache, void* v_cache, const int32_t* pairs, int64_t n_pairs) {
  if (p == nullptr) return ATTN_ERR_NULL;
  if (!dtype_ok(p->dtype)) return ATTN_ERR_DTYPE;
  if (!head_dim_ok(p->d)) return ATTN_ERR_HEADDIM;
  if (p->layers <= 0 || p->layers > (1 << 14) || n_pairs < 0 || n_pairs > p->pages) return ATTN_ERR_SHAPE;
  const int st = check_caches(p->pages, p->Hk, p->page_size, p->d, p->page_stride, p->head_stride, p->row_stride);
  if (st != ATTN_OK) return st;
  const Axis l = {p->layer_stride, p->layers}, pg = {p->page_stride, p->pages}, h = {p->head_stride, p->Hk}, n = {p->row_stride, p->page_size};
  if (!rows_ok({l}) || !rows_apart(p->d, l, pg, h, n)) return ATTN_ERR_SHAPE;
  if (!k_cache || !v_cache || (pairs == nullptr && n_pairs > 0)) return ATTN_ERR_NULL;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16)) return ATTN_ERR_SHAPE;
  if (n_pairs == 0) return ATTN_OK;
  // one byte a page: 1 a source, 2 a destination
  uint8_t* const role = new (std::nothrow) uint8_t[p->pages]();
  if (role == nullptr) return ATTN_ERR_PAGES;
  bool ok = true;
  for (int64_t i = 0; i < n_pairs && ok; ++i) {
    const int32_t src = pairs[2 * i], dst = pairs[2 * i + 1];
    ok = src >= 0 && src < p->pages && dst >= 0 && dst < p->pages && role[src] != 2 && role[dst] == 0 && src != dst;
    if (ok) {
      role[src] = 1;
      role[dst] = 2;
    }
  }
  delete[] role;
  if (!ok) return ATTN_ERR_PAGES;
  attn::CopyCall c = {k_cache, v_cache, p->layers, p->Hk, p->page_size, p->d, p->layer_stride, p->page_stride, p->head_stride, p->row_stride};
  return attn::launch_page_copy(c, pairs, n_pairs, (hipStream_t)p->stream) == 0 ? ATTN_OK : ATTN_ERR_LAUNCH;
}

}  // extern "C"
