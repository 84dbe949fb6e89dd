// extern "C" entry points of a model's step over its cache: host-side validation, then the launches on the caller's stream.
// No allocation, no synchronisation, no state.
#include "ea_attend.h"
#include "ea_mx.h"
#include "ea_step.h"
#include "ea_tree.h"

namespace ea {

static inline bool aligned(const void* p, uintptr_t to) { return p && ((uintptr_t)p & (to - 1)) == 0; }
static bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return na && nb && x < y + nb && y < x + na;
}
constexpr int kCutHeads = 256;     // most heads of a call that are cut each for itself
constexpr int kPlanCus = 256;      // a plan, and with it the size of its workspace, is the same wherever it is made

hipError_t launch_attend(const AttendArgs& a, const Dims& d, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.plan.rows)
    e = a.mx == 8 ? launch_attend_rows_mx8(a, d, st) : a.mx == 4 ? launch_attend_rows_mx4(a, d, st)
        : a.sees ? launch_attend_rows_tree(a, d, st) : launch_attend_rows(a, d, st);
  if (e != hipSuccess || !a.plan.tile) return e;
  if (a.mx) return a.mx == 8 ? launch_attend_tile_mx8(a, d, st) : launch_attend_tile_mx4(a, d, st);
  if (d.dtype != EA_BF16) return a.sees ? launch_attend_f32_tree(a, st) : launch_attend_f32(a, st);
  return a.sees ? launch_attend_tile_tree(a, d, st) : launch_attend_tile(a, d, st);
}

// MX pools: four tensors of their own
static ea_status check_mx(const Dims& d, const ea_mx* mx, const PageMap& pm, size_t* bytes, size_t* scales) {
  if (!mx || !aligned(mx->k, 16) || !aligned(mx->v, 16) || !aligned(mx->k_scale, 16) || !aligned(mx->v_scale, 16)) return EA_ERR_INVALID_ARG;
  if (mx->format != EA_MXFP8 && mx->format != EA_MXFP4) return EA_ERR_UNSUPPORTED;
  const size_t rows = ((size_t)pm.num_blocks << pm.sh) * d.Hkv;
  *bytes = rows * (mx->format == EA_MXFP8 ? d.D : d.D / 2);
  *scales = rows * (d.D / 32);
  const struct { const void* at; size_t bytes; } part[4] = {{mx->k, *bytes}, {mx->v, *bytes}, {mx->k_scale, *scales}, {mx->v_scale, *scales}};
  for (int i = 0; i < 4; ++i)
    for (int j = i + 1; j < 4; ++j)
      if (overlap(part[i].at, part[i].bytes, part[j].at, part[j].bytes)) return EA_ERR_INVALID_ARG;
  return EA_OK;
}
static bool over_mx(const void* at, size_t n, const ea_mx* mx, size_t bytes, size_t scales) {
  return overlap(at, n, mx->k, bytes) || overlap(at, n, mx->v, bytes) || overlap(at, n, mx->k_scale, scales) || overlap(at, n, mx->v_scale, scales);
}

static ea_status check_tree(const ea_step* step, const ea_tree* tree) {
  if (!step || !tree) return EA_ERR_INVALID_ARG;
  if (tree->words < 1 || step->max_new > (int64_t)64 * tree->words) return EA_ERR_INVALID_ARG;
  if (tree->words > EA_TREE_MAX / 64) return EA_ERR_UNSUPPORTED;
  if (step->n_tokens > 0 && !aligned(tree->sees, 8)) return EA_ERR_INVALID_ARG;
  return EA_OK;
}

// mx: k and v are its elements.  tree: null, or which new rows a token sees
static ea_status attend(const Dims& d, const void* q, const ea_step* step, const ea_tree* tree, const void* k, const void* v, const PageMap* pm,
                        const float* kscale, const float* vscale, const ea_mx* mx, const int32_t* lengths, bool per_head, int64_t n,
                        int64_t n_cap, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  ea_status s = check_step(d, step, n);
  if (s != EA_OK) return s;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(lengths, 4) || !aligned(ws, 256)) return EA_ERR_INVALID_ARG;
  if (step->n_tokens > 0 && (!aligned(q, 16) || !aligned(out, 16))) return EA_ERR_INVALID_ARG;
  if ((lse && !aligned(lse, 4)) || (kscale && !aligned(kscale, 4)) || (vscale && !aligned(vscale, 4))) return EA_ERR_INVALID_ARG;
  const size_t es = d.dtype == EA_BF16 ? 2 : 4;
  AttendArgs a = {};
  a.q_stride = step->q_stride ? step->q_stride : (long long)d.Hq * d.D;
  const size_t rows = (size_t)step->n_tokens, out_bytes = rows * d.Hq * d.D * es;
  if (overlap(out, out_bytes, q, rows ? ((rows - 1) * a.q_stride + (size_t)d.Hq * d.D) * es : 0)) return EA_ERR_INVALID_ARG;
  if (mx) {
    size_t bytes, scales;
    if ((s = check_mx(d, mx, *pm, &bytes, &scales)) != EA_OK) return s;
    if (over_mx(out, out_bytes, mx, bytes, scales)) return EA_ERR_INVALID_ARG;
  } else {
    const size_t cache = (pm ? ((size_t)pm->num_blocks << pm->sh) * d.Hkv : (size_t)d.units() * n_cap) * d.D * d.esize();
    if (overlap(out, out_bytes, k, cache) || overlap(out, out_bytes, v, cache)) return EA_ERR_INVALID_ARG;
  }
  if (tree && overlap(out, out_bytes, tree->sees, rows * tree->words * 8)) return EA_ERR_INVALID_ARG;
  a.plan = make_attend_plan(d, n, step->n_tokens, step->max_new, kPlanCus, mx != nullptr, tree != nullptr);
  // Workgroups of up to 512 threads, 2^32 threads to a launch.  (The launches of few rows are no larger than kAttendShares, their
  // joining one than that many times 64 rows; the stretches' joining one comes with few tiles only.)
  if (a.plan.tile && a.plan.grid > kAttendMaxGrid) return EA_ERR_UNSUPPORTED;
  // the stretches' kernel steps over a block by a 32-bit number of bytes
  const int per_channel = mx ? mx->format == EA_MXFP8 ? 8 : 4 : 8 * d.esize();      // bits
  if (pm && a.plan.tile && (((uint64_t)d.Hkv << pm->sh) * d.D * per_channel / 8) >> 32) return EA_ERR_UNSUPPORTED;
  if (ws_bytes < a.plan.total) return EA_ERR_WORKSPACE;
  if (step->n_tokens == 0) return EA_OK;
  a.q = q; a.k = k; a.v = v; a.cu = step->cu_tokens; a.lens = lengths; a.kscale = kscale; a.vscale = vscale;
  a.out = out; a.lse = lse; a.ws = (char*)ws;
  if (pm) a.pm = *pm;
  a.n_cap = n_cap;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.G; a.D = d.D;
  a.n = (int)n; a.n_tokens = (int)step->n_tokens; a.per_head = per_head;
  if (mx) {
    a.mx = mx->format == EA_MXFP8 ? 8 : 4;
    a.kscale8 = mx->k_scale;
    a.vscale8 = mx->v_scale;
  }
  if (tree) {
    a.sees = tree->sees;
    a.words = tree->words;
  }
  // (every workgroup looks at all that is cut)
  a.by_head = tree && per_head && d.units() <= kCutHeads;
  a.only_long = a.plan.rows;
  a.short_rows = a.plan.short_rows;
  a.scale = (float)(1.4426950408889634074 / (d.D == 64 ? 8.0 : d.D == 256 ? 16.0 : 11.313708498984760390));
  return launch_attend(a, d, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

// what a call reads of the new rows and writes of the queries: q, k, v, q_out
struct NewBytes { const void* at[4]; size_t bytes[4]; };
static NewBytes bytes_of_rows(const Dims& d, const ea_new_rows* r, const AppendArgs& a) {
  const size_t es = d.dtype == EA_BF16 ? 2 : 4, n = (size_t)r->n_tokens, qd = (size_t)d.Hq * d.D, kd = (size_t)d.Hkv * d.D;
  return {{r->q, r->k, r->v, a.q_out},
          {r->q ? ((n - 1) * a.q_stride + qd) * es : 0, ((n - 1) * a.k_stride + kd) * es, ((n - 1) * a.v_stride + kd) * es, r->q ? n * qd * es : 0}};
}
// the new rows by themselves; strides and q_out into a.  nothing: there are none
static ea_status check_rows(const Dims& d, const ea_new_rows* r, void* q_out, AppendArgs* a, bool* nothing) {
  if (!r || r->n_tokens < 0) return EA_ERR_INVALID_ARG;
  if (r->n_tokens > kAttendMaxTokens) return EA_ERR_UNSUPPORTED;
  const int64_t qd = (int64_t)d.Hq * d.D, kd = (int64_t)d.Hkv * d.D, per16 = d.dtype == EA_BF16 ? 8 : 4;
  a->q_stride = r->q_stride ? r->q_stride : qd;
  a->k_stride = r->k_stride ? r->k_stride : kd;
  a->v_stride = r->v_stride ? r->v_stride : kd;
  a->q_out = q_out;
  const int64_t far = (int64_t)1 << 40;
  if (a->q_stride < qd || a->k_stride < kd || a->v_stride < kd || a->q_stride > far || a->k_stride > far || a->v_stride > far) return EA_ERR_INVALID_ARG;
  if (a->q_stride % per16 || a->k_stride % per16 || a->v_stride % per16) return EA_ERR_INVALID_ARG;
  if (r->q && !r->inv_freq) return EA_ERR_INVALID_ARG;
  *nothing = r->n_tokens == 0;
  if (*nothing) return EA_OK;
  if (!aligned(r->k, 16) || !aligned(r->v, 16) || (r->q && (!aligned(r->q, 16) || !aligned(q_out, 16)))) return EA_ERR_INVALID_ARG;
  if (r->inv_freq && (!aligned(r->inv_freq, 8) || !aligned(r->pos, 4))) return EA_ERR_INVALID_ARG;
  const NewBytes b = bytes_of_rows(d, r, *a);
  for (int i = 0; i < 3; ++i) {
    const bool itself = i == 0 && q_out == r->q && a->q_stride == qd;
    if (!itself && overlap(b.at[i], b.bytes[i], q_out, b.bytes[3])) return EA_ERR_INVALID_ARG;
  }
  return EA_OK;
}

static ea_status append(const Dims& d, const ea_new_rows* r, AppendArgs a, size_t cache, void* q_out, void* stream) {
  bool nothing;
  const ea_status s = check_rows(d, r, q_out, &a, &nothing);
  if (s != EA_OK) return s;
  if (!aligned(a.k_cache, 16) || !aligned(a.v_cache, 16) || a.k_cache == a.v_cache) return EA_ERR_INVALID_ARG;
  if (overlap(a.k_cache, cache, a.v_cache, cache)) return EA_ERR_INVALID_ARG;
  if (nothing) return EA_OK;
  const NewBytes b = bytes_of_rows(d, r, a);
  for (int i = 0; i < 4; ++i)
    if (overlap(b.at[i], b.bytes[i], a.k_cache, cache) || overlap(b.at[i], b.bytes[i], a.v_cache, cache)) return EA_ERR_INVALID_ARG;
  a.q = r->q; a.k = r->k; a.v = r->v; a.pos = r->pos; a.inv_freq = r->inv_freq;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.n_tokens = (int)r->n_tokens; a.rope_layout = d.rope_layout;
  return launch_append(a, d, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

// new rows into MX pools: the checks of append(), against four tensors
static ea_status append_mx(const Dims& d, const ea_new_rows* r, const int64_t* slots, const ea_mx* mx, const PageMap& pm, void* q_out, void* stream) {
  size_t bytes, scales;
  ea_status s = check_mx(d, mx, pm, &bytes, &scales);
  if (s != EA_OK) return s;
  MxAppendArgs a = {};
  AppendArgs rows = {};
  bool nothing;
  if ((s = check_rows(d, r, q_out, &rows, &nothing)) != EA_OK || nothing) return s;
  if (!aligned(slots, 8)) return EA_ERR_INVALID_ARG;
  const NewBytes in = bytes_of_rows(d, r, rows);
  for (int i = 0; i < 4; ++i)
    if (over_mx(in.at[i], in.bytes[i], mx, bytes, scales)) return EA_ERR_INVALID_ARG;
  a.q = r->q; a.k = r->k; a.v = r->v; a.q_out = q_out; a.pos = r->pos; a.inv_freq = r->inv_freq; a.slots = slots;
  a.k_pool = mx->k; a.v_pool = mx->v; a.k_scale = mx->k_scale; a.v_scale = mx->v_scale;
  a.q_stride = rows.q_stride; a.k_stride = rows.k_stride; a.v_stride = rows.v_stride; a.num_blocks = pm.num_blocks;
  a.Hq = d.Hq; a.Hkv = d.Hkv; a.n_tokens = (int)r->n_tokens; a.sh = pm.sh; a.rope_layout = d.rope_layout;
  a.bits = mx->format == EA_MXFP8 ? 8 : 4;
  return launch_append_mx(a, d, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

static ea_status append_heads(const Dims& d, const ea_new_rows* rows, const int32_t* cu_tokens, const int32_t* lengths, void* k, void* v,
                              const float* k_scale, const float* v_scale, int64_t n_cap, void* q_out, void* stream) {
  if (!aligned(cu_tokens, 4) || !aligned(lengths, 4) || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  if ((k_scale && !aligned(k_scale, 4)) || (v_scale && !aligned(v_scale, 4))) return EA_ERR_INVALID_ARG;
  AppendArgs a = {};
  a.k_cache = k; a.v_cache = v; a.cu = cu_tokens; a.lens = lengths; a.n_cap = n_cap; a.k_scale = k_scale; a.v_scale = v_scale;
  return append(d, rows, a, (size_t)d.units() * n_cap * d.D * d.esize(), q_out, stream);
}

// what a path's rows are moved in, and the step they are of
static ea_status keep_path(const Dims& d, const ea_step* step, const int32_t* path, const int32_t* n_path, KeepArgs a, const size_t* bytes,
                           const int32_t* lengths, int32_t* len_out, bool per_head, void* stream) {
  const ea_status s = check_step(d, step, 0);
  if (s != EA_OK) return s;
  if (step->max_new > EA_TREE_MAX) return EA_ERR_UNSUPPORTED;
  if (!aligned(path, 4) || !aligned(n_path, 4) || !aligned(lengths, 4) || !aligned(len_out, 4)) return EA_ERR_INVALID_ARG;
  const size_t lens = (size_t)(per_head ? d.units() : d.B) * 4, b4 = (size_t)d.B * 4;
  const struct { const void* at; size_t bytes; } in[] = {{lengths, lens}, {n_path, b4}, {path, b4 * step->max_new}, {step->cu_tokens, b4 + 4}};
  for (const auto& x : in) {
    if (overlap(len_out, lens, x.at, x.bytes)) return EA_ERR_INVALID_ARG;
    for (int i = 0; i < a.count; ++i)
      if (overlap(a.at[i], bytes[i], x.at, x.bytes)) return EA_ERR_INVALID_ARG;
  }
  for (int i = 0; i < a.count; ++i)
    if (overlap(a.at[i], bytes[i], len_out, lens)) return EA_ERR_INVALID_ARG;
  a.cu = step->cu_tokens; a.path = path; a.n_path = n_path; a.lens = lengths; a.len_out = len_out;
  a.B = d.B; a.Hkv = d.Hkv; a.n_tokens = (int)step->n_tokens; a.max_new = (int)step->max_new; a.per_head = per_head;
  return launch_keep_path(a, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

}  // namespace ea

using namespace ea;

extern "C" {

ea_status ea_block_tables(const ea_params* p, const ea_paged* pg, const int32_t* len_old, const int32_t* len_new,
                          int32_t* free_list, const int32_t* free_in, int32_t* len_out, int32_t* free_out,
                          int32_t* cu_tokens, int64_t n_tokens, int64_t* slots, int32_t* pos,
                          const int32_t* seen, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d, true);
  if (s != EA_OK) return s;
  d.dtype = EA_BF16;                 // nothing of the pools is touched: any type's table will do
  PageMap pm;
  if ((s = check_paged(d, pg, 1, &pm)) != EA_OK) return s;
  if (d.B > EA_BLOCK_TABLES_MAX_BATCH || pg->num_blocks > 0x7fffffff) return EA_ERR_UNSUPPORTED;
  // (blocks are counted in 32 bits, those given back too, of which lengths that make no sense may claim a whole table)
  if ((int64_t)d.B * pg->max_blocks > 0x7fffffff) return EA_ERR_UNSUPPORTED;
  if (n_tokens < 0 || n_tokens > 0x7fffffff) return EA_ERR_INVALID_ARG;
  const void* ints[] = {len_old, len_new, free_list, free_in, len_out, free_out, cu_tokens};
  for (const void* x : ints)
    if (!aligned(x, 4)) return EA_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!aligned(slots, 8) || !aligned(pos, 4))) return EA_ERR_INVALID_ARG;
  if (seen && !aligned(seen, 4)) return EA_ERR_INVALID_ARG;
  // nothing that is read while others write it: every buffer that is written is apart from every other one
  const size_t b4 = (size_t)d.B * 4, table = (size_t)d.B * pg->max_blocks * 4, list = (size_t)pg->num_blocks * 4;
  struct { const void* at; size_t bytes; bool written; } buf[] = {
      {len_old, b4, false}, {len_new, b4, false}, {free_in, 4, false}, {seen, seen ? b4 : 0, false},
      {pg->block_table, table, true}, {free_list, list, true}, {len_out, b4, true}, {free_out, 4, true},
      {cu_tokens, b4 + 4, true}, {slots, (size_t)n_tokens * 8, true}, {pos, (size_t)n_tokens * 4, true}};
  const int count = (int)(sizeof buf / sizeof buf[0]);
  for (int i = 0; i < count; ++i)
    for (int j = i + 1; j < count; ++j)
      if ((buf[i].written || buf[j].written) && overlap(buf[i].at, buf[i].bytes, buf[j].at, buf[j].bytes)) return EA_ERR_INVALID_ARG;
  BlockTableArgs a = {};
  a.table = const_cast<int32_t*>(pg->block_table);
  a.len_old = len_old; a.len_new = len_new; a.free_in = free_in; a.seen = seen; a.free_list = free_list; a.len_out = len_out;
  a.free_out = free_out; a.cu_tokens = cu_tokens; a.pos = pos; a.slots = slots; a.n_tokens = n_tokens; a.num_blocks = pg->num_blocks;
  a.B = d.B; a.sh = pm.sh; a.max_blocks = pg->max_blocks;
  return launch_block_tables(a, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

ea_status ea_append_paged(const ea_params* p, const ea_new_rows* rows, const int64_t* slots, void* k_pool, void* v_pool,
                          const ea_paged* pg, void* q_out, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, 1, &pm)) != EA_OK) return s;
  if (rows && rows->n_tokens > 0 && !aligned(slots, 8)) return EA_ERR_INVALID_ARG;
  AppendArgs a = {};
  a.k_cache = k_pool; a.v_cache = v_pool; a.slots = slots; a.num_blocks = pg->num_blocks; a.sh = pm.sh;
  return append(d, rows, a, ((size_t)pg->num_blocks << pm.sh) * d.Hkv * d.D * d.esize(), q_out, stream);
}

ea_status ea_append(const ea_params* p, const ea_new_rows* rows, const int32_t* cu_tokens, const int32_t* lengths, void* k,
                    void* v, int64_t n_cap, void* q_out, void* stream) {
  Dims d;
  const ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  return append_heads(d, rows, cu_tokens, lengths, k, v, nullptr, nullptr, n_cap, q_out, stream);
}

ea_status ea_append_fp8(const ea_params* p, const ea_new_rows* rows, const int32_t* cu_tokens, const int32_t* lengths,
                        void* k8, void* v8, const float* k_scale, const float* v_scale, int64_t n_cap, void* q_out,
                        void* stream) {
  Dims d;
  const ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  if (d.dtype != EA_BF16 || d.D == 64) return EA_ERR_UNSUPPORTED;
  d.kv_fp8 = 1;
  return append_heads(d, rows, cu_tokens, lengths, k8, v8, k_scale, v_scale, n_cap, q_out, stream);
}

size_t ea_attend_workspace_bytes(const ea_params* p, const ea_step* step, int64_t n) {
  Dims d;
  if (check_params(p, &d) != EA_OK || check_step(d, step, n) != EA_OK) return 0;
  const size_t rows = make_attend_plan(d, n, step->n_tokens, step->max_new, kPlanCus).total;
  // whatever the cache is, with masks or without
  const bool wide = d.dtype == EA_BF16;
  const size_t other = make_attend_plan(d, n, step->n_tokens, step->max_new, kPlanCus, wide, !wide).total;
  return rows > other ? rows : other;
}

ea_status ea_attend(const ea_params* p, const void* q, const ea_step* step, const void* k, const void* v,
                    const int32_t* lengths, int64_t n, int64_t n_cap, void* out, float* lse, void* ws, size_t ws_bytes,
                    void* stream) {
  Dims d;
  const ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  if (n > n_cap || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  return attend(d, q, step, nullptr, k, v, nullptr, nullptr, nullptr, nullptr, lengths, true, n, n_cap, out, lse, ws, ws_bytes, stream);
}

ea_status ea_attend_paged(const ea_params* p, const void* q, const ea_step* step, const void* k_pool, const void* v_pool,
                          const ea_paged* pg, const int32_t* lengths, int64_t n, void* out, float* lse, void* ws,
                          size_t ws_bytes, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, n, &pm)) != EA_OK) return s;
  return attend(d, q, step, nullptr, k_pool, v_pool, &pm, nullptr, nullptr, nullptr, lengths, false, n, 0, out, lse, ws, ws_bytes, stream);
}

ea_status ea_attend_fp8(const ea_params* p, const void* q, const ea_step* step, const void* k8, const void* v8,
                        const float* k_scale, const float* v_scale, const int32_t* lengths, int64_t n, int64_t n_cap,
                        void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  Dims d;
  const ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  if (d.dtype != EA_BF16 || d.D == 64) return EA_ERR_UNSUPPORTED;
  if (n > n_cap || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  d.kv_fp8 = 1;
  return attend(d, q, step, nullptr, k8, v8, nullptr, k_scale, v_scale, nullptr, lengths, true, n, n_cap, out, lse, ws, ws_bytes, stream);
}

ea_status ea_append_mx(const ea_params* p, const ea_new_rows* rows, const int64_t* slots, const ea_mx* mx, const ea_paged* pg,
                       void* q_out, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, 1, &pm)) != EA_OK) return s;
  return append_mx(d, rows, slots, mx, pm, q_out, stream);
}

ea_status ea_read_mx(const ea_params* p, const ea_mx* mx, const ea_paged* pg, const int32_t* lengths, int64_t n, int64_t n_cap,
                     void* k_out, void* v_out, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  size_t bytes, scales;
  if (n < 0 || n > kMaxN || n > n_cap || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  if ((s = check_paged(d, pg, n, &pm)) != EA_OK || (s = check_mx(d, mx, pm, &bytes, &scales)) != EA_OK) return s;
  if (!aligned(lengths, 4) || (k_out && !aligned(k_out, 16)) || (v_out && !aligned(v_out, 16))) return EA_ERR_INVALID_ARG;
  const size_t out = (size_t)d.units() * n_cap * d.D * 2;
  if (k_out && v_out && overlap(k_out, out, v_out, out)) return EA_ERR_INVALID_ARG;
  if ((k_out && over_mx(k_out, out, mx, bytes, scales)) || (v_out && over_mx(v_out, out, mx, bytes, scales))) return EA_ERR_INVALID_ARG;
  if (n == 0 || (!k_out && !v_out)) return EA_OK;
  MxReadArgs a = {};
  a.k = mx->k; a.v = mx->v; a.k_scale = mx->k_scale; a.v_scale = mx->v_scale; a.lens = lengths; a.k_out = k_out; a.v_out = v_out;
  a.pm = pm; a.n_cap = n_cap; a.B = d.B; a.Hkv = d.Hkv; a.n = (int)n; a.bits = mx->format == EA_MXFP8 ? 8 : 4;
  return launch_read_mx(a, d, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

ea_status ea_attend_mx(const ea_params* p, const void* q, const ea_step* step, const ea_mx* mx, const ea_paged* pg,
                       const int32_t* lengths, int64_t n, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, n, &pm)) != EA_OK) return s;
  if (!mx) return EA_ERR_INVALID_ARG;
  return attend(d, q, step, nullptr, mx->k, mx->v, &pm, nullptr, nullptr, mx, lengths, false, n, 0, out, lse, ws, ws_bytes, stream);
}

ea_status ea_tree_masks(const ea_params* p, const ea_step* step, const int32_t* parents, const ea_tree* tree, const int32_t* seen,
                        int32_t* pos, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d, true);
  if (s != EA_OK || (s = check_step(d, step, 0)) != EA_OK || (s = check_tree(step, tree)) != EA_OK) return s;
  if (seen && !aligned(seen, 4)) return EA_ERR_INVALID_ARG;
  if (step->n_tokens == 0) return EA_OK;
  if (!aligned(parents, 4) || (pos && !aligned(pos, 4))) return EA_ERR_INVALID_ARG;
  const size_t t4 = (size_t)step->n_tokens * 4, b4 = (size_t)d.B * 4;
  const struct { const void* at; size_t bytes; } out[] = {{tree->sees, (size_t)step->n_tokens * tree->words * 8}, {pos, pos ? t4 : 0}},
      in[] = {{parents, t4}, {seen, seen ? b4 : 0}, {step->cu_tokens, b4 + 4}};
  for (const auto& o : out)
    for (const auto& x : in)
      if (overlap(o.at, o.bytes, x.at, x.bytes)) return EA_ERR_INVALID_ARG;
  if (overlap(out[0].at, out[0].bytes, out[1].at, out[1].bytes)) return EA_ERR_INVALID_ARG;
  TreeArgs a = {};
  a.cu = step->cu_tokens; a.parents = parents; a.seen = seen; a.sees = tree->sees; a.pos = pos;
  a.B = d.B; a.n_tokens = (int)step->n_tokens; a.words = tree->words;
  return launch_tree_masks(a, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

ea_status ea_tree_accept(const ea_params* p, const ea_step* step, const int32_t* tokens, const int32_t* parents, const int32_t* target,
                         int32_t* path, int32_t* n_path, int32_t* next, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d, true);
  if (s != EA_OK || (s = check_step(d, step, 0)) != EA_OK) return s;
  if (step->max_new > EA_TREE_MAX) return EA_ERR_UNSUPPORTED;
  if (!aligned(path, 4) || !aligned(n_path, 4) || !aligned(next, 4)) return EA_ERR_INVALID_ARG;
  if (step->n_tokens > 0 && (!aligned(tokens, 4) || !aligned(parents, 4) || !aligned(target, 4))) return EA_ERR_INVALID_ARG;
  const size_t t4 = (size_t)step->n_tokens * 4, b4 = (size_t)d.B * 4;
  const struct { const void* at; size_t bytes; } out[] = {{path, b4 * step->max_new}, {n_path, b4}, {next, b4}},
      in[] = {{tokens, t4}, {parents, t4}, {target, t4}, {step->cu_tokens, b4 + 4}};
  for (int i = 0; i < 3; ++i) {
    for (const auto& x : in)
      if (overlap(out[i].at, out[i].bytes, x.at, x.bytes)) return EA_ERR_INVALID_ARG;
    for (int j = i + 1; j < 3; ++j)
      if (overlap(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return EA_ERR_INVALID_ARG;
  }
  TreeArgs a = {};
  a.cu = step->cu_tokens; a.parents = parents; a.tokens = tokens; a.target = target; a.path = path; a.n_path = n_path; a.next = next;
  a.B = d.B; a.n_tokens = (int)step->n_tokens; a.max_new = (int)step->max_new;
  return launch_tree_accept(a, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

ea_status ea_attend_tree(const ea_params* p, const void* q, const ea_step* step, const ea_tree* tree, const void* k, const void* v,
                         const int32_t* lengths, int64_t n, int64_t n_cap, void* out, float* lse, void* ws, size_t ws_bytes,
                         void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK || (s = check_tree(step, tree)) != EA_OK) return s;
  if (n > n_cap || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  return attend(d, q, step, tree, k, v, nullptr, nullptr, nullptr, nullptr, lengths, true, n, n_cap, out, lse, ws, ws_bytes, stream);
}

ea_status ea_attend_tree_fp8(const ea_params* p, const void* q, const ea_step* step, const ea_tree* tree, const void* k8, const void* v8,
                             const float* k_scale, const float* v_scale, const int32_t* lengths, int64_t n, int64_t n_cap, void* out,
                             float* lse, void* ws, size_t ws_bytes, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK || (s = check_tree(step, tree)) != EA_OK) return s;
  if (d.dtype != EA_BF16 || d.D == 64) return EA_ERR_UNSUPPORTED;
  if (n > n_cap || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  d.kv_fp8 = 1;
  return attend(d, q, step, tree, k8, v8, nullptr, k_scale, v_scale, nullptr, lengths, true, n, n_cap, out, lse, ws, ws_bytes, stream);
}

ea_status ea_attend_tree_paged(const ea_params* p, const void* q, const ea_step* step, const ea_tree* tree, const void* k_pool,
                               const void* v_pool, const ea_paged* pg, const int32_t* lengths, int64_t n, void* out, float* lse,
                               void* ws, size_t ws_bytes, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK || (s = check_tree(step, tree)) != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, n, &pm)) != EA_OK) return s;
  return attend(d, q, step, tree, k_pool, v_pool, &pm, nullptr, nullptr, nullptr, lengths, false, n, 0, out, lse, ws, ws_bytes, stream);
}

ea_status ea_attend_tree_mx(const ea_params* p, const void* q, const ea_step* step, const ea_tree* tree, const ea_mx* mx,
                            const ea_paged* pg, const int32_t* lengths, int64_t n, void* out, float* lse, void* ws, size_t ws_bytes,
                            void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK || (s = check_tree(step, tree)) != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, n, &pm)) != EA_OK) return s;
  if (!mx) return EA_ERR_INVALID_ARG;
  return attend(d, q, step, tree, mx->k, mx->v, &pm, nullptr, nullptr, mx, lengths, false, n, 0, out, lse, ws, ws_bytes, stream);
}

ea_status ea_keep_path(const ea_params* p, const ea_step* step, const int32_t* path, const int32_t* n_path, void* k, void* v,
                       const int32_t* lengths, int64_t n_cap, int32_t* len_out, void* stream) {
  Dims d;
  const ea_status s = check_params(p, &d, true);
  if (s != EA_OK) return s;
  if (!aligned(k, 16) || !aligned(v, 16) || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  const int row = d.D * d.esize();
  const size_t bytes[2] = {(size_t)d.units() * n_cap * row, (size_t)d.units() * n_cap * row};
  if (overlap(k, bytes[0], v, bytes[1])) return EA_ERR_INVALID_ARG;
  KeepArgs a = {{(char*)k, (char*)v}, {row, row}, 2};
  a.n_cap = n_cap;
  return keep_path(d, step, path, n_path, a, bytes, lengths, len_out, true, stream);
}

ea_status ea_keep_path_paged(const ea_params* p, const ea_step* step, const int32_t* path, const int32_t* n_path, void* k_pool,
                             void* v_pool, const ea_paged* pg, const int64_t* slots, const int32_t* lengths, int32_t* len_out,
                             void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, 1, &pm)) != EA_OK) return s;
  if (!aligned(k_pool, 16) || !aligned(v_pool, 16) || (slots && !aligned(slots, 8))) return EA_ERR_INVALID_ARG;
  const size_t pool = ((size_t)pm.num_blocks << pm.sh) * d.Hkv * d.D * 2, bytes[2] = {pool, pool};
  if (overlap(k_pool, pool, v_pool, pool)) return EA_ERR_INVALID_ARG;
  KeepArgs a = {{(char*)k_pool, (char*)v_pool}, {d.D * 2, d.D * 2}, 2};
  a.pm = pm;
  a.slots = slots;
  return keep_path(d, step, path, n_path, a, bytes, lengths, len_out, false, stream);
}

ea_status ea_keep_path_mx(const ea_params* p, const ea_step* step, const int32_t* path, const int32_t* n_path, const ea_mx* mx,
                          const ea_paged* pg, const int64_t* slots, const int32_t* lengths, int32_t* len_out, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  size_t pool, scales;
  if ((s = check_paged(d, pg, 1, &pm)) != EA_OK || (s = check_mx(d, mx, pm, &pool, &scales)) != EA_OK) return s;
  if (slots && !aligned(slots, 8)) return EA_ERR_INVALID_ARG;
  const size_t bytes[4] = {pool, pool, scales, scales};
  const int row = mx->format == EA_MXFP8 ? d.D : d.D / 2;
  KeepArgs a = {{(char*)mx->k, (char*)mx->v, (char*)mx->k_scale, (char*)mx->v_scale}, {row, row, d.D / 32, d.D / 32}, 4};
  a.pm = pm;
  a.slots = slots;
  return keep_path(d, step, path, n_path, a, bytes, lengths, len_out, false, stream);
}

}  // extern "C"
