// extern "C" entry points of a model's step over its cache: host-side validation, then the launches on the caller's stream.
// No allocation, no synchronisation, no state.
#include "ea_attend.h"
#include "ea_step.h"

namespace ea {

static inline bool aligned(const void* p, uintptr_t to) { return p && ((uintptr_t)p & (to - 1)) == 0; }
static bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return na && nb && x < y + nb && y < x + na;
}
constexpr int kPlanCus = 256;      // a plan, and with it the size of its workspace, is the same wherever it is made

hipError_t launch_attend(const AttendArgs& a, const Dims& d, hipStream_t st) {
  hipError_t e = hipSuccess;
  if (a.plan.rows) e = launch_attend_rows(a, d, st);
  if (e != hipSuccess || !a.plan.tile) return e;
  return d.dtype == EA_BF16 ? launch_attend_tile(a, d, st) : launch_attend_f32(a, st);
}

static ea_status attend(const Dims& d, const void* q, const ea_step* step, const void* k, const void* v, const PageMap* pm,
                        const float* kscale, const float* vscale, const int32_t* lengths, bool per_head, int64_t n,
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
  const size_t cache = (pm ? ((size_t)pm->num_blocks << pm->sh) * d.Hkv : (size_t)d.units() * n_cap) * d.D * d.esize();
  if (overlap(out, out_bytes, k, cache) || overlap(out, out_bytes, v, cache)) return EA_ERR_INVALID_ARG;
  a.plan = make_attend_plan(d, n, step->n_tokens, step->max_new, kPlanCus);
  // Workgroups of up to 512 threads, 2^32 threads to a launch.  (The launches of few rows are no larger than 512 shares, their
  // joining one than 512 times 64 rows; the stretches' joining one comes with few tiles only.)
  if (a.plan.tile && a.plan.grid > kAttendMaxGrid) return EA_ERR_UNSUPPORTED;
  // the stretches' kernel steps over a block by a 32-bit number of bytes
  if (pm && a.plan.tile && (((uint64_t)d.Hkv << pm->sh) * d.D * d.esize()) >> 32) return EA_ERR_UNSUPPORTED;
  if (ws_bytes < a.plan.total) return EA_ERR_WORKSPACE;
  if (step->n_tokens == 0) return EA_OK;
  a.q = q; a.k = k; a.v = v; a.cu = step->cu_tokens; a.lens = lengths; a.kscale = kscale; a.vscale = vscale;
  a.out = out; a.lse = lse; a.ws = (char*)ws;
  if (pm) a.pm = *pm;
  a.n_cap = n_cap;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.G; a.D = d.D;
  a.n = (int)n; a.n_tokens = (int)step->n_tokens; a.per_head = per_head;
  a.only_long = a.plan.rows;
  a.short_rows = a.plan.short_rows;
  a.scale = (float)(1.4426950408889634074 / (d.D == 64 ? 8.0 : d.D == 256 ? 16.0 : 11.313708498984760390));
  return launch_attend(a, d, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

static ea_status append(const Dims& d, const ea_new_rows* r, AppendArgs a, size_t cache, void* q_out, void* stream) {
  if (!r || r->n_tokens < 0) return EA_ERR_INVALID_ARG;
  if (r->n_tokens > kAttendMaxTokens) return EA_ERR_UNSUPPORTED;
  const int64_t qd = (int64_t)d.Hq * d.D, kd = (int64_t)d.Hkv * d.D, per16 = d.dtype == EA_BF16 ? 8 : 4;
  const size_t es = d.dtype == EA_BF16 ? 2 : 4, n = (size_t)r->n_tokens;
  a.q_stride = r->q_stride ? r->q_stride : qd;
  a.k_stride = r->k_stride ? r->k_stride : kd;
  a.v_stride = r->v_stride ? r->v_stride : kd;
  const int64_t far = (int64_t)1 << 40;
  if (a.q_stride < qd || a.k_stride < kd || a.v_stride < kd || a.q_stride > far || a.k_stride > far || a.v_stride > far) return EA_ERR_INVALID_ARG;
  if (a.q_stride % per16 || a.k_stride % per16 || a.v_stride % per16) return EA_ERR_INVALID_ARG;
  if (!aligned(a.k_cache, 16) || !aligned(a.v_cache, 16) || a.k_cache == a.v_cache) return EA_ERR_INVALID_ARG;
  if (overlap(a.k_cache, cache, a.v_cache, cache)) return EA_ERR_INVALID_ARG;
  if (r->q && !r->inv_freq) return EA_ERR_INVALID_ARG;
  if (n == 0) return EA_OK;
  if (!aligned(r->k, 16) || !aligned(r->v, 16) || (r->q && (!aligned(r->q, 16) || !aligned(q_out, 16)))) return EA_ERR_INVALID_ARG;
  if (r->inv_freq && (!aligned(r->inv_freq, 8) || !aligned(r->pos, 4))) return EA_ERR_INVALID_ARG;
  const void* in[3] = {r->q, r->k, r->v};
  const size_t bytes[3] = {r->q ? ((n - 1) * a.q_stride + qd) * es : 0, ((n - 1) * a.k_stride + kd) * es, ((n - 1) * a.v_stride + kd) * es};
  const size_t q_bytes = r->q ? n * qd * es : 0;
  for (int i = 0; i < 3; ++i) {
    if (overlap(in[i], bytes[i], a.k_cache, cache) || overlap(in[i], bytes[i], a.v_cache, cache)) return EA_ERR_INVALID_ARG;
    const bool itself = i == 0 && q_out == r->q && a.q_stride == qd;
    if (!itself && overlap(in[i], bytes[i], q_out, q_bytes)) return EA_ERR_INVALID_ARG;
  }
  if (overlap(q_out, q_bytes, a.k_cache, cache) || overlap(q_out, q_bytes, a.v_cache, cache)) return EA_ERR_INVALID_ARG;
  a.q = r->q; a.k = r->k; a.v = r->v; a.q_out = q_out; a.pos = r->pos; a.inv_freq = r->inv_freq;
  a.B = d.B; a.Hq = d.Hq; a.Hkv = d.Hkv; a.n_tokens = (int)n; a.rope_layout = d.rope_layout;
  return launch_append(a, d, (hipStream_t)stream) == hipSuccess ? EA_OK : EA_ERR_DEVICE;
}

static ea_status append_heads(const Dims& d, const ea_new_rows* rows, const int32_t* cu_tokens, const int32_t* lengths, void* k, void* v,
                              const float* k_scale, const float* v_scale, int64_t n_cap, void* q_out, void* stream) {
  if (!aligned(cu_tokens, 4) || !aligned(lengths, 4) || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  if ((k_scale && !aligned(k_scale, 4)) || (v_scale && !aligned(v_scale, 4))) return EA_ERR_INVALID_ARG;
  AppendArgs a = {};
  a.k_cache = k; a.v_cache = v; a.cu = cu_tokens; a.lens = lengths; a.n_cap = n_cap; a.k_scale = k_scale; a.v_scale = v_scale;
  return append(d, rows, a, (size_t)d.units() * n_cap * d.D * d.esize(), q_out, stream);
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
  return make_attend_plan(d, n, step->n_tokens, step->max_new, kPlanCus).total;
}

ea_status ea_attend(const ea_params* p, const void* q, const ea_step* step, const void* k, const void* v,
                    const int32_t* lengths, int64_t n, int64_t n_cap, void* out, float* lse, void* ws, size_t ws_bytes,
                    void* stream) {
  Dims d;
  const ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  if (n > n_cap || n_cap < 1 || n_cap > ((int64_t)1 << 40)) return EA_ERR_INVALID_ARG;
  return attend(d, q, step, k, v, nullptr, nullptr, nullptr, lengths, true, n, n_cap, out, lse, ws, ws_bytes, stream);
}

ea_status ea_attend_paged(const ea_params* p, const void* q, const ea_step* step, const void* k_pool, const void* v_pool,
                          const ea_paged* pg, const int32_t* lengths, int64_t n, void* out, float* lse, void* ws,
                          size_t ws_bytes, void* stream) {
  Dims d;
  ea_status s = check_params(p, &d);
  if (s != EA_OK) return s;
  PageMap pm;
  if ((s = check_paged(d, pg, n, &pm)) != EA_OK) return s;
  return attend(d, q, step, k_pool, v_pool, &pm, nullptr, nullptr, lengths, false, n, 0, out, lse, ws, ws_bytes, stream);
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
  return attend(d, q, step, k8, v8, nullptr, k_scale, v_scale, lengths, true, n, n_cap, out, lse, ws, ws_bytes, stream);
}

}  // extern "C"
