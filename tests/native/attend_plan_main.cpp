// Host-only driver: what an attention call with masks launches.  It follows from bounds of what is cached, never from how much room a
// call has for tokens.
#include <stdio.h>
#include <string.h>

#include <initializer_list>

#include "../../paper_2510_00636_amd/csrc/ea_common.h"

static int failures = 0;
#define CHECK(cond, ...)                                                         \
  do {                                                                           \
    if (!(cond) && ++failures <= 20) {                                           \
      fprintf(stderr, "%s:%d: check failed: %s: ", __FILE__, __LINE__, #cond);   \
      fprintf(stderr, __VA_ARGS__);                                              \
      fprintf(stderr, "\n");                                                     \
    }                                                                            \
  } while (0)

static ea_params params(int B, int hq, int hkv, int d, int dtype) {
  ea_params p;
  memset(&p, 0, sizeof p);
  p.batch = B; p.n_q_heads = hq; p.n_kv_heads = hkv; p.head_dim = d; p.dtype = (ea_dtype)dtype;
  p.q_is_rotated = 1; p.horizon_T = 512;
  return p;
}

int main() {
  int with = 0, without = 0;
  for (int d : {64, 128, 256})
    for (int kind = 0; kind < 4; ++kind)       // bf16, 8 bits with a scale per head, MX rows, fp32
      for (int B : {1, 2, 16, 48, 300})
        for (int hkv : {1, 4, 8})
          for (int G : {1, 4, 5, 40})
            for (int64_t n : {(int64_t)0, (int64_t)100, (int64_t)1024, (int64_t)2048, (int64_t)16384, (int64_t)16385, (int64_t)131072})
              for (int64_t most : {(int64_t)1, (int64_t)16, (int64_t)61, (int64_t)200}) {
                const bool f32 = kind == 3;
                const ea_params p = params(B, hkv * G, hkv, d, f32 ? EA_F32 : EA_BF16);
                ea::Dims dims;
                CHECK(ea::check_params(&p, &dims) == EA_OK, "B %d heads %d", B, hkv * G);
                dims.kv_fp8 = kind == 1;
                const bool mx = kind == 2;
                const int64_t limit = d == 256 && (kind == 1 || mx) ? 16384 : 131072;
                const bool few = n <= 16384 && (int64_t)B * hkv * n <= limit;
                bool rows = false;
                for (int64_t room : {B * most, B * most + 1, B * most + 1000}) {
                  const ea::AttendPlan t = ea::make_attend_plan(dims, n, room, most, 256, mx, true), c = ea::make_attend_plan(dims, n, room, most, 256, mx, false);
                  CHECK(t.tile == c.tile && t.rows == (c.rows && !(c.tile && few)), "d %d kind %d B %d hkv %d G %d n %ld most %ld", d, kind, B, hkv, G, (long)n, (long)most);
                  CHECK(t.rows || t.tile, "nothing is launched");
                  if (room > B * most) CHECK(t.rows == (int)rows, "room for %ld tokens", (long)room);
                  rows = t.rows;
                  ++(t.rows ? with : without);
                }
              }
  CHECK(with > 1000 && without > 1000, "%d and %d plans", with, without);
  if (failures) {
    fprintf(stderr, "%d check(s) failed\n", failures);
    return 1;
  }
  printf("attention plans follow from what is cached\n");
  return 0;
}
