/* C99 client of the calls that fill caches and of 4-bit caches: struct layouts, refusals
 * and workspace sizes (no device is needed). Exits non-zero on the first failed check. */
#include <stddef.h>
#include <stdio.h>
#include <string.h>

#include "visionpulse.h"

static int failures = 0;
#define CHECK(cond)                                                   \
  do {                                                                \
    if (!(cond)) {                                                    \
      fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
      ++failures;                                                     \
    }                                                                 \
  } while (0)

int main(void) {
  static int lens[2], off[3];
  vp_shape s;
  vp_layout l;
  vp_rope r;
  vp_tokens t;
  vp_kv4 c;
  vp_window w;
  size_t bytes = 1;
  char* p = (char*)(1 << 20); /* an aligned address that nothing dereferences */
  memset(&s, 0, sizeof(s));
  memset(&l, 0, sizeof(l));
  memset(&r, 0, sizeof(r));
  memset(&t, 0, sizeof(t));
  memset(&c, 0, sizeof(c));
  memset(&w, 0, sizeof(w));
  s.batch = 2;
  s.n_q_heads = 28;
  s.n_kv_heads = 4;
  s.head_dim = 128;
  s.dtype = VP_BF16;
  s.max_seq_len = 4096;
  s.max_vis = s.max_segs = s.k_cap = 1;
  s.kv_stride_s = 128;
  s.kv_stride_h = 4096 * 128;
  s.kv_stride_b = 4 * s.kv_stride_h;
  l.seq_len = lens;
  r.cos_sin = (const float*)p;
  r.n_pos = 16;
  r.rot_dim = 128;
  r.n_axes = 1;
  t.q = t.k = t.v = p;
  t.q_stride = t.k_stride = t.v_stride = 36 * 128;
  t.new_off = off;
  t.n_tokens = 3;
  c.k_codes = p;
  c.k_scales = p;
  c.v_codes = p + 4096;
  c.v_scales = p + 4096;
  c.code_stride_h = 4096 * 64;
  c.code_stride_b = 4 * c.code_stride_h;
  c.scale_stride_h = 4096 * 4;
  c.scale_stride_b = 4 * c.scale_stride_h;
  printf("vp_rope %zu %zu %zu, vp_tokens %zu %zu, vp_kv4 %zu %zu\n", sizeof(vp_rope), offsetof(vp_rope, pos),
         offsetof(vp_rope, section), sizeof(vp_tokens), offsetof(vp_tokens, n_tokens), sizeof(vp_kv4),
         offsetof(vp_kv4, scale_stride_h));

  CHECK(vp_append_kv(NULL, &l, &r, &t, p, p, p + 4096, NULL) == VP_ERR_NULL);
  CHECK(vp_append_kv(&s, NULL, &r, &t, p + 64, p, p + 4096, NULL) == VP_ERR_NULL);
  CHECK(vp_append_kv(&s, &l, &r, NULL, p + 64, p, p + 4096, NULL) == VP_ERR_NULL);
  CHECK(vp_append_kv(&s, &l, &r, &t, NULL, p, p + 4096, NULL) == VP_ERR_NULL);
  CHECK(vp_append_kv(&s, &l, &r, &t, p + 64, p, p, NULL) == VP_ERR_SHAPE);
  r.rot_dim = 40;
  CHECK(vp_append_kv(&s, &l, &r, &t, p + 64, p, p + 4096, NULL) == VP_ERR_SHAPE);
  CHECK(strlen(vp_last_error()) > 0);
  r.rot_dim = 128;
  t.n_tokens = 0; /* nothing to append: nothing is enqueued */
  CHECK(vp_append_kv(&s, &l, &r, &t, p + 64, p, p + 4096, NULL) == VP_OK);
  CHECK(vp_append_kv4(&s, &l, NULL, &t, p + 64, &c, NULL) == VP_OK);
  t.n_tokens = 3;
  CHECK(vp_append_kv4(&s, &l, &r, &t, p + 64, NULL, NULL) == VP_ERR_NULL);
  c.code_stride_h -= 16;
  CHECK(vp_append_kv4(&s, &l, &r, &t, p + 64, &c, NULL) == VP_ERR_SHAPE);
  c.code_stride_h += 16;
  c.scale_stride_b = (int64_t)1 << 62; /* (as far apart as can be) */
  CHECK(vp_append_kv4(&s, &l, &r, &t, NULL, &c, NULL) == VP_ERR_NULL);
  c.scale_stride_b = 4 * c.scale_stride_h;
  CHECK(vp_kv4_read(&s, &l, &c, NULL, NULL, p, NULL) == VP_ERR_NULL);
  CHECK(vp_kv4_workspace_size(&s, &w, &bytes) == VP_OK && bytes > 0 && bytes % 256 == 0);
  CHECK(vp_kv4_workspace_size(&s, &w, NULL) == VP_ERR_NULL);
  CHECK(vp_kv4_decode_attn(&s, &l, &w, p, &c, p, NULL, 0, NULL) == VP_ERR_WORKSPACE);
  w.window = -1;
  CHECK(vp_kv4_decode_attn(&s, &l, &w, p, &c, p, p, bytes, NULL) == VP_ERR_RANGE);
  if (failures == 0) printf("all checks passed\n");
  return failures != 0;
}
