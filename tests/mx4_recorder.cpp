// The launchers of kd_ops.h without a device, for kd_ops_api.cpp compiled next to this
// file: they launch nothing. Pointers are never dereferenced.
#include "../paper_2608_03796_amd/csrc/kd_ops.h"

extern "C" {
int kd_launch_mx4_write(const void*, int, int64_t, uint8_t*, uint8_t*, void*) { return 0; }
int kd_launch_mx4_read(const uint8_t*, const uint8_t*, int, int64_t, void*, void*) { return 0; }
int kd_launch_mx4_logits(const KdMx4Args*, void*) { return 0; }
int kd_launch_topk(const KdTopkArgs*, void*) { return 0; }
int kd_launch_cache_read(const KdCacheReadArgs*, void*) { return 0; }
int kd_launch_ckpt_write(const void*, int, int64_t, uint8_t*, uint8_t*, void*) { return 0; }
int kd_launch_ckpt_read(const uint8_t*, const uint8_t*, int, int64_t, void*, void*) { return 0; }
int kd_launch_verify(const KdVerifyArgs*, void*) { return 0; }

// the plan of a product: kind, nb, r, ks, tok, splits, rows, bytes
void rec_plan(int64_t N, int64_t D, int64_t V, int dtype, int64_t ld, int64_t* out) {
  const KdMx4Plan p = kd_mx4_plan(N, D, V, dtype, ld);
  const int64_t v[8] = {p.kind, p.nb, p.r, p.ks, p.tok, p.splits, p.rows, (int64_t)p.total};
  for (int i = 0; i < 8; ++i) out[i] = v[i];
}
}
