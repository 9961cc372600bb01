// How the attention over 4 bits is dealt out, for tests/test_cache_attend_plan.py:
// the host code of csrc/cache_attend_e2m1.hip, compiled for the host alone.
#include "../paper_2607_29221_amd/csrc/cache_attend_e2m1.hip"

namespace mosaic {
namespace {
template <int XT, int DP> int lds_of(int tiles, bool accumulate) {
  return tiles == 2 ? Lds<XT, DP, 2, 16>::bytes(accumulate) + 2 * kWaves * kHeadTile * 8
                    : Lds<XT, DP, 1, 16>::bytes(accumulate) + kWaves * kHeadTile * 8;
}
template <int XT> void plan(const AttendLaunch& a, int32_t* out) {
  const Plan p = plan_for<XT>(a);
  out[0] = p.workgroups;
  out[1] = p.tile_groups;
  out[2] = a.c.head_dim <= 64    ? lds_of<XT, 64>(p.wave_tiles, a.accumulate)
           : a.c.head_dim <= 128 ? lds_of<XT, 128>(p.wave_tiles, a.accumulate)
                                 : lds_of<XT, 256>(1, a.accumulate);
  out[3] = plan_of(a.c, a.heads, a.max_len).workgroups;       // of the workspace
}
}  // namespace
}  // namespace mosaic

// out: workgroups per key/value head and block of query heads, such blocks, bytes of
// LDS of a workgroup, workgroups that the workspace has room for
extern "C" void attend_plan(int x_dtype, int batch, int heads, int kv_heads, int head_dim, int64_t max_len, int accumulate, int32_t* out) {
  mosaic::AttendLaunch a{};
  a.c.batch = batch;
  a.c.kv_heads = kv_heads;
  a.c.head_dim = head_dim;
  a.c.dtype = MOSAIC_E2M1;
  a.heads = heads;
  a.max_len = max_len;
  a.accumulate = accumulate;
  if (x_dtype == MOSAIC_F32) mosaic::plan<MOSAIC_F32>(a, out);
  else if (x_dtype == MOSAIC_BF16) mosaic::plan<MOSAIC_BF16>(a, out);
  else mosaic::plan<MOSAIC_F16>(a, out);
}
