// Host-only stand-ins for the kernel launchers of the cached decoding, linked
// with its ABI layer (abi_cache.cpp) in the sanitizer build of
// tests/test_cache_host.py: a call that validation lets through is counted.
#include "../paper_2607_29221_amd/csrc/cache.h"

int g_launches = 0;

namespace mosaic {
hipError_t launch_cache_append(const AppendLaunch&, hipStream_t) { ++g_launches; return hipSuccess; }
int64_t cache_attend_workspace(const CacheView& c, int32_t heads, int64_t max_len, int32_t) {
  return (int64_t)c.batch * heads * max_len * 4;
}
hipError_t launch_cache_attend(const AttendLaunch&, hipStream_t) { ++g_launches; return hipSuccess; }
int64_t cache_evict_workspace(const CacheView& c, int64_t max_len, int64_t) { return (int64_t)c.batch * max_len * 4; }
hipError_t launch_cache_evict(const EvictLaunch&, hipStream_t) { ++g_launches; return hipSuccess; }
}  // namespace mosaic
