// Host-only stand-ins for the launchers behind abi_cache_norm.cpp, beside those of
// cache_stub_launchers.cpp, in the sanitizer build of tests/test_cache_norm_host.py.
#include "../paper_2607_29221_amd/csrc/cache.h"

extern int g_launches;

namespace mosaic {
hipError_t launch_cache_read(const ReadLaunch&, hipStream_t) { ++g_launches; return hipSuccess; }
}  // namespace mosaic
