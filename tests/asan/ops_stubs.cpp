// Host-only stand-ins for the launchers of forge_ops_api.cpp, so that it can be built with g++
// and AddressSanitizer for its boundary tests, which never reach a launch.
#include <cstdio>
#include <cstdlib>

#include "forge_ops_internal.h"

namespace forge_impl {

[[noreturn]] static void unreachable(const char *what)
{
    std::fprintf(stderr, "launch stub reached: %s\n", what);
    std::abort();
}

hipError_t launch_rmsnorm(const NormArgs &, hipStream_t) { unreachable("launch_rmsnorm"); }
hipError_t launch_rmsnorm_backward(const NormGradArgs &, hipStream_t) { unreachable("launch_rmsnorm_backward"); }
hipError_t launch_grad_norm(const MtTable &, float, float *, double *, hipStream_t) { unreachable("launch_grad_norm"); }
hipError_t launch_adamw_multi(const MtTable &, const MtHyper &, const float *, hipStream_t)
{
    unreachable("launch_adamw_multi");
}

}  // namespace forge_impl
