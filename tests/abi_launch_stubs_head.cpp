// Host-only stand-ins for the launchers of tmamba_head.h's kernels, linked with
// abi_head.cpp into a sanitizer build of its argument checks: reaching one is a
// failure.  The workspace sizes are simple functions of the sizes.
#include <cstdio>
#include <cstdlib>

#include "../paper_2606_18114_amd/csrc/head.hpp"

namespace tmk {

[[noreturn]] static void reached(const char* name) {
  std::fprintf(stderr, "launcher %s reached in the host-only build\n", name);
  std::abort();
}

int64_t head_loss_bytes(int64_t T, int64_t V, int64_t D) { return 256 * (T + V + D); }
hipError_t launch_head_loss(const HeadIn&, const void*, int, float*, float*, void*, hipStream_t) {
  reached("head_loss");
}
int64_t head_loss_bwd_bytes(int64_t T, int64_t V, int64_t D) { return 256 * (T + V + D); }
hipError_t launch_head_loss_bwd(const HeadIn&, const float*, const float*, uint16_t*, void*, int,
                                bool, void*, hipStream_t) {
  reached("head_loss_bwd");
}
hipError_t launch_block_norm(const float*, const float*, int64_t, int, const float*, float, float*,
                             uint16_t*, hipStream_t) {
  reached("block_norm");
}
int64_t block_norm_bwd_bytes(int64_t T, int64_t d) { return 256 * (T + d); }
hipError_t launch_block_norm_bwd(const float*, int64_t, int, const float*, float, const uint16_t*,
                                 const float*, float*, float*, void*, hipStream_t) {
  reached("block_norm_bwd");
}

}  // namespace tmk
