// Host-only stand-ins for the launchers of the sequence kernels, linked with
// abi_seq.cpp into a sanitizer build of its argument checks (as
// abi_launch_stubs.cpp does for the other calls): reaching one is a failure.
// The workspace sizes are simple functions of the sizes.
#include <cstdio>
#include <cstdlib>

#include "../paper_2606_18114_amd/csrc/launchers.hpp"
#include "../paper_2606_18114_amd/csrc/seq_launch.hpp"

namespace tmk {

[[noreturn]] static void reached(const char* name) {
  std::fprintf(stderr, "launcher %s reached in the host-only build\n", name);
  std::abort();
}

hipError_t launch_seq_conv(const SeqIn&, const float*, const float*, const uint16_t*, const int*,
                           uint16_t*, uint16_t*, hipStream_t) {
  reached("seq_conv");
}
int64_t seq_conv_bwd_bytes(int64_t T, int64_t nheads) { return 256 * (T + nheads); }
hipError_t launch_seq_conv_bwd(const SeqIn&, const float*, const float*, const uint16_t*, void*,
                               float*, float*, void*, hipStream_t) {
  reached("seq_conv_bwd");
}
hipError_t launch_seq_norm(const SeqIn&, const uint16_t*, const float*, float, uint16_t*,
                           hipStream_t) {
  reached("seq_norm");
}
int64_t seq_norm_bwd_bytes(int64_t T, int64_t nheads) { return 256 * (T + nheads); }
hipError_t launch_seq_norm_bwd(const SeqIn&, const uint16_t*, const float*, float, const uint16_t*,
                               void*, uint16_t*, float*, void*, hipStream_t) {
  reached("seq_norm_bwd");
}
int64_t seq_scan_bytes(int64_t T, int64_t nheads) {
  return T > 512 ? 256 * (T + nheads) : 0;
}
hipError_t launch_seq_scan(const SeqIn&, const uint16_t*, const float*, const float*, const float*,
                           const uint16_t*, uint16_t*, uint16_t*, void*, hipStream_t) {
  reached("seq_scan");
}
int64_t seq_scan_bwd_bytes(int64_t T, int64_t, int64_t nheads) { return 256 * (T + nheads); }
hipError_t launch_seq_scan_bwd(const SeqIn&, const uint16_t*, const float*, const float*,
                               const float*, const uint16_t*, void*, uint16_t*, float*, float*,
                               float*, void*, hipStream_t) {
  reached("seq_scan_bwd");
}
hipError_t launch_embed(const void*, bool, int64_t, const void*, int, int64_t, int64_t, float,
                        float*, hipStream_t) {
  reached("embed");
}
int64_t embed_bwd_bytes(int64_t T, int64_t V, int64_t) { return 256 * (T + V); }
hipError_t launch_embed_bwd(const void*, bool, int64_t, const float*, int64_t, int64_t, float,
                            float*, bool, void*, hipStream_t) {
  reached("embed_bwd");
}

}  // namespace tmk
