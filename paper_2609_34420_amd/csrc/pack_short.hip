// Instantiations of pack_short.hpp.
#include "pack_short.hpp"

namespace gt {

// head dims 8 and 16 run on 32-wide tiles whose extra features are zero
hipError_t launch_pack_short_bf16(const PackArgs& a, int d, int blocks, bool cap, bool drop, hipStream_t s) {
  switch (d + (blocks == 4)) {
    case 8: return launch_pack_short<Bf16Pack<32, 8>, 2>(a, cap, drop, s);
    case 9: return launch_pack_short<Bf16Pack<32, 8>, 4>(a, cap, drop, s);
    case 16: return launch_pack_short<Bf16Pack<32, 16>, 2>(a, cap, drop, s);
    case 17: return launch_pack_short<Bf16Pack<32, 16>, 4>(a, cap, drop, s);
    case 32: return launch_pack_short<Bf16Pack<32, 32>, 2>(a, cap, drop, s);
    case 33: return launch_pack_short<Bf16Pack<32, 32>, 4>(a, cap, drop, s);
    default: return launch_pack_short<Bf16Pack<64, 64>, 2>(a, cap, drop, s);
  }
}

}  // namespace gt
