// Instantiations of pack_short.hpp.
#include "pack_short.hpp"

namespace gt {

// head dims 8 and 16 run on 32-wide tiles whose extra features are zero
hipError_t launch_pack_short_bf16(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s) {
  switch (d) {
    case 8: return launch_pack_short<Bf16Pack<32, 8>>(a, cap, drop, s);
    case 16: return launch_pack_short<Bf16Pack<32, 16>>(a, cap, drop, s);
    case 32: return launch_pack_short<Bf16Pack<32, 32>>(a, cap, drop, s);
    default: return launch_pack_short<Bf16Pack<64, 64>>(a, cap, drop, s);
  }
}

}  // namespace gt
