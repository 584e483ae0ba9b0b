// fp32 instantiations of pack_fwd.hpp.
#include "pack_fwd.hpp"

namespace gt {

hipError_t launch_pack_fwd_f32(const PackArgs& a, int d, bool cap, bool drop, hipStream_t s) {
  switch (d) {
    case 8: return launch_pack_fwd<F32Pack<8>>(a, cap, drop, s);
    case 16: return launch_pack_fwd<F32Pack<16>>(a, cap, drop, s);
    case 32: return launch_pack_fwd<F32Pack<32>>(a, cap, drop, s);
    default: return launch_pack_fwd<F32Pack<64>>(a, cap, drop, s);
  }
}

}  // namespace gt
