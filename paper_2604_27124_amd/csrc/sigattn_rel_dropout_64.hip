// Kernels with the relative position bias and dropout, d = 64: see sigattn_mod.hpp.
#include "sigattn_mod_launch.hpp"

namespace sigattn {
namespace mod {

int fwd_rel_dropout_64(const Params &p, const Extra &x, hipStream_t stream) { return launch_fwd<64, true, true>(p, x, stream); }
int bwd_rel_dropout_64(const Params &kv, const Params &q, const Extra &x, hipStream_t stream) { return launch_bwd<64, true, true>(kv, q, x, stream); }

}  // namespace mod
}  // namespace sigattn
