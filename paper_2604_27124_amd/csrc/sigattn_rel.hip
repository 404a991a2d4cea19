// Kernels with the relative position bias, see sigattn_mod.hpp.
#include "sigattn_mod_launch.hpp"

namespace sigattn {
namespace mod {

int fwd_rel(const Params &p, const Extra &x, int d, hipStream_t stream) { return launch_fwd<true, false>(p, x, d, stream); }
int bwd_rel(const Params &kv, const Params &q, const Extra &x, int d, hipStream_t stream) { return launch_bwd<true, false>(kv, q, x, d, stream); }

}  // namespace mod
}  // namespace sigattn
