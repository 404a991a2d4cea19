// Kernels with the relative position bias and dropout, see sigattn_mod.hpp.
#include "sigattn_mod_launch.hpp"

namespace sigattn {
namespace mod {

int fwd_rel_dropout(const Params &p, const Extra &x, int d, hipStream_t stream) { return launch_fwd<true, true>(p, x, d, stream); }
int bwd_rel_dropout(const Params &kv, const Params &q, const Extra &x, int d, hipStream_t stream) { return launch_bwd<true, true>(kv, q, x, d, stream); }

}  // namespace mod
}  // namespace sigattn
