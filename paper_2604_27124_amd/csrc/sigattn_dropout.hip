// Kernels with dropout of the attention weights, see sigattn_mod.hpp.
#include "sigattn_mod_launch.hpp"

namespace sigattn {
namespace mod {

int fwd_dropout(const Params &p, const Extra &x, int d, hipStream_t stream) { return launch_fwd<false, true>(p, x, d, stream); }
int bwd_dropout(const Params &kv, const Params &q, const Extra &x, int d, hipStream_t stream) { return launch_bwd<false, true>(kv, q, x, d, stream); }

}  // namespace mod
}  // namespace sigattn
