// Kernels with dropout of the attention weights, d = 128: see sigattn_mod.hpp.
#include "sigattn_mod_launch.hpp"

namespace sigattn {
namespace mod {

int fwd_dropout_128(const Params &p, const Extra &x, hipStream_t stream) { return launch_fwd<128, false, true>(p, x, stream); }
int bwd_dropout_128(const Params &kv, const Params &q, const Extra &x, hipStream_t stream) { return launch_bwd<128, false, true>(kv, q, x, stream); }

}  // namespace mod
}  // namespace sigattn
