// Launches of sigattn_rel_few.hpp.
#include "sigattn_host.hpp"
#include "sigattn_rel_few.hpp"

namespace sigattn {
namespace few {

template <int D, int R>
static int run(const Few &f, hipStream_t stream) {
    const long long heads = (long long)f.p.B * f.p.H * f.groups;
    if (const int e = enqueue(sigattn_rel_few<D, R>, heads * f.splits, THREADS, 0, stream, f)) return e;
    if (f.splits == 1) return SIGATTN_OK;
    return enqueue(sigattn_rel_few_join<D, R>, (heads * (R * D) + 255) / 256, 256, 0, stream, f);
}

template <int D>
static int rows(const Few &f, hipStream_t stream) {
    return f.p.N == 1 ? run<D, 1>(f, stream) : f.p.N == 2 ? run<D, 2>(f, stream) : f.p.N <= 4 ? run<D, 4>(f, stream) : run<D, 8>(f, stream);
}

int launch(const Few &f, int d, hipStream_t stream) { return d == 64 ? rows<64>(f, stream) : rows<128>(f, stream); }

}  // namespace few
}  // namespace sigattn
