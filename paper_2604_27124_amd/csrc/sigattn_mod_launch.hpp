// The kernels of sigattn_mod.hpp and their launches.  Each combination (bias, dropout, both) is a translation unit of its own.
#pragma once
#include "sigattn_host.hpp"
#include "sigattn_mod.hpp"

namespace sigattn {
namespace mod {

struct Scratch {
    MapScratch map;
    float ring[512 + 32];
};

template <int MODE, int D, int QB, int NW, int LD1, int LD2, int OCC, int RING, bool BIAS, bool DROP>
__global__ void __launch_bounds__(NW * 64, OCC) sigattn_mod(const Params p, const Extra x) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ Scratch s;
    using C = Cfg<MODE, D, QB, NW, 64, LD1, LD2, RING>;
    using M = Mods<MODE, QB, NW, BIAS, DROP, BIAS && MODE == DQ>;
    run_pass<MODE, D, QB, NW, 64, LD1, LD2, RING, false, M>(p, map_work<C::BM, C::THREADS>(p, blockIdx.x, s.map), smem, nullptr, M(p, x, s.ring));
}

// Both passes of the backward in one launch, as in sigattn_bwd_kernel (d = 64) and sigattn_half_bwd (d = 128).
template <int D, int NW, int LD, int LD_Q, int OCC, int RING_KV, int RING_Q, bool BIAS, bool DROP>
__global__ void __launch_bounds__(NW * 64, OCC) sigattn_mod_bwd(const Params kv, const Params q, const Extra x, const int q_first, const int first_tiles) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ Scratch s;
    using C = Cfg<DKDV, D, 1, NW, 64, LD, LD, RING_KV>;
    using MK = Mods<DKDV, 1, NW, BIAS, DROP, false>;
    using MQ = Mods<DQ, 1, NW, BIAS, DROP, BIAS>;
    const int id = blockIdx.x;
    Work w;
    bool is_kv;
    if (kv.in_order) {
        const int t_kv = owner_tiles<C::BM>(kv), t_q = owner_tiles<C::BM>(q);
        int tile;
        batch_order_tile(id, kv.H, t_kv + t_q, w.z, w.h, tile);
        is_kv = tile < t_kv;
        w.n = owner_length(is_kv ? kv : q, w.z);
        w.m0 = (is_kv ? tile : tile - t_kv) * C::BM;
        w.count = 1;
        w.share = w.shares = 0;
    } else {
        is_kv = (id < first_tiles) != (q_first != 0);
        const int rest = id < first_tiles ? id : id - first_tiles;
        w = is_kv ? map_work<C::BM, C::THREADS>(kv, rest, s.map) : map_work<C::BM, C::THREADS>(q, rest, s.map);
    }
    if (is_kv) run_pass<DKDV, D, 1, NW, 64, LD, LD, RING_KV, false, MK>(kv, w, smem, nullptr, MK(kv, x, s.ring));
    else run_pass<DQ, D, 1, NW, 64, LD, LD_Q, RING_Q, false, MQ>(q, w, smem, nullptr, MQ(q, x, s.ring));
}

template <int MODE, int D, int QB, int NW, int LD1, int LD2, int OCC, int RING, bool BIAS, bool DROP>
int launch_pass(Params p, const Extra &x, hipStream_t stream) {
    using C = Cfg<MODE, D, QB, NW, 64, LD1, LD2, RING>;
    const long long wgs = tiles_of<C>(p);
    p.in_order = batch_order(p, wgs, C::BM);
    return enqueue(sigattn_mod<MODE, D, QB, NW, LD1, LD2, OCC, RING, BIAS, DROP>, wgs, C::THREADS, C::LDS_BYTES, stream, p, x);
}

template <int D, int NW, int LD, int LD_Q, int OCC, int RING_KV, int RING_Q, bool BIAS, bool DROP>
int launch_joint(Params kv, Params q, const Extra &x, hipStream_t stream) {
    using C = Cfg<DKDV, D, 1, NW, 64, LD, LD, RING_KV>;
    using CQ = Cfg<DQ, D, 1, NW, 64, LD, LD_Q, RING_Q>;
    static_assert(C::BM == CQ::BM, "one tile height for both passes");
    const long long kv_tiles = tiles_of<C>(kv), q_tiles = tiles_of<C>(q);
    kv.in_order = q.in_order = batch_order(kv, kv_tiles + q_tiles, C::BM) || batch_order(q, kv_tiles + q_tiles, C::BM);
    const int q_first = kv.N_str < q.N_str;                    // the pass whose workgroups stream more rows starts
    return enqueue(sigattn_mod_bwd<D, NW, LD, LD_Q, OCC, RING_KV, RING_Q, BIAS, DROP>, kv_tiles + q_tiles, C::THREADS,
                   C::LDS_BYTES > CQ::LDS_BYTES ? C::LDS_BYTES : CQ::LDS_BYTES, stream, kv, q, x, q_first, (int)(q_first ? q_tiles : kv_tiles));
}

// The shapes, and the rules that choose them, are those of the plain calls, but for the backward pass: d = 64 has an operand ring of
// four in dK/dV too, which leaves the generator its registers (with eight they spill in the loop).  d = 128 with a bias has
// a ring of two in dQ (B = 8, H = 16, N = 2048: 1107 -> 1041 us of the backward pass; the sums' registers; what is left over goes through scratch, two
// instructions a tile with the bias alone and 23 with dropout too), and goes in one launch up to 256
// owner tiles of queries, where two launches would each leave CUs idle (us, one / two: B = 6, H = 4, 513 x 3001 138 / 237; B = 8, H = 16,
// N = 2048, 2048 tiles, 1243 / 1112).
inline long long tiles128(const Params &p) { return ((long long)p.N + 127) / 128 * p.B * p.H; }

template <int D, bool BIAS, bool DROP>
int launch_fwd(const Params &p, const Extra &x, hipStream_t stream) {
    if constexpr (D == 64) {
        if (p.N <= 128 || (long long)p.B * p.H * ((p.N + 255) / 256) <= 256) return launch_pass<FWD, 64, 1, 4, 72, 72, 2, 4, BIAS, DROP>(p, x, stream);
        return launch_pass<FWD, 64, 2, 4, 72, 72, 2, 4, BIAS, DROP>(p, x, stream);
    } else {
        if (tiles128(p) <= 256) return launch_pass<FWD, 128, 1, 4, 136, 144, 1, 4, BIAS, DROP>(p, x, stream);
        return launch_pass<FWD, 128, 1, 8, 136, 144, 1, 4, BIAS, DROP>(p, x, stream);
    }
}

template <int D, bool BIAS, bool DROP>
int launch_bwd(const Params &kv, const Params &q, const Extra &x, hipStream_t stream) {
    if constexpr (D == 64) {
        return launch_joint<64, 4, 72, 72, 2, 4, 4, BIAS, DROP>(kv, q, x, stream);
    } else {
        if (tiles128(kv) + tiles128(q) <= 512 || (BIAS && tiles128(q) <= 256)) return launch_joint<128, 4, 144, 136, 1, 4, 4, BIAS, DROP>(kv, q, x, stream);
        if (const int e = launch_pass<DKDV, 128, 1, 4, 144, 144, 1, 4, BIAS, DROP>(kv, x, stream)) return e;
        return launch_pass<DQ, 128, 1, 8, 144, 136, 1, BIAS ? 2 : 4, BIAS, DROP>(q, x, stream);
    }
}

// A translation unit for each, so that they are compiled side by side: sigattn_{rel,dropout,rel_dropout}_{64,128}.hip.
int fwd_rel_64(const Params &, const Extra &, hipStream_t);
int fwd_rel_128(const Params &, const Extra &, hipStream_t);
int fwd_dropout_64(const Params &, const Extra &, hipStream_t);
int fwd_dropout_128(const Params &, const Extra &, hipStream_t);
int fwd_rel_dropout_64(const Params &, const Extra &, hipStream_t);
int fwd_rel_dropout_128(const Params &, const Extra &, hipStream_t);
int bwd_rel_64(const Params &kv, const Params &q, const Extra &, hipStream_t);
int bwd_rel_128(const Params &kv, const Params &q, const Extra &, hipStream_t);
int bwd_dropout_64(const Params &kv, const Params &q, const Extra &, hipStream_t);
int bwd_dropout_128(const Params &kv, const Params &q, const Extra &, hipStream_t);
int bwd_rel_dropout_64(const Params &kv, const Params &q, const Extra &, hipStream_t);
int bwd_rel_dropout_128(const Params &kv, const Params &q, const Extra &, hipStream_t);

}  // namespace mod
}  // namespace sigattn
