// Host helpers of the library's translation units: argument checks, the order of a launch's workgroups, the launch itself.
#pragma once
#include "sigattn_kernels.hpp"
#include "sigmoid_attn.h"

namespace sigattn {

inline int check_shape(int B, int N, int H, int d) {
    if (B <= 0 || N <= 0 || H <= 0) return SIGATTN_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return SIGATTN_ERR_UNSUPPORTED_D;
    if ((long long)B * H > 2147483647LL) return SIGATTN_ERR_TOO_LARGE;     // grid.x limit
    if ((long long)B * N * H * d >= (1LL << 40)) return SIGATTN_ERR_TOO_LARGE;
    if ((long long)H * d > (1LL << 20)) return SIGATTN_ERR_TOO_LARGE;      // 32-bit lane offsets within one streamed tile
    if (B > 256 && (long long)N > 262144LL) return SIGATTN_ERR_TOO_LARGE;  // a documented limit; the work mapping no longer needs it
    return SIGATTN_OK;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Work mapping of a launch of `wgs` workgroups (two to a CU, 512 in flight): 1 = batch order, 0 = longest sequences
// first.  Ranking B sequences costs every workgroup about 0.08 B us of the 5 us + 0.9 us per streamed 64-row tile
// it lives (measured with the wavefronts of both workgroups ranking at once); batch order costs about half a
// workgroup's life at the end of the launch, so 0.5 / (wgs / 512) of its time.  Batch order where that is less,
// or where the ranking has no class for every tile count.  Measured, sorted against batch order, us: dK/dV + dQ
// at B = 512, N = 512: 2106 / 1850; B = 32, H = 32, N = 512: 225 / 191; B = 16, H = 32, N = 1024: 326 / 309; B = 16, H = 12,
// N = 4096 (just below the line): 951 / 946; B = 24, H = 12, N = 4096: 2179 / 2182; B = 4, H = 32, N = 4096: 953 / 972;
// B = 8, H = 12, N = 2048: 125 / 132; forward at B = 24, H = 12, N = 1500: 72 / 78.
// The host does not know the lengths.  Near the line, a batch of 64-row sequences with a long one at its end (or every
// tenth) loses by batch order what other spreads gain: forward at B = 40, H = 12, N = 1000 one 30 / 35, every tenth 37 / 42,
// uniform 90 / 87, lognormal 31 / 24, all valid 153 / 142; backward 80 / 55, 114 / 79, 299 / 274, 88 / 49, 543 / 500.
inline int batch_order(const Params &p, long long wgs, int owner_rows) {
    if (p.B > MAP_WAVE_B && ((long long)p.N + owner_rows - 1) / owner_rows > MAP_CLASSES) return 1;
    return p.B * wgs > 16000 + 45LL * p.N_str;
}

template <class Kern, class... Args>
int enqueue(Kern kern, long long wgs, int threads, size_t lds, hipStream_t stream, Args... args) {
    if (wgs > 2147483647LL) return SIGATTN_ERR_TOO_LARGE;
    if (lds > 65536) {   // more dynamic LDS than the default limit: opt in (idempotent, host-side only)
        if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                (int)lds) != hipSuccess)
            return SIGATTN_ERR_LAUNCH;
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs, 1, 1), dim3(threads, 1, 1), lds, stream, args...);
    return hipGetLastError() == hipSuccess ? SIGATTN_OK : SIGATTN_ERR_LAUNCH;
}

template <class C>
long long tiles_of(const Params &p) {                                       // one workgroup per owner tile
    return ((long long)p.N + C::BM - 1) / C::BM * p.B * p.H;
}

}  // namespace sigattn
