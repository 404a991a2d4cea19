// Forward pass with a relative position bias for a few queries a sequence, 64 at most: single tokens against a long context.
//
// Every key and value is used by few queries, so the call is bound by reading them once, and matrix instructions, which take
// 32 queries at a time, would mostly multiply padding.  A wave reads whole rows (d = 64: eight lanes of 16 bytes a row, eight rows a load; d = 128: 16 and
// four), four loads of each tensor in flight, multiplies on the vector unit (dot products of bf16 pairs, exact products, fp32
// sums) and keeps one query row's share of O in eight registers a lane.  Scores and weights stay in fp32: the only rounding
// to fewer bits is that of O.  The bias of a chunk of keys lies in LDS by distance.
//
// A workgroup takes a (z, h), or one of `splits` parts of its keys; parts are added in a second launch, in order.
// One query, d = 64, B = 32, H = 12, up to 4096 keys (238 MB in all, ragged): 52 us, 4.6 TB/s; a large copy reaches 5.1.  With
// eight queries the vector unit bounds it (B = 8, 8192 keys: 57 us for what one query reads in 35).
#pragma once
#include "sigattn_mod.hpp"

namespace sigattn {
namespace few {

constexpr int NW = 8, THREADS = 64 * NW, MOST = 64;            // most: queries of a sequence, in groups of eight
constexpr int CHUNK = 2048;                                    // keys whose bias is in LDS

template <int CTRL>
__device__ __forceinline__ float dpp(const float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
// {lower half of the wave: a of both halves, upper half: b of both}; the same for pairs of rows of 16 lanes.
__device__ __forceinline__ float join32(const float a, const float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned x = r[0], y = r[1];
    return __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float join16(const float a, const float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned x = r[0], y = r[1];
    return __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
}
__device__ __forceinline__ float dot(const u32x4 a, const u32x4 b) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned x = a[i], y = b[i];
        s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, x), __builtin_bit_cast(bf16x2, y), s, false);
    }
    return s;
}

struct Few {
    Params p;                        // q, k, v, out0, seqlens (queries), seqlens_str (keys), bias, scale, B, N, N_str, H
    mod::Extra x;
    int splits, groups;              // parts of the keys; groups of R queries
    float *part;                     // [splits][B][H][groups][R][D] where there are several
};

template <int D, int R>
__global__ void __launch_bounds__(THREADS, 2) sigattn_rel_few(const Few f) {
    constexpr int LANES = D / 8, ROWS = 64 / LANES, U = 4, STEP = ROWS * U;        // lanes of a row; rows of a load; loads; keys of a wave's step
    __shared__ float bias[CHUNK + R];
    __shared__ float red[NW][R][D];
    const Params &p = f.p;
    const int zhg = blockIdx.x / f.splits, split = blockIdx.x % f.splits, zh = zhg / f.groups, r0 = zhg % f.groups * R, z = zh / p.H, h = zh % p.H;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane % LANES, row = lane / LANES;
    int nq = p.seqlens[z], ns = p.seqlens_str[z];
    nq = nq < 0 ? 0 : (nq > p.N ? p.N : nq);
    ns = ns < 0 ? 0 : (ns > p.N_str ? p.N_str : ns);
    int start = f.x.q_start ? f.x.q_start[z] : 0;
    start = start < -(1 << 29) ? -(1 << 29) : (start > (1 << 29) ? (1 << 29) : start);
    const size_t stride = (size_t)p.H * D;
    constexpr float LOG2E = 1.4426950408889634f;
    const float c1 = -p.scale * LOG2E;
    const float cb = __builtin_amdgcn_exp2f(__builtin_fminf(__builtin_fmaxf(-p.bias[z] * LOG2E, -126.0f), 126.0f));

    u32x4 q[R];
    float acc[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        q[r] = u32x4{0u, 0u, 0u, 0u};
        if (r0 + r < nq) q[r] = *reinterpret_cast<const u32x4 *>(p.q + ((size_t)z * p.N + r0 + r) * stride + (size_t)h * D + 8 * col);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] = 0.f;
    }
    // this part's keys: whole chunks' worth of wave steps
    const long long each = ((long long)ns + f.splits - 1) / f.splits, rounded = (each + STEP - 1) / STEP * STEP;
    const long long k_lo = rounded * split, k_hi = k_lo + rounded < ns ? k_lo + rounded : ns;
    const unsigned off = (unsigned)row * (unsigned)stride * 2u + 16u * col, load_bytes = (unsigned)ROWS * (unsigned)stride * 2u;
    const bf16_t *const k0 = p.k + (size_t)z * p.N_str * stride + (size_t)h * D, *const v0 = p.v + (size_t)z * p.N_str * stride + (size_t)h * D;

    for (long long base = k_lo; base < k_hi; base += CHUNK) {
        const int count = (int)(k_hi - base < CHUNK ? k_hi - base : CHUNK);
        __syncthreads();
        for (int e = threadIdx.x; e < count + R - 1; e += THREADS) {           // entry e: distance base + e - (R - 1) - r0 - start
            const int j = (int)base + e - (R - 1) - r0;
            int t = j - start;
            t = t < -f.x.reach ? -f.x.reach : (t > f.x.reach ? f.x.reach : t);
            int b = f.x.buckets[t + f.x.reach];
            b = b < 0 ? 0 : (b >= f.x.num_buckets ? f.x.num_buckets - 1 : b);
            bias[e] = (float)f.x.table[(size_t)b * p.H + h] * -LOG2E;
        }
        __syncthreads();
        for (int k = wave * STEP; k < count; k += NW * STEP) {
            const int left = count - k < STEP ? count - k : STEP;              // rows behind them are zeros, not read
            const int bytes = __builtin_amdgcn_readfirstlane(left * (int)stride * 2);
            const auto dk = __builtin_amdgcn_make_buffer_rsrc(uniform_ptr(k0 + (size_t)(base + k) * stride), 0, bytes, 0x00027000);
            const auto dv = __builtin_amdgcn_make_buffer_rsrc(uniform_ptr(v0 + (size_t)(base + k) * stride), 0, bytes, 0x00027000);
            u32x4 a[U], b[U];
#pragma unroll
            for (int u = 0; u < U; ++u) a[u] = __builtin_amdgcn_raw_buffer_load_b128(dk, (int)off, u * (int)load_bytes, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) b[u] = __builtin_amdgcn_raw_buffer_load_b128(dv, (int)off, u * (int)load_bytes, 0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = u * ROWS + row;                                  // key of this lane in the step
                float w[R];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float s = dot(q[r], a[u]);                                 // over the lanes of a row: sums in each of them
                    s += dpp<0xB1>(s);                                         // quad_perm 1, 0, 3, 2
                    s += dpp<0x4E>(s);                                         // quad_perm 2, 3, 0, 1
                    s += dpp<0x141>(s);                                        // half mirror: the other four of eight
                    if (D == 128) s += dpp<0x140>(s);                          // mirror: the other eight of 16
                    const float t = __builtin_fmaf(s, c1, bias[k + j + R - 1 - r]);
                    const float y = __builtin_amdgcn_rcpf(__builtin_fmaf(cb, __builtin_amdgcn_exp2f(t), 1.0f));
                    w[r] = j < left ? y : 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned two = b[u][i];
                    const float lo = __builtin_bit_cast(float, two << 16), hi = __builtin_bit_cast(float, two & 0xFFFF0000u);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        acc[r][2 * i] = __builtin_fmaf(w[r], lo, acc[r][2 * i]);
                        acc[r][2 * i + 1] = __builtin_fmaf(w[r], hi, acc[r][2 * i + 1]);
                    }
                }
            }
        }
    }
    // over the rows of the wave: every lane ends with two of its eight columns
    const int first = 2 * ((lane >> 4) & 1) + 4 * (lane >> 5);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float a[4], b[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = join32(acc[r][e], acc[r][e + 4]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            b[e] = join16(a[e], a[e + 2]);
            if (D == 64) b[e] += dpp<0x128>(b[e]);                             // the other row of these 16 lanes
        }
        if (D == 128 || (lane & 8) == 0) {
            red[wave][r][8 * col + first] = b[0];
            red[wave][r][8 * col + first + 1] = b[1];
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < R * D; e += THREADS) {
        const int r = e / D, c = e % D;
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) t += red[w][r][c];
        if (f.splits > 1) f.part[((size_t)split * p.B * p.H * f.groups + zhg) * (R * D) + e] = t;
        else if (r0 + r < p.N) p.out0[((size_t)z * p.N + r0 + r) * stride + (size_t)h * D + c] = (bf16_t)(r0 + r < nq ? t : 0.f);
    }
}

// The parts of a (z, h), in order.
template <int D, int R>
__global__ void __launch_bounds__(256) sigattn_rel_few_join(const Few f) {
    const Params &p = f.p;
    const size_t all = (size_t)p.B * p.H * f.groups * (R * D), at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= all) return;
    const size_t zhg = at / (R * D), zh = zhg / f.groups;
    const int r = (int)(zhg % f.groups) * R + (int)(at % (R * D)) / D, c = (int)(at % D);
    const int z = (int)(zh / p.H), h = (int)(zh % p.H);
    int nq = p.seqlens[z];
    nq = nq < 0 ? 0 : (nq > p.N ? p.N : nq);
    float t = 0.f;
    for (int s = 0; s < f.splits; ++s) t += f.part[s * all + at];
    if (r < p.N) p.out0[((size_t)z * p.N + r) * (size_t)p.H * D + (size_t)h * D + c] = (bf16_t)(r < nq ? t : 0.f);
}

int launch(const Few &f, int d, hipStream_t stream);           // sigattn_rel_few.hip

}  // namespace few
}  // namespace sigattn
