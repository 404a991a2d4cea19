// Host side of the calls with a relative position bias and with dropout (include/sigmoid_attn.h), and the kernels that add up the
// gradient of the bias table.
#include "sigattn_mod_launch.hpp"
#include "sigattn_rel_few.hpp"

#include <cmath>

using namespace sigattn;
using mod::Extra;
using mod::RowSums;

namespace {

constexpr int MOST_REACH = 1 << 24, MOST_BUCKETS = 1 << 16, MOST_ROWS = 1 << 29;

struct Lengths {
    const int32_t *q, *k, *start;    // [B]; start may be null
    const float *bias;
    int L_q, L_k, H, B;
};

__device__ __forceinline__ int clamped(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

__device__ __forceinline__ int start_of(const Lengths &l, int z) { return l.start ? clamped(l.start[z], -(1 << 29), 1 << 29) : 0; }

// Sum over the rows of a sequence that have entry `c` of chunk `chunk`: of 32 queries each, from row `first` on every `step`.
__device__ __forceinline__ float sum_rows(const Lengths &l, const Extra &x, const int z, const int h, const int chunk, const int c, const bool far,
                                          const int first, const int step, const int entries) {
    const int blocks = (l.L_q + 31) / 32;
    const size_t stride = (size_t)(entries + mod::FAR);
    const int nq = clamped(l.q[z], 0, l.L_q), ns = clamped(l.k[z], 0, l.L_k);
    if (nq == 0 || ns == 0) return 0.f;
    const RowSums r(x.reach, start_of(l, z), blocks);
    const int k = r.first + chunk, key_blocks = 2 * ((ns + 63) / 64);
    // b = k + ob is a near block's, or b - 1 is (what the last near block leaves behind)
    int from = -k, to = key_blocks - k;                                        // key blocks 0 .. key_blocks - 1
    if (chunk > 0) ++to;                                                       // and the one behind, of diagonal k - 1
    if (k > r.last) { ++from; if (k > r.last + 1 || chunk == 0) to = from; }   // only as what is left
    const int all = (nq + 31) / 32;
    if (far) { from = 0; to = c < 2 ? all : 0; }
    from = from < 0 ? 0 : from;
    to = to > all ? all : to;
    const float *const rows = x.part + ((size_t)z * l.H + h) * blocks * stride + 32 * chunk + c;
    float t = 0.f;
    int ob = from + first;
    for (; ob + 3 * step < to; ob += 4 * step) {                               // four loads in flight
        const float a = rows[ob * stride], b = rows[(ob + step) * stride], e = rows[(ob + 2 * step) * stride], f = rows[(ob + 3 * step) * stride];
        t += (a + b) + (e + f);
    }
    for (; ob < to; ob += step) t += rows[ob * stride];
    // the rows are of dS / cb, without 1 / keep.  cb / keep may pass fp32 (cb is up to 2^126), where t is zero or nearly so: one after the other.
    const float cb = __builtin_amdgcn_exp2f(__builtin_fminf(__builtin_fmaxf(-l.bias[z] * 1.4426950408889634f, -126.0f), 126.0f));
    return t * cb * x.inv_keep;
}

// Sums over rows, in fixed order and without atomics.  Group s of `groups` takes sequences s, s + groups, ...: [group][H][entries + FAR].  A
// workgroup takes 32 entries of a head; of its eight groups of 32 lanes `seqs` take a sequence each, and the others share the
// rows of these.
__global__ void __launch_bounds__(256) sigattn_rel_rows(const Lengths l, const Extra x, const int groups, const int seqs) {
    __shared__ float s[8][32];
    const int entries = RowSums::entries(x.reach, l.L_q, l.L_k), chunks = entries / 32 + 1;
    const int chunk = blockIdx.x % chunks, rest = blockIdx.x / chunks, h = rest % l.H, group = rest / l.H;
    const int c = threadIdx.x & 31, mine = threadIdx.x >> 5, step = 8 / seqs;
    const bool far = chunk == chunks - 1;
    const size_t stride = (size_t)(entries + mod::FAR);
    float total = 0.f;
    for (long long z = group + (long long)groups * (mine % seqs); z < l.B; z += (long long)groups * seqs)
        total += sum_rows(l, x, (int)z, h, chunk, c, far, mine / seqs, step, entries);
    s[mine][c] = total;
    __syncthreads();
    if (mine == 0) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += s[i][c];
        x.by_distance[((size_t)group * l.H + h) * stride + 32 * chunk + c] = t;
    }
}

// dtable[b][h] for 16 buckets of a head: the entries of all groups (of one group where every sequence has a start of its own), a
// thousand at a time, with their buckets, in LDS; each wave goes through them for its four buckets.  (Sequences with starts follow each other here, about 1.7 us
// each: B = 256, H = 12, N = 512 backward 1182 us without starts, 1605 with; B = 1024, N = 128 558 and 2320.)  DIRECT: a few rows,
// taken as they are, without the launch above (B = 2, H = 2, N = 256: backward 19.7 -> 17.7 us); a group is a sequence then.
constexpr int TABLE_BUCKETS = 16, TABLE_ENTRIES = 1024, DIRECT_ROWS = 64;
template <bool DIRECT>
__global__ void __launch_bounds__(256) sigattn_rel_table(const Lengths l, const Extra x, const int groups, bf16_t *dtable) {
    __shared__ float value[TABLE_ENTRIES];
    __shared__ int bucket[TABLE_ENTRIES];
    const int wide = (x.num_buckets + TABLE_BUCKETS - 1) / TABLE_BUCKETS;
    const int h = blockIdx.x / wide, b0 = blockIdx.x % wide * TABLE_BUCKETS + 4 * (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int entries = RowSums::entries(x.reach, l.L_q, l.L_k);
    const size_t stride = (size_t)(entries + mod::FAR), head = stride * l.H;
    float total[4] = {0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < groups; g = l.start ? g + 1 : groups) {
        const int start = start_of(l, g), count = l.start ? 1 : groups;        // without starts all sequences have the same distances
        const RowSums r(x.reach, start, (l.L_q + 31) / 32);
        const float *const from = x.by_distance + g * head + h * stride;
        for (int e0 = 0; e0 < entries + 2; e0 += TABLE_ENTRIES) {
            __syncthreads();
            const int most = entries + 2 - e0 < TABLE_ENTRIES ? entries + 2 - e0 : TABLE_ENTRIES;
            for (int i = threadIdx.x; i < most; i += 256) {
                const int e = e0 + i, t = e < entries ? 32 * r.first - start - 31 + e : (e == entries ? -x.reach : x.reach);
                bucket[i] = clamped(x.buckets[clamped(t, -x.reach, x.reach) + x.reach], 0, x.num_buckets - 1);
                float v = 0.f;
                int c = 0;
                if (DIRECT) {
                    for (; c < count; ++c) v += sum_rows(l, x, g + c, h, e / 32, e % 32, e >= entries, 0, 1, entries);
                } else {
                    for (; c + 4 <= count; c += 4) v += (from[c * head + e] + from[(c + 1) * head + e]) + (from[(c + 2) * head + e] + from[(c + 3) * head + e]);
                    for (; c < count; ++c) v += from[c * head + e];
                }
                value[i] = v;
            }
            __syncthreads();
            for (int i = lane; i < most; i += 64) {
                const int b = bucket[i];
                const float v = value[i];
#pragma unroll
                for (int w = 0; w < 4; ++w) total[w] += b == b0 + w ? v : 0.f;
            }
        }
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) total[w] += __shfl_xor(total[w], off, 64);
        if (lane == 0 && b0 + w < x.num_buckets) dtable[(size_t)(b0 + w) * l.H + h] = (bf16_t)total[w];
    }
}

bool aligned(const void *p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

struct Bias {
    const void *table;
    const int32_t *buckets;
    int num_buckets, reach;
    const int32_t *q_start;
};
struct Drop {
    float p;
    const uint64_t *rng;
};

int check(const void *q, const void *k, const void *v, const int32_t *seqlens_q, const int32_t *seqlens_k, const float *bias, float scale,
          const Bias *rel, const Drop *drop, int B, int L_q, int L_k, int H, int d) {
    if (!q || !k || !v || !seqlens_q || !seqlens_k || !bias || !std::isfinite(scale)) return SIGATTN_ERR_INVALID_ARG;
    if (rel && (!rel->table || !rel->buckets || rel->num_buckets <= 0 || rel->reach < 0)) return SIGATTN_ERR_INVALID_ARG;
    if (drop && (!drop->rng || !(drop->p >= 0.0f && drop->p < 1.0f))) return SIGATTN_ERR_INVALID_ARG;
    if (int e = check_shape(B, L_q, H, d)) return e;
    if (int e = check_shape(B, L_k, H, d)) return e;
    if (L_q > MOST_ROWS || L_k > MOST_ROWS) return SIGATTN_ERR_TOO_LARGE;
    if (rel && (rel->reach > MOST_REACH || rel->num_buckets > MOST_BUCKETS)) return SIGATTN_ERR_TOO_LARGE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned(seqlens_q, 4) || !aligned(seqlens_k, 4) || !aligned(bias, 4)) return SIGATTN_ERR_MISALIGNED;
    if (rel && (!aligned(rel->table, 2) || !aligned(rel->buckets, 4) || !aligned(rel->q_start, 4))) return SIGATTN_ERR_MISALIGNED;
    if (drop && !aligned(drop->rng, 8)) return SIGATTN_ERR_MISALIGNED;
    return SIGATTN_OK;
}

// Of 65536 weights, those that stay: at least one; 65536 of them is no dropout.
unsigned kept(float p) {
    const unsigned k = (unsigned)std::floor((1.0 - (double)p) * 65536.0 + 0.5);
    return k < 1 ? 1 : k;
}

Extra extra(const Bias *rel, const Drop *drop) {
    Extra x{};
    x.inv_keep = 1.0f;
    if (rel) {
        x.table = static_cast<const bf16_t *>(rel->table);
        x.buckets = rel->buckets;
        x.q_start = rel->q_start;
        x.num_buckets = rel->num_buckets;
        x.reach = rel->reach;
    }
    if (drop) {
        x.rng = reinterpret_cast<const mod::u64 *>(drop->rng);
        x.keep = kept(drop->p);
        x.inv_keep = (float)(65536.0 / x.keep);
    }
    return x;
}

// Which calls with a bias and no dropout take the kernel for few queries (sigattn_rel_few.hpp).  It reads the keys once for every
// eight queries and grows with their number, but can split a head's keys; the tiled kernel takes as long for one query as for 128 and has
// a workgroup a head.  us, d = 64 (d = 128), H = 12, whole context valid, few / tiled:
//    1 query,   B = 32, 4096 keys   52 / 97              4 queries, B = 32, 4096 keys   89 / 97  (158 / 237)
//   16 queries, B = 1, 8192 keys    22 / 120 (37 / 177)  8 queries, B = 8, 8192 keys    57 / 121 (108 / 181)
//   64 queries, B = 1, 8192 keys    54 / 120 (94 / 177)  64 queries, B = 1, 2048 keys   21 / 33  (36 / 48)
//   48 queries, B = 2, 2048 keys    39 / 33  (65 / 49)   16 queries, B = 8, 8192 keys  105 / 121 (200 / 181)
//   16 queries, B = 1, 1000 keys    18 / 19  (29 / 27)   16 queries, B = 1, 64 keys    6.4 / 5.1 (6.4 / 6.4)
// So it takes five queries and more only where there are keys to split and, without that, less than half of the CUs had work.
int few_groups(int L_q) { return (L_q + 7) / 8; }
bool few_queries(int B, int L_q, int L_k, int H) {
    return L_q <= 4 || (L_q <= few::MOST && L_k > 1024 && (long long)B * H * few_groups(L_q) <= 128);
}
// Parts of a (z, h)'s keys.  A part is at least 1024 keys long (its start, and the second launch, take as long as reading some hundreds), and
// one group of queries has no more than give every CU two workgroups; up to eight groups have as many each (64 queries of 12 heads against
// 100000 keys: 4032 workgroups).  us, d = 64, H = 12, whole / in parts: one query, B = 1, 2048 keys 8.5 / 8.1, 8192
// keys 33.2 / 9.3; B = 8, 8192 keys 39.8 / 34.7; 16 queries, B = 1, 8192 keys 112 / 22.
int few_splits(int B, int L_k, int H) {
    const long long room = 512 / ((long long)B * H), longest = ((long long)L_k + 1023) / 1024;
    const long long s = room < longest ? room : longest;
    return s < 1 ? 1 : (int)s;
}
int few_rows(int L_q) { return L_q == 1 ? 1 : L_q == 2 ? 2 : L_q <= 4 ? 4 : 8; }
size_t few_bytes(int B, int L_q, int L_k, int H, int d) {
    if (check_shape(B, L_q, H, d) != SIGATTN_OK || check_shape(B, L_k, H, d) != SIGATTN_OK || !few_queries(B, L_q, L_k, H)) return 0;
    const int s = few_splits(B, L_k, H);
    return s == 1 ? 0 : (size_t)s * B * H * few_groups(L_q) * few_rows(L_q) * d * sizeof(float);
}

int forward(const void *q, const void *k, const void *v, void *o, const int32_t *seqlens_q, const int32_t *seqlens_k, const float *bias, float scale,
            const Bias *rel, const Drop *drop, int B, int L_q, int L_k, int H, int d, void *workspace, size_t workspace_bytes, void *stream) {
    if (!o) return SIGATTN_ERR_INVALID_ARG;
    if (int e = check(q, k, v, seqlens_q, seqlens_k, bias, scale, rel, drop, B, L_q, L_k, H, d)) return e;
    if (!aligned16(o)) return SIGATTN_ERR_MISALIGNED;
    if (drop && kept(drop->p) == 65536) drop = nullptr;
    if (!rel && !drop) return sigmoid_attn_cross_fwd(q, k, v, o, seqlens_q, seqlens_k, bias, scale, B, L_q, L_k, H, d, stream);
    Params p{};
    p.q = static_cast<const bf16_t *>(q);
    p.k = static_cast<const bf16_t *>(k);
    p.v = static_cast<const bf16_t *>(v);
    p.out0 = static_cast<bf16_t *>(o);
    p.seqlens = seqlens_q; p.N = L_q;
    p.seqlens_str = seqlens_k; p.N_str = L_k;
    p.bias = bias; p.scale = scale; p.B = B; p.H = H;
    const Extra x = extra(rel, drop);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (rel && !drop && few_queries(B, L_q, L_k, H)) {
        const size_t need = few_bytes(B, L_q, L_k, H, d);
        const bool parts = need > 0 && workspace && workspace_bytes >= need && aligned16(workspace);
        return few::launch(few::Few{p, x, parts ? few_splits(B, L_k, H) : 1, few_groups(L_q), static_cast<float *>(workspace)}, d, s);
    }
    if (d == 64) return rel && drop ? mod::fwd_rel_dropout_64(p, x, s) : rel ? mod::fwd_rel_64(p, x, s) : mod::fwd_dropout_64(p, x, s);
    return rel && drop ? mod::fwd_rel_dropout_128(p, x, s) : rel ? mod::fwd_rel_128(p, x, s) : mod::fwd_dropout_128(p, x, s);
}

// The workspace of a backward call with a bias table: a row of sums for every 32 queries, and their sums by group.
size_t row_floats(int B, int L_q, int L_k, int H, int reach) {
    return (size_t)B * H * (((size_t)L_q + 31) / 32) * (RowSums::entries(reach, L_q, L_k) + mod::FAR);
}
size_t group_floats(int B, int L_q, int L_k, int H, int reach) { return (size_t)B * H * (RowSums::entries(reach, L_q, L_k) + mod::FAR); }

size_t rel_bytes(int B, int L_q, int L_k, int H, int d, int reach) {
    if (check_shape(B, L_q, H, d) != SIGATTN_OK || check_shape(B, L_k, H, d) != SIGATTN_OK) return 0;
    if (L_q > MOST_ROWS || L_k > MOST_ROWS || reach < 0 || reach > MOST_REACH) return 0;
    return (row_floats(B, L_q, L_k, H, reach) + group_floats(B, L_q, L_k, H, reach)) * sizeof(float);
}

int backward(const void *q, const void *k, const void *v, const void *d_o, void *dq, void *dk, void *dv, void *dtable,
             const int32_t *seqlens_q, const int32_t *seqlens_k, const float *bias, float scale, const Bias *rel, const Drop *drop,
             int B, int L_q, int L_k, int H, int d, void *workspace, size_t workspace_bytes, void *stream) {
    if (!d_o || !dq || !dk || !dv || (rel && !dtable)) return SIGATTN_ERR_INVALID_ARG;
    if (int e = check(q, k, v, seqlens_q, seqlens_k, bias, scale, rel, drop, B, L_q, L_k, H, d)) return e;
    if (!aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) || !aligned(dtable, 2)) return SIGATTN_ERR_MISALIGNED;
    if (rel && (!workspace || workspace_bytes < rel_bytes(B, L_q, L_k, H, d, rel->reach))) return SIGATTN_ERR_WORKSPACE;
    if (rel && !aligned16(workspace)) return SIGATTN_ERR_MISALIGNED;
    if (drop && kept(drop->p) == 65536) drop = nullptr;
    if (!rel && !drop) return sigmoid_attn_cross_bwd(q, k, v, d_o, dq, dk, dv, seqlens_q, seqlens_k, bias, scale, B, L_q, L_k, H, d, stream);
    Params p{};
    p.q = static_cast<const bf16_t *>(q);
    p.k = static_cast<const bf16_t *>(k);
    p.v = static_cast<const bf16_t *>(v);
    p.d_o = static_cast<const bf16_t *>(d_o);
    p.bias = bias; p.scale = scale; p.B = B; p.H = H;
    Params pk = p, pq = p;
    pk.seqlens = seqlens_k; pk.N = L_k;
    pk.seqlens_str = seqlens_q; pk.N_str = L_q;
    pk.out0 = static_cast<bf16_t *>(dk);
    pk.out1 = static_cast<bf16_t *>(dv);
    pq.seqlens = seqlens_q; pq.N = L_q;
    pq.seqlens_str = seqlens_k; pq.N_str = L_k;
    pq.out0 = static_cast<bf16_t *>(dq);
    Extra x = extra(rel, drop);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!rel) return d == 64 ? mod::bwd_dropout_64(pk, pq, x, s) : mod::bwd_dropout_128(pk, pq, x, s);

    // Groups of sequences (sigattn_rel_rows): B = 256, H = 12, N = 512 backward 622 us with 16, 632 with 4, 634 with 64.
    const int entries = RowSums::entries(rel->reach, L_q, L_k), groups = rel->q_start || B < 16 ? B : 16;
    const long long row_wgs = (long long)groups * H * (entries / 32 + 1), table_wgs = (long long)H * ((rel->num_buckets + TABLE_BUCKETS - 1) / TABLE_BUCKETS);
    int seqs = 1;
    while (seqs < 8 && seqs * 2LL * groups <= B) seqs *= 2;
    if (row_wgs > 2147483647LL || table_wgs > 2147483647LL) return SIGATTN_ERR_TOO_LARGE;
    x.part = static_cast<float *>(workspace);
    x.by_distance = x.part + row_floats(B, L_q, L_k, H, rel->reach);
    const int e64 = d != 64 ? 0 : drop ? mod::bwd_rel_dropout_64(pk, pq, x, s) : mod::bwd_rel_64(pk, pq, x, s);
    const int e128 = d == 64 ? 0 : drop ? mod::bwd_rel_dropout_128(pk, pq, x, s) : mod::bwd_rel_128(pk, pq, x, s);
    if (e64 || e128) return e64 ? e64 : e128;
    const Lengths l{seqlens_q, seqlens_k, rel->q_start, bias, L_q, L_k, H, B};
    if ((long long)B * ((L_q + 31) / 32) <= DIRECT_ROWS) return enqueue(sigattn_rel_table<true>, table_wgs, 256, 0, s, l, x, B, static_cast<bf16_t *>(dtable));
    if (int e = enqueue(sigattn_rel_rows, row_wgs, 256, 0, s, l, x, groups, seqs)) return e;
    return enqueue(sigattn_rel_table<false>, table_wgs, 256, 0, s, l, x, groups, static_cast<bf16_t *>(dtable));
}

}  // namespace

extern "C" {

int sigmoid_attn_rel_buckets(int32_t *buckets, int num_buckets, int reach) {
    if (!buckets || num_buckets <= 0 || reach < 0) return SIGATTN_ERR_INVALID_ARG;
    if (num_buckets > MOST_BUCKETS || reach > MOST_REACH) return SIGATTN_ERR_TOO_LARGE;
    const int half = num_buckets / 2 > 1 ? num_buckets / 2 : 1, exact = half / 2 > 1 ? half / 2 : 1;
    for (int t = -reach; t <= reach; ++t) {
        const int a = t < 0 ? -t : t;
        int b;
        if (num_buckets >= 2 * reach + 1) {
            b = t + reach;
        } else {
            b = a;
            if (a >= exact)
                b = exact + (int)(std::log((double)a / exact) / std::log((double)(reach > exact ? reach : exact + 1) / exact) * (half - exact));
            if (b > half - 1) b = half - 1;
            if (t > 0) b += half;
            if (b > num_buckets - 1) b = num_buckets - 1;
        }
        buckets[t + reach] = b;
    }
    return SIGATTN_OK;
}

size_t sigmoid_attn_rel_fwd_workspace_bytes(int B, int L_q, int L_k, int H, int d) { return few_bytes(B, L_q, L_k, H, d); }

int sigmoid_attn_rel_fwd(const void *q, const void *k, const void *v, void *o, const int32_t *seqlens_q, const int32_t *seqlens_k,
                         const float *bias, float scale, const void *table, const int32_t *buckets, int num_buckets, int reach,
                         const int32_t *q_start, int B, int L_q, int L_k, int H, int d, void *workspace, size_t workspace_bytes, void *stream) {
    const Bias rel{table, buckets, num_buckets, reach, q_start};
    return forward(q, k, v, o, seqlens_q, seqlens_k, bias, scale, &rel, nullptr, B, L_q, L_k, H, d, workspace, workspace_bytes, stream);
}

int sigmoid_attn_dropout_fwd(const void *q, const void *k, const void *v, void *o, const int32_t *seqlens_q, const int32_t *seqlens_k,
                             const float *bias, float scale, float p, const uint64_t *rng, int B, int L_q, int L_k, int H, int d, void *stream) {
    const Drop drop{p, rng};
    return forward(q, k, v, o, seqlens_q, seqlens_k, bias, scale, nullptr, &drop, B, L_q, L_k, H, d, nullptr, 0, stream);
}

int sigmoid_attn_rel_dropout_fwd(const void *q, const void *k, const void *v, void *o, const int32_t *seqlens_q, const int32_t *seqlens_k,
                                 const float *bias, float scale, const void *table, const int32_t *buckets, int num_buckets, int reach,
                                 const int32_t *q_start, float p, const uint64_t *rng, int B, int L_q, int L_k, int H, int d, void *stream) {
    const Bias rel{table, buckets, num_buckets, reach, q_start};
    const Drop drop{p, rng};
    return forward(q, k, v, o, seqlens_q, seqlens_k, bias, scale, &rel, &drop, B, L_q, L_k, H, d, nullptr, 0, stream);
}

size_t sigmoid_attn_rel_bwd_workspace_bytes(int B, int L_q, int L_k, int H, int d, int reach) { return rel_bytes(B, L_q, L_k, H, d, reach); }

int sigmoid_attn_rel_bwd(const void *q, const void *k, const void *v, const void *d_o, void *dq, void *dk, void *dv, void *dtable,
                         const int32_t *seqlens_q, const int32_t *seqlens_k, const float *bias, float scale, const void *table,
                         const int32_t *buckets, int num_buckets, int reach, const int32_t *q_start, int B, int L_q, int L_k, int H, int d,
                         void *workspace, size_t workspace_bytes, void *stream) {
    const Bias rel{table, buckets, num_buckets, reach, q_start};
    return backward(q, k, v, d_o, dq, dk, dv, dtable, seqlens_q, seqlens_k, bias, scale, &rel, nullptr, B, L_q, L_k, H, d, workspace, workspace_bytes, stream);
}

int sigmoid_attn_dropout_bwd(const void *q, const void *k, const void *v, const void *d_o, void *dq, void *dk, void *dv,
                             const int32_t *seqlens_q, const int32_t *seqlens_k, const float *bias, float scale, float p, const uint64_t *rng,
                             int B, int L_q, int L_k, int H, int d, void *stream) {
    const Drop drop{p, rng};
    return backward(q, k, v, d_o, dq, dk, dv, nullptr, seqlens_q, seqlens_k, bias, scale, nullptr, &drop, B, L_q, L_k, H, d, nullptr, 0, stream);
}

int sigmoid_attn_rel_dropout_bwd(const void *q, const void *k, const void *v, const void *d_o, void *dq, void *dk, void *dv, void *dtable,
                                 const int32_t *seqlens_q, const int32_t *seqlens_k, const float *bias, float scale, const void *table,
                                 const int32_t *buckets, int num_buckets, int reach, const int32_t *q_start, float p, const uint64_t *rng,
                                 int B, int L_q, int L_k, int H, int d, void *workspace, size_t workspace_bytes, void *stream) {
    const Bias rel{table, buckets, num_buckets, reach, q_start};
    const Drop drop{p, rng};
    return backward(q, k, v, d_o, dq, dk, dv, dtable, seqlens_q, seqlens_k, bias, scale, &rel, &drop, B, L_q, L_k, H, d, workspace, workspace_bytes, stream);
}

}  // extern "C"
