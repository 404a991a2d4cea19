// Attention whose scores carry a learned relative position bias and whose weights go through dropout, on the kernels of
// sigattn_kernels.hpp:
//
//   x_ij  = scale <q_i, k_j> + bias[z] + table[b_ij][h],   b_ij = buckets[clamp(j - i - q_start[z], -reach, reach) + reach]
//   O_i   = sum_j m_ij P_ij v_j / keep,                    P = sigma(x),  m_ij in {0, 1} with share `keep` of ones
//   dS_ij = P_ij (1 - P_ij) m_ij dP_ij / keep,             dV_j = sum_i m_ij P_ij dO_i / keep
//   dtable[b][h] = sum over z, i, j with b_ij = b of dS_ij
//
// The bias depends on j - i alone.  Streamed rows pass an owner row in order, so the values that the score tiles of an owner
// tile start from (the accumulators of the score contraction: no vector instruction adds them) are a window of one vector
// over the distances, which moves on by 64 entries a tile.  It lives in a ring in LDS; a tile's new entries are looked up
// (bucket, then table) some tiles ahead of each other and stored with the tile.  Any reach costs the same here; the sums of dS by distance take longer,
// and memory, with more of the distances within it (RowSums).  (A forward pass that started
// the tiles beyond +-reach, which have one bias, from zeros and took the bias as a factor of the sequence's gained 4 % where nearly all tiles
// are such, lost 2 % where none are and 11 % in the smallest calls, and had two loops.)
#pragma once
#include "sigattn_kernels.hpp"

namespace sigattn {
namespace mod {

typedef unsigned long long u64;

// The far sums of a sequence of many blocks, and everything else about dS, are of dS / c (c = 2^(-bias log2 e), as in run_pass) and without
// 1 / keep: the kernel that adds up the rows applies both.
struct Extra {                       // what the calls take besides Params
    const bf16_t *table;             // [num_buckets][H]
    const int32_t *buckets;          // [2 reach + 1]
    const int32_t *q_start;          // [B], or null for zeros: position of query row 0 among the keys
    int num_buckets, reach;
    const u64 *rng;                  // {seed, offset}
    unsigned keep;                   // of 65536 weights, those that stay
    float inv_keep;                  // 65536 / keep
    float *part;                     // sums of dS by distance, see RowSums below
    float *by_distance;
};

// ---- sums of dS by distance
//
// For 32 queries [32 ob, 32 ob + 32) and 32 keys [32 b, 32 b + 32) the distances j - i - q_start are 32 (b - ob) - q_start + [-31, 31].
// Blocks wholly at or beyond +-reach belong to one bucket each and are summed as they are; of the others ("near") every
// distance is summed on its own.  For each ob a row of partial sums: entry 32 (k - first) + c, k = b - ob, is that of distance
// 32 k - q_start - 31 + c; behind the entries of all near blocks and one more the sums of the two far sides.
struct RowSums {
    int first, last;                 // near block diagonals k of a sequence: [first, last]
    __host__ __device__ static int down(int a) { return a >> 5; }                                  // a / 32, rounded down
    __device__ __forceinline__ RowSums(int reach, int start, int row_blocks) {
        first = down(start - reach - 31) + 1;                  // smallest k with 32 k - start + 31 > -reach
        last = -down(-(start + reach + 31)) - 1;               // largest k with 32 k - start - 31 < reach
        const int low = 1 - row_blocks;                        // no smaller k exists
        first = first < low ? low : first;
    }
    // entries of a row (a multiple of 32), for any q_start: all of them for every 32 queries, so the rows of a call whose reach is of the order of its
    // length grow with the square of that (us of the backward pass and MB, B = 4, H = 12, N = 8192, all valid: reach 256 3417, 33; 1024 3645,
    // 109; 8192 4290, 812)
    __host__ __device__ static int entries(int reach, int L_q, int L_k) {
        const int near = (2 * reach + 62) / 32 + 2, all = (L_q + 31) / 32 + 2 * ((L_k + 63) / 64);
        return 32 * ((near < all ? near : all) + 1);
    }
};
constexpr int FAR = 32;              // floats behind the entries of a row: [0] the far side below, [1] the one above

// What one pass adds to a kernel.  BIASED: the position bias; SIFTED: dropout; SUMMED: sums of dS by distance (DQ).  Not SCALED: scores are
// contracted from the queries and keys as they are and multiplied by scale log2 e in fp32, one instruction more for each.  The
// results are 2.4e-3 (2-norm) from 64 bits, the rounding of P (dS) and of the result itself, and not 2.9e-3; forward and backward
// pass of B = 8, H = 12, N = 2048 with dropout take 2 % longer each, of B = 4, H = 12, N = 8192 with a bias 5 % and 3 %.
//
// us, forward + backward, beside the plain calls' two-pass kernels (the same lengths): d = 64, B = 8, H = 12, N = 2048, bias 136 + 457
// (every distance near: 136 + 545), dropout 159 + 490, plain 112 to 128 + 376 to 385; d = 128, B = 8, H = 16, N = 2048, bias 293 + 1101, both 336 +
// 1309, plain 251 + 973.  What bounds them with dropout is the issue of vector instructions, 17.7 for each matrix instruction of the d = 64 forward pass
// and 15.8 of the backward for the plain kernels' 7.4 and 8.2: their port is busy 82 and 87 % of the time (plain 69 and 75 %).  With a bias no unit is busy
// most of the time (vector issue 64 to 67 %, matrix units 35 to 40 %, LDS 35 to 47 %, waves waiting to issue 30 to 34 %).  The clock is 1.9 to 2.1 GHz
// where the plain kernels' is 1.7 to 1.9: the power limit, which holds those, holds these less.
template <int MODE, int QB, int NW, bool BIAS, bool DROP, bool SUM>
struct Mods {
    static constexpr bool BIASED = BIAS, SIFTED = DROP, SUMMED = SUM, SCALED = false;
    static constexpr int BM = 32 * QB * NW, THREADS = 64 * NW;
    static constexpr int RING = 512, MIRROR = 32;              // floats; what is read past the end is kept there again
    static_assert(BM + 160 <= RING, "live entries: an owner tile, the tile in hand and two more");
    static_assert(!SUM || (MODE == DQ && QB == 1), "sums ride on the dQ pass");

    const Params &p;
    const Extra &x;
    float *const ring;                                         // LDS [RING + MIRROR]
    int h, n, ns, m0, start_pos;
    int wave, lane;

    // bias
    unsigned at;                                               // byte in the ring of this lane's first entry, owner block 0
    float unit;                                                // of the ring's values: they are added to scores before c1 = -scale log2 e
    int chunk;                                                 // the 64 entries that are stored next: those of tile `chunk`
    int bucket;
    unsigned short looked_up;
    // dropout
    unsigned keep, key0, key1, c3, c2, row, group;             // row, group: counter words of owner block 0, this block
    unsigned ph[DROP ? QB : 1][4], stays[DROP ? QB : 1];

    // sums
    float *out_row;
    int k, first, last, entries;
    bool active, open_window;
    f32x4 acc;                                                 // near: four distances a lane; far: every row holds 16 sums
    float below;

    __device__ __forceinline__ Mods(const Params &p_, const Extra &x_, float *ring_) : p(p_), x(x_), ring(ring_) {}

    // What scores are multiplied with.  The ring divides by it: scales below 2^-60 in size count as that, which no sum of a score and a
    // bias in fp32 can tell from what they are.
    __device__ __forceinline__ static float factor(const float c1) {
        return BIAS && __builtin_fabsf(c1) < 0x1p-60f ? __builtin_copysignf(0x1p-60f, c1) : c1;
    }

    // ---------------------------------------------------------------- bias
    // Distance (streamed - owner) `d` -> value; 0 for distances that no valid pair has, which padding alone reads.
    __device__ __forceinline__ int bucket_at(const int d) const {
        int t = MODE == DKDV ? -d - start_pos : d - start_pos;
        t = t < -x.reach ? -x.reach : (t > x.reach ? x.reach : t);
        return x.buckets[t + x.reach];
    }
    __device__ __forceinline__ unsigned short entry(const int b) const {
        const int c = b < 0 ? 0 : (b >= x.num_buckets ? x.num_buckets - 1 : b);
        return reinterpret_cast<const unsigned short *>(x.table)[(size_t)c * p.H + h];
    }
    __device__ __forceinline__ float value_of(const unsigned short entry, const int d) const {
        const float v = __builtin_bit_cast(float, (unsigned)entry << 16) * unit;
        return d > -n && d < ns ? v : 0.f;
    }

    __device__ __forceinline__ void open(const int z, const int h_, const int n_, const int ns_, const int m0_, const float c1) {
        h = h_; n = n_; ns = ns_; m0 = m0_;
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int c = lane & 31, g = lane >> 5;
        if constexpr (BIAS) {
            int s = x.q_start ? x.q_start[z] : 0;
            s = s < -(1 << 29) ? -(1 << 29) : (s > (1 << 29) ? (1 << 29) : s);
            start_pos = __builtin_amdgcn_readfirstlane(s);
            at = 4u * (unsigned)((BM - 32 * QB * wave - c + 4 * g) & (RING - 1));
            unit = -1.4426950408889634f / c1;
            chunk = 2;
            bucket = bucket_at(64 * own_chunk() - m0 + lane);
        }
        if constexpr (DROP) {
            keep = __builtin_amdgcn_readfirstlane(x.keep);
            const u64 seed = x.rng[0], offset = x.rng[1];
            key0 = __builtin_amdgcn_readfirstlane((unsigned)seed);
            key1 = __builtin_amdgcn_readfirstlane((unsigned)(seed >> 32));
            c3 = __builtin_amdgcn_readfirstlane((unsigned)offset);
            c2 = __builtin_amdgcn_readfirstlane((unsigned)z * (unsigned)p.H + (unsigned)h);
            if constexpr (MODE == DKDV) { row = c; group = 2 * (m0 / 32 + wave) + g; }
            else { row = m0 + 32 * QB * wave + c; group = g; }
        }
        if constexpr (SUM) {
            const int ob = m0 / 32 + wave, blocks = (p.N + 31) / 32;
            const RowSums r(x.reach, start_pos, blocks);
            first = r.first; last = r.last;
            entries = RowSums::entries(x.reach, p.N, p.N_str);
            k = -ob;                                           // diagonal of key block 0
            active = 32 * ob < n;
            open_window = false;
            out_row = x.part + (((size_t)z * p.H + h) * blocks + ob) * (size_t)(entries + FAR);
            acc = f32x4{0.f, 0.f, 0.f, 0.f};
            below = 0.f;
        }
    }
    // The waves take turns with the entries of a tile: this wave's first one.
    __device__ __forceinline__ int own_chunk() const { return 2 + ((wave - 2) & (NW - 1)); }
    // The entries of the first two tiles and of the owner tile in front of them.
    __device__ __forceinline__ void fill() {
        for (int e = threadIdx.x; e < BM + 128; e += THREADS) {
            const int d = e - BM - m0;
            const float v = value_of(entry(bucket_at(d)), d);
            ring[e] = v;
            if (e < MIRROR) ring[RING + e] = v;
        }
        looked_up = entry(bucket);
        bucket = bucket_at(64 * (own_chunk() + NW) - m0 + lane);
    }
    // With a tile's stores: its entries, if it is this wave's turn, and the look-ups for the next turns: the table's entry for the
    // next one, the bucket for the one behind it.  Nothing waits for them until then.  (With look-ups by all waves in
    // every tile, a tile of the forward pass had 30 of 254 vector instructions more.)
    __device__ __forceinline__ void store() {
        if ((chunk & (NW - 1)) == wave) {                      // uniform
            const int pos = (BM + 64 * chunk) & (RING - 1), d = 64 * chunk - m0 + lane;
            const float v = value_of(looked_up, d);
            ring[pos + lane] = v;
            if (pos == 0 && lane < MIRROR) ring[RING + lane] = v;
            looked_up = entry(bucket);
            bucket = bucket_at(d + 128 * NW);
        }
        ++chunk;
    }
    // What the score tile of owner block qb starts from, next streamed block.
    template <int qb>
    __device__ __forceinline__ void start(f32x16 &s) const {
        // the address as one register: the offsets of all reads then fit their instructions
        unsigned from = (unsigned)(uintptr_t)SIGATTN_LDS_PTR(float, ring) + ((at - 128u * qb) & (4 * RING - 1));
        asm("" : "+v"(from));
        const auto *const r = (const __attribute__((address_space(3))) float *)(uintptr_t)from;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = r[8 * (i / 4) + i % 4];
    }
    __device__ __forceinline__ void advance() { at = (at + 128u) & (4 * RING - 1); }

    // ---------------------------------------------------------------- dropout
    __device__ __forceinline__ float scale() const { return x.inv_keep; }

    // Functions of three words in one instruction each; the byte is the function's truth table.
    __device__ __forceinline__ static unsigned majority(unsigned a, unsigned b, unsigned c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0xE8); }
    __device__ __forceinline__ static unsigned xor3(unsigned a, unsigned b, unsigned c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
    __device__ __forceinline__ static unsigned choose(unsigned mask, unsigned a, unsigned b) { return __builtin_amdgcn_bitop3_b32(mask, a, b, 0xCA); }
    // All ones where bit `at` of v is set, else zero.
    __device__ __forceinline__ static unsigned smear(unsigned v, int at) { return (unsigned)__builtin_amdgcn_sbfe((int)v, at, 1); }

    // Part `item` of the generator of owner block qb: seven rounds of Philox4x32 (Salmon, Moraes, Dror, Shaw 2011), then the 16
    // decisions of a lane.  Decision t takes bits t and t + 8 of each of the four words as its byte; its 16-bit number u is that
    // byte and, below it and bit-reversed, the byte of decision t ^ 16.  It stays where u + keep carries out of 16 bits, and
    // the carries of all decisions run through the bits of `keep` at once, one majority a bit.
    template <int qb, int item>
    __device__ __forceinline__ void generate() {
        unsigned (&c)[4] = ph[qb];
        if constexpr (item == 0) {
            c[0] = row + (MODE == DKDV ? 0 : 32 * qb);
            c[1] = group + (MODE == DKDV ? 2 * qb : 0);
            c[2] = c2;
            c[3] = c3;
        }
        if constexpr (item < 7) {
            const u64 a = (u64)0xD2511F53u * c[0], b = (u64)0xCD9E8D57u * c[2];
            const unsigned k0 = key0 + item * 0x9E3779B9u, k1 = key1 + item * 0xBB67AE85u;
            const unsigned n0 = xor3((unsigned)(b >> 32), c[1], k0), n2 = xor3((unsigned)(a >> 32), c[3], k1);
            c[0] = n0; c[1] = (unsigned)b; c[2] = n2; c[3] = (unsigned)a;
        } else {
            unsigned m = 0;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                m = majority(c[(7 - s) / 2] >> (8 * ((7 - s) % 2)), m, smear(keep, s));
            }
            m = __builtin_amdgcn_alignbit(m, m, 16);
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                m = majority(c[s / 2] >> (8 * (s % 2)), m, smear(keep, 8 + s));
            }
            stays[qb] = MODE == DKDV ? turned(m) : m;
        }
    }
    // Bits w and 16 + w (w < 8) of lane (c, g) are the decisions of query c for keys 8 (w / 2) + 4 g + 2 (w % 2) + {0, 1}; with
    // keys and queries exchanged in the result.  The words of both halves of the wave are joined into rows of 32 bits, and
    // each of five steps exchanges one bit of the lane's number with the bit of the position that stands for the same bit of
    // the other tensor's row.
    // One such step: `other` is the word of the lane whose number differs in one bit (`upper` smeared: it is set in this one's),
    // STRIDE the bit of the position.  Both shifts of it side by side, then the lane's own part and the other's.
    template <int STRIDE>
    __device__ __forceinline__ static unsigned exchange(const unsigned own, const unsigned other, const unsigned upper) {
        constexpr unsigned LOW = STRIDE == 1 ? 0x55555555u : STRIDE == 2 ? 0x33333333u : STRIDE == 4 ? 0x0F0F0F0Fu : STRIDE == 8 ? 0x00FF00FFu : 0x0000FFFFu;
        const unsigned crossed = STRIDE == 16  ? __builtin_amdgcn_alignbit(other, other, 16)
                                 : STRIDE == 8 ? __builtin_amdgcn_perm(other, other, 0x02030001)
                                               : choose(LOW, other >> STRIDE, other << STRIDE);
        return choose(LOW ^ upper, own, crossed);
    }
    template <int CTRL>
    __device__ __forceinline__ static unsigned dpp(const unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
    __device__ __forceinline__ unsigned turned(unsigned m) const {
        const int g = lane >> 5;
        m = (m & 0x00FF00FFu) << (8 * g);
        const auto halves = __builtin_amdgcn_permlane32_swap(m, m, false, false);     // {lower half's words, upper half's} in every lane
        unsigned v = halves[0] | halves[1];
        v = exchange<16>(v, dpp<0xB1>(v), smear(lane, 0));                                   // quad_perm 1, 0, 3, 2
        v = exchange<1>(v, dpp<0x4E>(v), smear(lane, 1));                                    // quad_perm 2, 3, 0, 1
        v = exchange<8>(v, dpp<0x1B>(dpp<0x141>(v)), smear(lane, 2));                        // half mirror, then quad_perm 3, 2, 1, 0
        v = exchange<2>(v, dpp<0x128>(v), smear(lane, 3));                                   // rotation of a row of 16 by 8
        const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = exchange<4>(v, choose(smear(lane, 4), rows[0], rows[1]), smear(lane, 4));
        return v >> (8 * g);
    }

    // The share of slot K of SLOTS of a step.
    template <int K, int SLOTS>
    __device__ __forceinline__ void slot() {
        static_for<(K * 8 * QB) / SLOTS, ((K + 1) * 8 * QB) / SLOTS>([&](auto i_) {
            constexpr int i = decltype(i_)::value;
            generate<i / 8, i % 8>();
        });
    }
    template <int qb, bool WEIGHTS, bool DS>
    __device__ __forceinline__ void sift(u32x4 (&w)[2], u32x4 (&ds)[2]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const s16x2 both = __builtin_bit_cast(s16x2, stays[qb] << (15 - i));
            const unsigned keep = __builtin_bit_cast(unsigned, (s16x2)(both >> 15));
            if (WEIGHTS) w[i / 4][i % 4] &= keep;
            if (DS) ds[i / 4][i % 4] &= keep;
        }
    }
    __device__ __forceinline__ void next_block() {
        if (MODE == DKDV) row += 32;
        else group += 2;
    }

    // ---------------------------------------------------------------- sums of dS
    // A near block: the bf16 values that also feed dQ (two rows a register) go to LDS as 32 columns (queries) of 32 words, moved up
    // by a word every second column, so that what belongs to one distance lies in one line: word u of an odd column holds
    // distances 2 u and 2 u + 1 of the block's 63, of an even column 2 u + 1 and 2 u + 2; the rest of a column is zeros.  Columns c % 4 lie in four
    // pieces of scratch, and the 16 lanes that read one add up eight columns, four distances a lane.  The four groups of
    // lanes are joined when the 32 distances that no later block reaches go out; the others move down by as much.
    // Every sum has its order: no atomics.  What is summed is dS as the dQ contraction takes it, rounded to bf16; the sums are fp32.  Roundings of
    // either sign cancel as the terms do: dtable is 2.5e-3 to 3e-3 (2-norm) from 64 bits, as dQ is, of which its own rounding to bf16 is 1.7e-3; with
    // terms in fp32 twice the words would go through LDS, which already makes the near blocks 21 % dearer (not built).
    // (With ds_add_f32 into such a window a block took 16 of them, at about a lane a
    // clock: backward of B = 256, H = 12, N = 512 1657 us.)
    static constexpr int ROW_SHR_1 = 0x111, ROW_SHL_8 = 0x108;
    template <int CTRL>
    __device__ __forceinline__ static float moved(const float v) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
    }
    __device__ __forceinline__ static float join32(const float a, const float b) {     // lower half: a of both halves, upper: b
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
        return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    __device__ __forceinline__ static float join16(const float a, const float b) {     // the same for pairs of rows of 16
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
        return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    }
    __device__ __forceinline__ void flush() {
        const float out = join16(join32(acc[0], acc[2]), join32(acc[1], acc[3]));
        const int v = lane & 15;
        if (v < 8) out_row[32 * (k - first) + 4 * v + (lane >> 4)] = out;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = moved<ROW_SHL_8>(acc[i]);
    }
    __device__ __forceinline__ void sum_block(unsigned char *const put, const unsigned char *const get, const u32x4 (&ds)[2], const bool mine) {
        if (k >= first && k <= last) {                         // uniform
            if (!open_window) { below = acc[0]; acc = f32x4{0.f, 0.f, 0.f, 0.f}; open_window = true; }
            if (mine) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {                  // rows 8 q + 4 g + 0..3
                    unsigned *const w = reinterpret_cast<unsigned *>(put) + 4 * q;
                    w[0] = ds[q / 2][2 * (q % 2)];
                    w[1] = ds[q / 2][2 * (q % 2) + 1];
                }
            }
            asm volatile("" ::: "memory");
            float t[4] = {0.f, 0.f, 0.f, 0.f};
            // (1, 0) and (0, 1) in scalar registers: as inline constants their packed form would be the instruction's own affair
            unsigned lo = 0x00003F80u, hi = 0x3F800000u;
            asm("" : "+s"(lo), "+s"(hi));
            const bf16x2 one_lo = __builtin_bit_cast(bf16x2, lo), one_hi = __builtin_bit_cast(bf16x2, hi);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const u32x2 w = *reinterpret_cast<const u32x2 *>(get + 128 * j);
                const unsigned w0 = w[0], w1 = w[1];           // a bit cast of a vector's element itself reads element 0
                const bf16x2 a = __builtin_bit_cast(bf16x2, w0), b = __builtin_bit_cast(bf16x2, w1);
                t[0] = __builtin_amdgcn_fdot2_f32_bf16(a, one_lo, t[0], false);
                t[1] = __builtin_amdgcn_fdot2_f32_bf16(a, one_hi, t[1], false);
                t[2] = __builtin_amdgcn_fdot2_f32_bf16(b, one_lo, t[2], false);
                t[3] = __builtin_amdgcn_fdot2_f32_bf16(b, one_hi, t[3], false);
            }
            // 0 x Inf and 0 x NaN: a value that is not finite belongs to its own distance alone, not to the other of its word as well.
            if (__builtin_amdgcn_ballot_w64(__builtin_isunordered(t[0], t[1]) || __builtin_isunordered(t[2], t[3]))) {
#pragma unroll
                for (int i = 0; i < 4; ++i) t[i] = 0.f;
#pragma unroll 1
                for (int j = 0; j < 8; ++j) {
                    const u32x2 w = *reinterpret_cast<const u32x2 *>(get + 128 * j);
                    const unsigned w0 = w[0], w1 = w[1];
                    t[0] += __builtin_bit_cast(float, w0 << 16);
                    t[1] += __builtin_bit_cast(float, w0 & 0xFFFF0000u);
                    t[2] += __builtin_bit_cast(float, w1 << 16);
                    t[3] += __builtin_bit_cast(float, w1 & 0xFFFF0000u);
                }
            }
            asm volatile("" ::: "memory");
            const bool even = ((lane >> 4) & 1) == 0;          // lanes of even columns are a distance ahead
            const float t3 = moved<ROW_SHR_1>(t[3]);
            acc[0] += even ? t3 : t[0];
            acc[1] += even ? t[0] : t[1];
            acc[2] += even ? t[1] : t[2];
            acc[3] += even ? t[2] : t[3];
            flush();
        } else {
            if (k > last && open_window) { flush(); acc = f32x4{0.f, 0.f, 0.f, 0.f}; open_window = false; }
            bf16x8 ones;
#pragma unroll
            for (int i = 0; i < 8; ++i) ones[i] = (bf16_t)1.0f;
            u32x4 d0 = ds[0], d1 = ds[1];
            if (n - m0 - 32 * wave < 32) {                     // uniform
                const unsigned ok = mine ? ~0u : 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    d0[i] &= ok;
                    d1[i] &= ok;
                }
            }
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, d0), acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, d1), acc, 0, 0, 0);
        }
        ++k;
    }
    // A tile's two blocks.  Scratch of this wave: 1024 bytes each at a, a + a_step, b, b + b_step.
    __device__ __forceinline__ void sum(unsigned char *const a, const int a_step, unsigned char *const b, const int b_step, const u32x4 (&first_ds)[2],
                                        const u32x4 (&second_ds)[2]) {
        if (!active) return;                                   // uniform
        const int c = lane & 31, g = lane >> 5;
        asm volatile("" ::: "memory");
        if (k <= last && k + 1 >= first) {
            const u32x4 z4 = {0u, 0u, 0u, 0u};
            *reinterpret_cast<u32x4 *>(a + 16 * lane) = z4;
            *reinterpret_cast<u32x4 *>(a + a_step + 16 * lane) = z4;
            *reinterpret_cast<u32x4 *>(b + 16 * lane) = z4;
            *reinterpret_cast<u32x4 *>(b + b_step + 16 * lane) = z4;
        }
        asm volatile("" ::: "memory");
        auto piece = [&](const int i) { return (i & 2 ? b : a) + (i & 1 ? (i & 2 ? b_step : a_step) : 0); };
        unsigned char *const put = piece(c & 3) + (c >> 2) * 128 + 4 * (15 - (c >> 1)) + 8 * g;
        const unsigned char *const get = piece(lane >> 4) + 8 * (lane & 15);
        const bool mine = m0 + 32 * wave + c < n;              // rows behind the valid queries: a key of Inf would make them NaN
        sum_block(put, get, first_ds, mine);
        sum_block(put, get, second_ds, mine);
    }
    // Behind the last block: what is left in the window, and the far sums (row 0 of the accumulators, lanes 0 to 15).
    __device__ __forceinline__ void close() {
        if (!active) return;
        if (open_window) { flush(); acc = f32x4{0.f, 0.f, 0.f, 0.f}; }
        const bool all_below = k <= first;                     // not one block was near, or beyond
        float v = lane < 16 ? acc[0] : 0.f, u = lane < 16 ? below : 0.f;
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) {
            v += __shfl_xor(v, off, 64);
            u += __shfl_xor(u, off, 64);
        }
        if (lane == 0) {
            out_row[entries] = all_below ? v : u;
            out_row[entries + 1] = all_below ? 0.f : v;
        }
    }
};

}  // namespace mod
}  // namespace sigattn
