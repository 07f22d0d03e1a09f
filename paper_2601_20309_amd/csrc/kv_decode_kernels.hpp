// Device kernels of a decode step over the paged cache (gfx950, wave64): new
// tokens into their pages, attention of one new token per request, eviction of
// blocks by the weight attention gave them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace dkv {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w32x2 __attribute__((ext_vector_type(2)));
typedef w32x4 w32x4_by8 __attribute__((aligned(8)));  // where rows of 8-bit values begin on multiples of 8 bytes
// where rows of 4-bit values begin anywhere
typedef w32x4 w32x4_any __attribute__((aligned(1)));
typedef w32x2 w32x2_any __attribute__((aligned(1)));
typedef uint32_t w32_any __attribute__((aligned(1)));
typedef uint16_t w16_any __attribute__((aligned(1)));

// Bits of a number in the cache.  4 bits: a sign and 0, 0.5, 1, 1.5, 2, 3, 4 or 6, times 2^(byte - 127) of its 32 dimensions
// (byte 255: NaN).  A token has its heads' numbers first, the even dimension of two in a byte's low half, then its heads' bytes.
enum Kind { kBits16, kBits8, kBits4 };

// What of a weight of up to 2^-8 meets a bf16 value: a power of 2, and it again where two bf16 numbers have their exponents.  As many as
// there may be tokens, of the largest value each, add up to less than 2^128 (of up to 2^28 tokens: no less than 2^-20, which leaves a
// weight of 2^-90 of the largest a number); and no less than that takes, since products of small values are lost below 2^-149.
struct Share {
    float part;
    uint32_t exponents;
    static Share of(uint32_t max_tokens)
    {
        uint32_t bits = 0;
        while (bits < 20u && max_tokens >> 7 > 1u << bits) bits++;
        return Share{1.0f / (float)(1u << bits), bits << 7 | bits << 23};
    }
};

// The 16-bit types of q, k, v and the outputs.
struct Bf16 {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    // Weights are exp2(score - reference), the largest between 2^kBias and 2^(kBias + kSlack), so that the reference and
    // all sums change scale only when a score is kSlack above what was met before.  Between 2^-16 and 2^-8 here, and a Share of
    // that as they meet the values.
    static constexpr float kBias = -16.0f, kSlack = 8.0f;
    static __device__ __forceinline__ f32x4 mma(w32x4 a, w32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        const x2 v = {(__bf16)lo, (__bf16)hi};
        return __builtin_bit_cast(uint32_t, v);
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_fp8(uint32_t w)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    }
    // two 4-bit numbers of byte BYTE, times a power of 2 (its exponent alone is looked at; 255: NaN); no bits are lost
    template <int BYTE>
    static __device__ __forceinline__ uint32_t from_fp4(uint32_t w, float power)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, BYTE));
    }
    static constexpr int kLowPower = -126, kHighPower = 125;  // of 4-bit numbers: half of the one and 6 of the other are bf16 numbers
    // bits for either of two that is infinity or NaN: the carry out of an exponent of ones
    static __device__ __forceinline__ uint32_t odd(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
    static __device__ __forceinline__ bool nan(uint32_t w) { return (w & 0x7FFFu) > 0x7F80u; }  // the lower of two
    static constexpr float kMost = 0x1.FEp127f;
    // Each of two weights as the sum of two numbers of 8 digits, the upper cut off, the lower the nearest to what that leaves:
    // within 2^-15, times the share.  The lower one gets 2^-20 of the weight on top, and the least normal number if that is less, so
    // that it is never 0 beside one: 0 times a value of infinity is NaN.
    static __device__ __forceinline__ void split(float a, float b, const Share &share, uint32_t &upper, uint32_t &lower)
    {
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        constexpr u16x2 least = {0x80, 0x80};
        const float part = share.part * (1.0f + 0x1p-20f);
        const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
        // (exponents, down to 0; a weight of NaN becomes a number here, but their sum stays NaN)
        const u16x2 up = __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, __builtin_amdgcn_perm(y, x, 0x07060302u)), __builtin_bit_cast(u16x2, share.exponents));
        upper = __builtin_bit_cast(uint32_t, up);
        const u16x2 low = __builtin_bit_cast(u16x2, pack(__builtin_fmaf(a, part, -lo(upper)), __builtin_fmaf(b, part, -hi(upper))));
        lower = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(low, __builtin_elementwise_min(up, least)));
    }
};

struct Fp16 {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    // fp16 has numbers from 2^-24 to 2^15: the largest weights lie between 2^12 and 2^15, so that its
    // smallest number is 2^-36 of them and less.
    static constexpr float kBias = 12.0f, kSlack = 3.0f;
    static __device__ __forceinline__ f32x4 mma(w32x4 a, w32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi)
    {
        const x2 v = {(_Float16)lo, (_Float16)hi};
        return __builtin_bit_cast(uint32_t, v);
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(x2, w).x; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(x2, w).y; }
    template <bool HI>
    static __device__ __forceinline__ uint32_t from_fp8(uint32_t w)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
    }
    template <int BYTE>
    static __device__ __forceinline__ uint32_t from_fp4(uint32_t w, float power)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, power, BYTE));
    }
    static constexpr int kLowPower = -23, kHighPower = 13;
    static __device__ __forceinline__ uint32_t odd(uint32_t w) { return ((w & 0x7C007C00u) + 0x04000400u) & 0x80008000u; }
    static __device__ __forceinline__ bool nan(uint32_t w) { return (w & 0x7FFFu) > 0x7C00u; }
    static constexpr float kMost = 65504.0f;
    static constexpr uint32_t kOnes = 0x3C003C00u;
    // As above, of 11 digits each, within 2^-21; each at least the smallest number there is, 2^-24, if there is a weight (no
    // weight that is one is below 2^-126).
    static __device__ __forceinline__ void split(float a, float b, const Share &, uint32_t &upper, uint32_t &lower)
    {
        const float u = fminf(a * 0x1p102f, 0x1p-24f), v = fminf(b * 0x1p102f, 0x1p-24f);
        const auto cut = __builtin_amdgcn_cvt_pkrtz(fmaxf(a, u), fmaxf(b, v));
        upper = __builtin_bit_cast(uint32_t, cut);
        lower = pack(fmaxf(a - (float)cut[0], u), fmaxf(b - (float)cut[1], v));
    }
};

// Weights are exp2(score - reference), the largest between 2^bias and 2^(bias + slack).  Fp16 and Bf16 say what they are in
// kv_attend.  Beside 4 bits, and in kv_attend_rows, the products of as many as there may be tokens with bf16's largest value add up to less
// than 2^127: between 2^-16 and 2^-13 in a decoder of 4096 tokens, half of that in one of twice as many.
struct Weights {
    float bias, slack;
};
constexpr float kBf16Slack = 3.0f;
inline float bf16_bias(uint32_t max_tokens)
{
    int bits = 12;
    while (bits < 31 && 1u << bits < max_tokens) bits++;
    return -(float)(bits + 1) - kBf16Slack;
}

// bf16 beside 4 bits, where there is no infinity: weights meet the values as they are, and Weights says how large they get.
struct Bf16Of4 : Bf16 {
    static __device__ __forceinline__ void split(float a, float b, const Share &, uint32_t &upper, uint32_t &lower)
    {
        const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
        upper = __builtin_amdgcn_perm(y, x, 0x07060302u);
        lower = pack(a - hi(x), b - hi(y));
    }
};

// Quotients of whole numbers below 2^31 by a divisor that the host knows: with 2^(bits - 1) < divisor <= 2^bits and
// magic = ceil(2^(31 + bits) / divisor), x / divisor = x * magic >> (31 + bits).
struct Divide {
    uint32_t magic, shift;  // 0: the divisor is 1
    static Divide by(uint32_t divisor)
    {
        uint32_t bits = 0;
        while ((1ull << bits) < divisor) bits++;
        if (bits == 0) return Divide{0u, 0u};
        return Divide{(uint32_t)(((1ull << (31 + bits)) + divisor - 1) / divisor), bits - 1u};
    }
    __host__ __device__ __forceinline__ uint32_t quotient(uint32_t x) const
    {
        return magic ? (uint32_t)((uint64_t)x * magic >> 32) >> shift : x;
    }
};

// ---- attention of one new token --------------------------------------------------------------
//
// scores s_t = q.k_t, weights w_t = exp2(c s_t - m), out = sum w_t v_t / sum w_t with a running
// reference m.  Every key and value is read once, so HBM bounds it: a matrix instruction per
// 16 x 16 x 32 products does what the vector units could not beside the loads.
//
// Work is cut into tiles of 32 tokens of one request.  The tiles of all requests, one behind the other, are dealt
// to `groups` equal ranges, whatever the requests' lengths; a range belongs to one workgroup (or several that share
// the KV heads).  A wave has one KV head and up to 16 of its query heads (a unit); where there are fewer units than
// waves, several waves take turns at the tiles of a range and join in LDS.  A request that lies in one range is
// finished there; others leave sum, reference and unnormalised output per range, and kv_join_kernel joins them.
// Where no request can be longer than a few steps of a workgroup's waves, a range is a request (by_request), and
// the second launch, which would take longer than they do, is not made.
//
// No operand passes through LDS.  The products are taken transposed, tokens x heads and
// dimensions x heads, so that the weights come out where the second product wants
// them: lane (n, kq) = (lane % 16, lane / 16) holds of head n the tokens kq * 4 + r and
// 16 + kq * 4 + r (r < 4), which are the eight its operand takes if the values are
// brought in the same order (the order of a contraction is free).  For the values it loads
// 8 dimensions of each of those eight tokens, 16 lanes a row, whole rows of 256 bytes, and puts
// the pairs of tokens that a dimension's operand is made of together with byte permutes.
//
// Scores, references, weights and both sums are held in 32 bits.  The second product takes two operands of one type, and
// the values have 16 bits or fewer.  So a weight meets 16-bit (and 4-bit) values as the sum of two such numbers, in two products: the
// result is as far from 64 bits as its own rounding.  Beside outputs in bf16 8-bit values are taken as fp16, which holds them
// exactly, and one fp16 number is enough for a weight.  Root of the mean square of the relative error, 1e-4, a number
// of the output's type / so: bf16, 3 requests of 100 tokens 16.8 / 15.6, 32 around 1000 17.0 / 16.5; fp16 1.62 / 1.53; bf16 beside
// 8-bit values 16.8 / 16.5.  us: 5.6 / 5.7; 35.3 / 35.7; 4 requests of 32768 tokens 87.7 / 88.1; fp16, 37 to 1700 13.9 / 14.5, 119 to 1100
// and one head of 128 17.3 / 18.0; 8-bit, 128 around 600 38.1 / 38.4 (two numbers 39.0).
//
// Keys are read with plain loads (a row's 128-byte lines are met by several loads of a wave, which find them in the
// CU's cache), whole values past the caches: 16 lanes take a row at once.  us of this kernel as it is / with keys past the
// caches too / with values through them (weights of one number each): 32 requests around 1000 tokens, 32 query heads over 8 of 128, bf16 35.6 /
// 38.1 / 40.9; 4 of 32768 tokens, 64 over 8 of 128, 88.8 / 88.9 / 95.0; 4 of 32768, 8 heads of 96, 77.0 / 87.9 / 76.3;
// 8-bit, 128 around 600, 37.4 / 39.2 / 41.6.
//
// The 4 requests of 32768 tokens are 537 MB: 6.1 TB/s, of them some 5 us until all keys are under way and 6.4 TB/s from
// then on.  Counters: 4.199 million reads of 128 bytes, 537 MB: each byte of the cache once; no LDS bank conflicts.

struct AttendParams {
    const uint8_t *k, *v;      // the layer's planes
    const int32_t *table, *lens;
    const uint8_t *q;
    uint8_t *out;
    float *lse;                // nullptr: not wanted
    // What ranges leave of requests that go on in others, unnormalised and as it lies in a wave's registers:
    // [groups * 2][units][sum i][kq][part_rows], a vector of the dimensions i + (kq * 4 + r) * (8, or 4 up to 64 dimensions)
    f32x4 *part;
    f32x4 *part_ml;            // [groups * 2][n_heads]: reference, sum of weights as they met the values, as they were, its log2 + reference
    float *lse2;               // [n_seqs][n_heads], base 2; written where granules is
    float *granules;           // nullptr, or [n_seqs][max_granules][n_heads]: log2 of the weight of `granule` tokens
    const float *mass;
    float *mass_out;
    int64_t mass_stride;
    uint64_t q_row, q_head, out_row, out_head;  // bytes
    int64_t table_stride;
    uint32_t n_seqs, n_heads, max_blocks, max_tokens;
    uint32_t dim, token_bytes, head_bytes;
    uint32_t block_size, cells_per_block, n_blocks;  // a block begins cells_per_block rows of token_bytes behind the one before it
    Divide by_block;
    uint32_t groups, wgs_per_group, units, units_per_wg, subs, group_heads, head_tiles;
    uint32_t part_rows, part_vecs;  // heads of a unit, and vectors: sums * 4 * part_rows
    Divide by_items, by_rows, by_head_tiles;  // by part_vecs / 4, part_rows, head_tiles
    uint32_t granule, granule_bits, max_granules;
    uint32_t joins;            // workgroups that join, per request
    uint32_t mass_bits;        // log2 of the lanes that add up a block's weights
    uint32_t by_request;       // a range is a request: nothing to join
    float qk_scale;            // to base 2
    float v_scale;
    uint32_t exponents;        // 4 bits: from a token's first byte to its heads' bytes
    float bias;                // 4 bits beside bf16: of Weights
    Share share;               // 16 bits, bf16
};

constexpr uint32_t kTile = 32;
constexpr uint32_t kNoCell = ~0u;
constexpr float kLowest = -3.402823466e38f;  // a reference below every score, and finite: a score of -inf has weight 0 beside it

// The row of the cache, in rows of one token, that row `row` of page `page` is; kNoCell for an id that is no page.
__host__ __device__ __forceinline__ uint32_t cell_in(uint32_t page, uint32_t n_blocks, uint32_t cells_per_block, uint32_t row)
{
    return page < n_blocks ? page * cells_per_block + row : kNoCell;
}

__device__ __forceinline__ uint32_t seq_tokens(const int32_t *lens, uint32_t s, uint32_t most)
{
    return (uint32_t)min(max(lens[s], 0), (int32_t)most);
}

__device__ __forceinline__ uint32_t tiles_of(uint32_t tokens) { return (tokens + kTile - 1u) / kTile; }

// Inclusive sum over the wave's lanes, in steps of 1, 2, 4, 8 within rows of 16 lanes, then from row to row.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v)
{
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);
    return v;
}

// Where the tiles of all requests go.  Every wave finds out for itself.
struct Deal {
    uint32_t total, per;  // tiles, and tiles of a range
    // Of request (n_seqs - 1) / 64 * 64 + lane: its tokens, its tiles, and those of its 64 up to and with it.
    uint32_t tokens, mine, upto;
    uint32_t before;  // tiles of the requests before the one asked for
    __device__ __forceinline__ Deal(const AttendParams &p, uint32_t lane, uint32_t asked) : total(0), before(0)
    {
        if (p.by_request) return;
        for (uint32_t base = 0; base < p.n_seqs; base += 64) {
            tokens = base + lane < p.n_seqs ? seq_tokens(p.lens, base + lane, p.max_tokens) : 0u;
            mine = tiles_of(tokens);
            upto = wave_scan(mine);
            if (asked >= base && asked - base < 64u) before = total + (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), (int)(asked - base));
            total += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        // (As few as one: a range of a tile for each of its waves meets the ends of several short requests one after the
        // other.  50 requests around 75 tokens, one KV head, us: 22.9 with at least a tile a wave, 14.5 so.)
        per = max((total + p.groups - 1u) / p.groups, 1u);
    }
    __device__ __forceinline__ uint32_t tokens_of(uint32_t s) const { return (uint32_t)__builtin_amdgcn_readlane((int)tokens, (int)s); }
    // The request that tile `at` is one of, and which of its tiles.
    __device__ __forceinline__ void find(const AttendParams &p, uint32_t lane, uint32_t at, uint32_t &s, uint32_t &t) const
    {
        uint32_t m = mine, u = upto, before = 0;
        for (uint32_t base = 0; base < p.n_seqs; base += 64) {
            if (p.n_seqs > 64u) {
                m = base + lane < p.n_seqs ? tiles_of(seq_tokens(p.lens, base + lane, p.max_tokens)) : 0u;
                u = wave_scan(m);
            }
            const uint64_t beyond = __ballot(before + u > at);
            if (beyond) {
                const uint32_t first = (uint32_t)__builtin_ctzll(beyond);
                s = base + first;
                t = at - before - (uint32_t)__builtin_amdgcn_readlane((int)(u - m), (int)first);
                return;
            }
            before += (uint32_t)__builtin_amdgcn_readlane((int)u, 63);
        }
        s = t = 0;  // not reached: `at` is below total
    }
};

template <int DP>
struct Step {
    static constexpr int KJ = DP / 32;              // steps of 32 dimensions of q.k
    static constexpr int VW = DP == 64 ? 4 : 8;     // dimensions of a row that a lane loads at once,
    static constexpr int NV = DP == 64 ? 1 : DP / 128;  // and how often
    static constexpr int ACC = VW * NV;
    // Waves of a workgroup, one or two per SIMD: rows of 256 dimensions need more than half of its registers.  us with
    // four / eight: 4 requests of 32768 tokens, 4 heads of 256, 92 / 171.
    static constexpr uint32_t WAVES = DP == 256 ? 4 : 8;
};

template <int BYTES>
struct Raw;
template <>
struct Raw<16> { typedef w32x4 type; };
template <>
struct Raw<8> { typedef w32x2 type; };
template <>
struct Raw<4> { typedef uint32_t type; };

__device__ __forceinline__ void clear(w32x4 &v) { v = w32x4{0u, 0u, 0u, 0u}; }
__device__ __forceinline__ void clear(w32x2 &v) { v = w32x2{0u, 0u}; }
__device__ __forceinline__ void clear(uint32_t &v) { v = 0u; }

// WHOLE: heads have exactly DP dimensions.  Otherwise lanes whose dimensions are not there read the row's
// first ones, in vain.
template <typename X, int KIND, int DP, bool WHOLE>
__global__ __launch_bounds__(64 * Step<DP>::WAVES) void kv_attend_kernel(const AttendParams p)
{
    using T = Step<DP>;
    constexpr bool FP8 = KIND == kBits8, FP4 = KIND == kBits4;
    constexpr int KJ = T::KJ, VW = T::VW, NV = T::NV, ACC = T::ACC;
    constexpr uint32_t WAVES = T::WAVES;
    // Of a key a lane takes 16 bytes at once: in 16 bits the 8 dimensions of a step of 32, 32 j + 8 kq on; in 8 bits
    // 16 dimensions, 64 l + 16 kq on, of which 8 go into each of two steps (q is brought in the same order); in 4 bits
    // 32 dimensions, which share one power of 2, 8 of them in each of four steps (16 of a row of up to 64).
    constexpr int KL = FP4 ? (KJ + 3) / 4 : FP8 ? KJ / 2 : KJ;
    constexpr uint32_t K4 = DP == 64 ? 16u : 32u;  // 4 bits: dimensions of a key that a lane takes at once
    // In 8 bits there is room for two tiles of values: they are asked for a tile ahead, like the keys.  us without / with:
    // 128 requests around 600 tokens, 8 heads of 128, 39.4 / 37.4; 4 of 32768 tokens, 8 heads of 128 48.4 / 50.4, of 192
    // 102 / 85, 4 heads of 256 51.4 / 55.2; in 16 bits, 32 requests around 1000, 8 heads of 128, 35.6 / 39.7.
    // In 4 bits a step has so few bytes that all of the next one's are asked for before this one's products.  Half of what it takes
    // then are vector instructions, some 360 for 32 tokens of 128 dimensions, 64 of them conversions, 36 for pairs of tokens: they are
    // busy 53 % of a SIMD's cycles; and its two waves wait 43 % of theirs for memory, a step of little ahead, or for shuffles.  us, both
    // launches: 4 requests of 32768 tokens, 8 heads of 128 (143 MB) 53.3, with places multiplied before the shuffles 51 (2.8 TB/s), with all
    // pages in the caches 39; 128 around 600 (95 MB) 51.
    constexpr bool EARLY = FP4;
    constexpr bool AHEAD = FP4 || (FP8 && !(WHOLE && DP == 256));
    auto k_dim = [](int j, uint32_t kq) { return FP4 ? (uint32_t)(j / 4) * 128u + kq * K4 + (uint32_t)(j & 3) * 8u : FP8 ? (uint32_t)(j / 2) * 64u + kq * 16u + (uint32_t)(j & 1) * 8u : (uint32_t)j * 32u + kq * 8u; };
    typedef typename Raw<FP4 ? 4 : (FP8 ? 1 : 2) * VW>::type vraw;
    // Values go past the caches, except short rows that share 128-byte lines with other heads' all along.  us past /
    // through them: 4 requests of 32768 tokens, 8-bit, 8 heads of 40 30.8 / 26.2, of 80 46.7 / 45.0, of 64 28.9 / 32.2;
    // 16-bit, 4 heads of 192 78.3 / 83.0, 8 of 96 76.0 / 77.2.
    constexpr bool PAST = WHOLE || (!FP8 && DP > 64);
    // The type of the second product, and whether a weight is two numbers of it.
    using Y = std::conditional_t<FP8, Fp16, std::conditional_t<FP4 && std::is_same_v<X, Bf16>, Bf16Of4, X>>;
    constexpr bool SPLIT = !FP8 || std::is_same_v<X, Fp16>;
    const Weights largest = std::is_same_v<Y, Bf16Of4> ? Weights{p.bias, kBf16Slack} : Weights{Y::kBias, Y::kSlack};
    __shared__ f32x4 joined[WAVES][ACC][64];
    __shared__ f32x4 ml[WAVES][16];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n = lane & 15u, kq = lane >> 4;
    const uint32_t group = blockIdx.x / p.wgs_per_group;
    const uint32_t unit = (blockIdx.x - group * p.wgs_per_group) * p.units_per_wg + wave % p.units_per_wg;
    const uint32_t sub = wave / p.units_per_wg;
    const bool active = unit < p.units;
    const Deal deal(p, lane, 0u);
    uint32_t at = p.by_request ? 0u : group * deal.per;
    const uint32_t end = p.by_request ? tiles_of(seq_tokens(p.lens, group, p.max_tokens)) : min(at + deal.per, deal.total);
    if (at >= end && !p.by_request) return;
    uint32_t s = group, t = 0;
    if (!p.by_request) deal.find(p, lane, at, s, t);
    const uint32_t kv_head = active ? unit / p.head_tiles : 0u, ht = active ? unit - kv_head * p.head_tiles : 0u;
    const uint32_t rows = min(16u, p.group_heads - ht * 16u);      // query heads of this wave
    const uint32_t head = kv_head * p.group_heads + ht * 16u + n;  // this lane's
    const bool has_row = active && n < rows;
    // bytes of so many dimensions
    auto bytes = [](uint32_t dims) { return FP4 ? dims / 2u : FP8 ? dims : dims * 2u; };
    if (at >= end) {  // a request of its own range, without a token
        for (uint32_t d = kq * 4u; has_row && sub == 0u && d < p.dim; d += 16u)
            *reinterpret_cast<w32x2 *>(p.out + (uint64_t)s * p.out_row + (uint64_t)head * p.out_head + d * 2u) = w32x2{0u, 0u};
        if (p.lse && has_row && sub == 0u && kq == 0u) p.lse[(uint64_t)s * p.n_heads + head] = -__builtin_inff();
        return;
    }
    const uint8_t *const kb = p.k + (uint64_t)kv_head * p.head_bytes + (WHOLE ? bytes(k_dim(0, kq)) : 0u);
    const uint8_t *const vb = p.v + (uint64_t)kv_head * p.head_bytes + (WHOLE ? bytes(n * VW) : 0u);
    // (Where rows are not whole, found anew for every row: kept, they are what does not fit the registers.)
    auto k_off = [&](int l, uint32_t kq) {
        constexpr uint32_t step = FP4 ? 128u : FP8 ? 64u : 32u, each = FP4 ? K4 : FP8 ? 16u : 8u;
        return WHOLE ? bytes((uint32_t)l * step) : bytes(min((uint32_t)l * step + kq * each, p.dim - each));
    };
    auto v_off = [&](int c, uint32_t n) {
        const uint32_t d = (uint32_t)c * 128u + n * VW;
        return WHOLE ? bytes((uint32_t)c * 128u) : bytes(min(d, p.dim - VW));
    };
    // 4 bits: from a token's numbers of this head to the head's powers of 2
    const uint32_t powers = FP4 ? p.exponents + kv_head * (p.dim / 32u) - kv_head * p.head_bytes : 0u;
    const uint8_t *const v_row = p.v + (uint64_t)kv_head * p.head_bytes;
    auto power = [](uint32_t byte) { return __builtin_bit_cast(float, byte << 23); };

    // What a step needs is asked for a step (its pages two steps) ahead, across the ends of requests,
    // too: a range goes on in the next request with its first keys under way.
    struct Part {
        uint32_t s, first, here;  // request, its tiles in this range
        uint32_t tokens, upto;    // its tokens, and those that lie in its tiles up to here
    };
    auto tokens_of = [&](uint32_t i) { return p.n_seqs > 64u || p.by_request ? seq_tokens(p.lens, i, p.max_tokens) : deal.tokens_of(i); };
    // The part that begins with tile `flat` of all, in request `i` or the first one behind it that has tiles.
    auto part_at = [&](uint32_t i, uint32_t first, uint32_t flat) {
        Part part = {i, first, 0u, 0u, 0u};
        for (; flat < end && part.s < p.n_seqs; part.s++, part.first = 0u) {
            part.tokens = tokens_of(part.s);
            const uint32_t n_tiles = tiles_of(part.tokens);
            if (n_tiles > part.first) {
                part.here = min(n_tiles - part.first, end - flat);
                part.upto = min(part.tokens, (part.first + part.here) * kTile);
                break;
            }
        }
        return part;
    };
    // The page of this lane's token of half tile h from `tile` on, and the row of the cache that makes it.
    auto page_of = [&](const Part &part, uint32_t tile, int h) {
        const uint32_t token = tile * kTile + (uint32_t)h * 16u + n;
        return token < part.upto ? (uint32_t)p.table[(int64_t)part.s * p.table_stride + p.by_block.quotient(token)] : kNoCell;
    };
    auto cell_of = [&](uint32_t tile, int h, uint32_t page) {
        const uint32_t token = tile * kTile + (uint32_t)h * 16u + n;
        return cell_in(page, p.n_blocks, p.cells_per_block, token - p.by_block.quotient(token) * p.block_size);
    };
    Part now = {s, t, 0u, 0u, 0u}, next = part_at(s, t, at);
    w32x4 qf[KJ];
    w32x4 kr[2][KL];
    uint32_t kx[2][KL];  // 4 bits: the lane's powers of 2
    auto load_keys = [&](w32x4(&to)[KL], uint32_t (&x)[KL], uint32_t cell) {
        const uint64_t off = (uint64_t)(cell == kNoCell ? 0u : cell) * p.token_bytes;
        uint32_t k = kq;
        if constexpr (!WHOLE) asm volatile("" : "+v"(k));
        if constexpr (FP4) {
            const uint8_t *const row = p.k + (uint64_t)kv_head * p.head_bytes + off;
#pragma unroll
            for (int l = 0; l < KL; l++) {
                const uint32_t d = WHOLE ? k_dim(4 * l, k) : min(k_dim(4 * l, k), p.dim - K4);
                if constexpr (DP == 64) {
                    const w32x2 y = *reinterpret_cast<const w32x2_any *>(row + d / 2u);
                    to[l] = w32x4{y[0], y[1], 0u, 0u};
                } else {
                    to[l] = *reinterpret_cast<const w32x4_any *>(row + d / 2u);
                }
                x[l] = row[powers + d / 32u];
            }
            return;
        }
        if constexpr (FP8 && !WHOLE && DP == 64) {
            if (p.dim < 16u) {  // a row of 8 bytes, and nothing behind the last one
                const w32x2 x = *reinterpret_cast<const w32x2 *>(kb + off);
                to[0] = w32x4{0u, 0u, x[0], x[1]};
                return;
            }
        }
#pragma unroll
        for (int l = 0; l < KL; l++) {
            if constexpr (FP8 && !WHOLE) to[l] = *reinterpret_cast<const w32x4_by8 *>(kb + off + k_off(l, k));
            else to[l] = *reinterpret_cast<const w32x4 *>(kb + off + k_off(l, k));
        }
    };
    uint32_t cell[2], page[2];
    // The lane's 8 tokens of the step whose cells are `cell`, and their values.
    uint32_t vcell[8];
    uint64_t voff[8];  // 4 bits: their bytes
    auto find_values = [&](uint32_t &present) {
        if constexpr (FP4) {
            // (a lane has both halves' tokens n: two products here instead of eight behind the shuffles, and a bit for each token)
            uint32_t bits[2];
            uint64_t off[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                bits[h] = (uint32_t)__ballot(cell[h] != kNoCell) & 0xFFFFu;
                off[h] = (uint64_t)(cell[h] == kNoCell ? 0u : cell[h]) * p.token_bytes;
            }
            present = (bits[0] >> (kq * 4u) & 15u) | (bits[1] >> (kq * 4u) & 15u) << 4;
#pragma unroll
            for (int r = 0; r < 8; r++) {
                const int from = (int)((kq * 4u + (r & 3)) * 4u);
                const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(uint32_t)off[r / 4]), hi = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(off[r / 4] >> 32));
                voff[r] = (uint64_t)hi << 32 | lo;
            }
            return;
        }
        present = 0;
#pragma unroll
        for (int r = 0; r < 8; r++) {
            const uint32_t c = (uint32_t)__shfl((int)cell[r / 4], (int)(kq * 4u + (r & 3)), 64);
            present |= c == kNoCell ? 0u : 1u << r;
            vcell[r] = c == kNoCell ? 0u : c;
        }
    };
    auto load_values = [&](vraw(&to)[8][NV], uint32_t (&x)[8][NV], int c) {
        uint32_t v = n;
        if constexpr (!WHOLE) asm volatile("" : "+v"(v));
        if constexpr (FP4) {
            const uint32_t d = WHOLE ? (uint32_t)c * 128u + v * VW : min((uint32_t)c * 128u + v * VW, p.dim - VW);
#pragma unroll
            for (int r = 0; r < 8; r++) {
                const uint8_t *const row = v_row + d / 2u + voff[r];
                if constexpr (DP == 64) to[r][c] = *reinterpret_cast<const w16_any *>(row);
                else to[r][c] = *reinterpret_cast<const w32_any *>(row);
                x[r][c] = v_row[powers + d / 32u + voff[r]];
            }
            return;
        }
#pragma unroll
        for (int r = 0; r < 8; r++)
        {
            const vraw *const from = reinterpret_cast<const vraw *>(vb + (uint64_t)vcell[r] * p.token_bytes + v_off(c, v));
            if constexpr (PAST) to[r][c] = __builtin_nontemporal_load(from);
            else to[r][c] = *from;
        }
    };
    vraw next_vr[8][NV];
    uint32_t next_vx[8][NV];  // 4 bits: powers of 2
    w32x4 next_kr[2][KL];
    uint32_t next_kx[2][KL];
    uint32_t next_present = 0;
    for (;;) {
        uint32_t next_page[2];
        const uint32_t next_first = next.first + sub, next_stop = active ? next.first + next.here : 0u;
#pragma unroll
        for (int h = 0; h < 2; h++) next_page[h] = next_first < next_stop ? page_of(next, next_first, h) : kNoCell;
        f32x4 acc[ACC], sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ACC; i++) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        float ref = kLowest;
        float own = 0.f;     // this lane's part of the sum of weights as they are, before they are rounded
        const uint32_t stop = active ? now.first + now.here : 0u;
        // at least once: a wave without a tile here still asks for what comes next
        uint32_t tt = now.first + sub;
        do {
            const bool have = tt < stop, last = tt + p.subs >= stop;
            vraw vr[8][NV];
            uint32_t vx[8][NV];
            uint32_t present = 0;  // bit r: token r of the lane's 8 is there
            f32x4 sc[2];
            // scores: token x head
            auto take_scores = [&] {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    w32x4(&key)[KL] = kr[h];
                    if constexpr (!WHOLE) {
                        // dimensions that are not there meet zeros of q: they must not be NaN
#pragma unroll
                        for (int l = 0; l < KL; l++) {
                            const uint32_t d = k_dim(FP4 ? 4 * l : FP8 ? 2 * l : l, kq);
                            if (d >= p.dim) {
                                clear(key[l]);
                                if constexpr (FP4) kx[h][l] = 0u;
                            }
                            else if (FP8 && d + 16u > p.dim) key[l] = w32x4{key[l][2], key[l][3], 0u, 0u};  // 8 are there: the last 16 were read
                        }
                    }
                    sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < KJ; j++) {
                        w32x4 a;
                        if constexpr (FP4) {
                            const uint32_t y = key[j / 4][j & 3];
                            const float x = power(kx[h][j / 4]);
                            a = w32x4{X::template from_fp4<0>(y, x), X::template from_fp4<1>(y, x), X::template from_fp4<2>(y, x),
                                      X::template from_fp4<3>(y, x)};
                        } else if constexpr (FP8) {
                            const uint32_t lo = key[j / 2][2 * (j & 1)], hi = key[j / 2][2 * (j & 1) + 1];
                            a = w32x4{X::template from_fp8<false>(lo), X::template from_fp8<true>(lo), X::template from_fp8<false>(hi),
                                      X::template from_fp8<true>(hi)};
                        } else {
                            a = key[j];
                        }
                        sc[h] = X::mma(a, qf[j], sc[h]);
                    }
                }
            };
            if (have) {
                if constexpr (AHEAD) {
                    present = next_present;
#pragma unroll
                    for (int r = 0; r < 8; r++) {
#pragma unroll
                        for (int c = 0; c < NV; c++) {
                            vr[r][c] = next_vr[r][c];
                            if constexpr (FP4) vx[r][c] = next_vx[r][c];
                        }
                    }
                } else {
                    find_values(present);
#pragma unroll
                    for (int c = 0; c < NV; c++) load_values(vr, vx, c);
                }
                if constexpr (!EARLY) take_scores();
            }
            // the step after this one (`next`: the first of the next request)
            const uint32_t tile = last ? next_first : tt + p.subs;
            const bool more = tile < (last ? next_stop : stop);
            auto read_queries = [&](uint32_t request) {
#pragma unroll
                for (int j = 0; j < KJ; j++) {
                    const uint32_t d = k_dim(j, kq);
                    qf[j] = w32x4{0u, 0u, 0u, 0u};
                    if (has_row && (WHOLE || d < p.dim))
                        qf[j] = *reinterpret_cast<const w32x4 *>(p.q + (uint64_t)request * p.q_row + (uint64_t)head * p.q_head + d * 2u);
                }
            };
            if constexpr (EARLY) {
                if (more) {
                    Part part = now;
                    if (last) part = next;
#pragma unroll
                    for (int h = 0; h < 2; h++) cell[h] = cell_of(tile, h, last ? next_page[h] : page[h]);
#pragma unroll
                    for (int h = 0; h < 2; h++) load_keys(next_kr[h], next_kx[h], cell[h]);
                    find_values(next_present);
#pragma unroll
                    for (int c = 0; c < NV; c++) load_values(next_vr, next_vx, c);
#pragma unroll
                    for (int h = 0; h < 2; h++) page[h] = page_of(part, tile + p.subs, h);
                }
                if (have) take_scores();
            }
            // the next step's keys, while this one's values arrive
            if constexpr (EARLY) {
                if (more) {
                    if (last) read_queries(next.s);
#pragma unroll
                    for (int h = 0; h < 2; h++) {
#pragma unroll
                        for (int l = 0; l < KL; l++) {
                            kr[h][l] = next_kr[h][l];
                            kx[h][l] = next_kx[h][l];
                        }
                    }
                }
            } else if (more) {
                Part part = now;
                if (last) part = next;
#pragma unroll
                for (int h = 0; h < 2; h++) cell[h] = cell_of(tile, h, last ? next_page[h] : page[h]);
                if (last) read_queries(part.s);
#pragma unroll
                for (int h = 0; h < 2; h++) load_keys(kr[h], kx[h], cell[h]);
                if constexpr (AHEAD) {
                    find_values(next_present);
#pragma unroll
                    for (int c = 0; c < NV; c++) load_values(next_vr, next_vx, c);
                }
#pragma unroll
                for (int h = 0; h < 2; h++) page[h] = page_of(part, tile + p.subs, h);
            }
            if (!have) break;
            float w[8], top = -__builtin_inff();
#pragma unroll
            for (int r = 0; r < 8; r++) w[r] = sc[r / 4][r & 3] * p.qk_scale;
            const bool gaps = __any(present != 0xFFu);
            if (gaps) {
#pragma unroll
                for (int r = 0; r < 8; r++) w[r] = present >> r & 1u ? w[r] : -__builtin_inff();
            }
#pragma unroll
            for (int r = 0; r < 8; r++) top = fmaxf(top, w[r]);
            if (__any(top > ref + largest.bias + largest.slack)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float higher = fmaxf(ref, top - largest.bias), shrink = __builtin_amdgcn_exp2f(ref - higher);
                ref = higher;
#pragma unroll
                for (int i = 0; i < ACC; i++) acc[i] *= shrink;
                if constexpr (!SPLIT) sum *= shrink;
                own *= shrink;
            }
#pragma unroll
            for (int r = 0; r < 8; r++) {
                w[r] = __builtin_amdgcn_exp2f(w[r] - ref);
                own += w[r];
            }
            w32x4 pw, pl;  // of two numbers the lower one
#pragma unroll
            for (int r = 0; r < 4; r++) {
                uint32_t upper, lower = 0u;
                if constexpr (SPLIT) Y::split(w[2 * r], w[2 * r + 1], p.share, upper, lower);
                else upper = Y::pack(w[2 * r], w[2 * r + 1]);
                pw[r] = upper;
                pl[r] = lower;
            }
            // Weights of one number: out is divided by the sum of the rounded ones, which it is made of (rows of ones beside
            // the values); lse and the blocks' weights go by the sum of those that they were.
            if constexpr (!SPLIT) sum = Y::mma(w32x4{Y::kOnes, Y::kOnes, Y::kOnes, Y::kOnes}, pw, sum);
            auto add_values = [&](f32x4 &to, w32x4 values) {
                if constexpr (SPLIT) to = Y::mma(values, pl, to);
                to = Y::mma(values, pw, to);
            };
#pragma unroll
            for (int c = 0; c < NV; c++) {
                if (gaps) {  // a weight of 0 does not make up for NaN
#pragma unroll
                    for (int r = 0; r < 8; r++)
                        if (!(present >> r & 1u)) {
                            clear(vr[r][c]);
                            if constexpr (FP4) vx[r][c] = 0u;
                        }
                }
                // of token r: dimensions 2i and 2i + 1
                auto pair = [&](int r, int i) {
                    const vraw &v = vr[r][c];
                    if constexpr (FP4) {
                        const float x = power(vx[r][c]);
                        return i == 0   ? Y::template from_fp4<0>(v, x)
                               : i == 1 ? Y::template from_fp4<1>(v, x)
                               : i == 2 ? Y::template from_fp4<2>(v, x)
                                        : Y::template from_fp4<3>(v, x);
                    } else if constexpr (FP8 && VW == 8) return i & 1 ? Y::template from_fp8<true>(v[i / 2]) : Y::template from_fp8<false>(v[i / 2]);
                    else if constexpr (FP8) return i & 1 ? Y::template from_fp8<true>(v) : Y::template from_fp8<false>(v);
                    else return v[i];
                };
#pragma unroll
                for (int i = 0; i < VW / 2; i++) {
                    w32x4 even, odd;
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const uint32_t a = pair(2 * k, i), b = pair(2 * k + 1, i);
                        even[k] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                        odd[k] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                    }
                    add_values(acc[c * VW + 2 * i], even);
                    add_values(acc[c * VW + 2 * i + 1], odd);
                }
            }
            if (p.granules) {
                // weights of runs of `granule` tokens (1, 4, 8 or 16: it divides a block)
                float *const g = p.granules + (uint64_t)now.s * p.max_granules * p.n_heads;
                auto put = [&](uint32_t token, float weight) {
                    if (has_row && token < now.upto) g[(uint64_t)(token >> p.granule_bits) * p.n_heads + head] = ref + __builtin_amdgcn_logf(weight);
                };
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const uint32_t first = tt * kTile + (uint32_t)h * 16u + kq * 4u;
                    if (p.granule == 1u) {
#pragma unroll
                        for (uint32_t r = 0; r < 4; r++) put(first + r, w[4 * h + r]);
                    } else {
                        float y = (w[4 * h] + w[4 * h + 1]) + (w[4 * h + 2] + w[4 * h + 3]);
                        const float y8 = y + __shfl_xor(y, 16, 64), y16 = y8 + __shfl_xor(y8, 32, 64);
                        y = p.granule == 16u ? y16 : p.granule == 8u ? y8 : y;
                        if (((kq * 4u) & (p.granule - 1u)) == 0u) put(first, y);
                    }
                }
            }
            tt += p.subs;
        } while (tt < stop);
        if (now.here) {
            own += __shfl_xor(own, 16, 64);
            own += __shfl_xor(own, 32, 64);
            if constexpr (SPLIT) sum[0] = std::is_same_v<Y, Bf16> ? own * p.share.part : own;  // as they met the values
            const bool whole = now.here == tiles_of(now.tokens);
            const uint32_t slot = group * 2u + (now.first > 0u ? 0u : 1u);
            f32x4 *const part = p.part + ((uint64_t)slot * p.units + unit) * p.part_vecs;
            uint8_t *const out = p.out + (uint64_t)now.s * p.out_row;
            // Waves that took turns at the tiles leave what they have in LDS, and share the sums out among them.
            float scale[WAVES];  // of each one's: 2^(its reference - the largest)
            if (p.subs > 1u) {
                const uint32_t u = wave % p.units_per_wg;
                if (kq == 0u) ml[wave][n] = f32x4{ref, sum[0], own, 0.f};
#pragma unroll
                for (int i = 0; i < ACC; i++) joined[wave][i][lane] = acc[i];
                __syncthreads();
                f32x4 x[WAVES];
#pragma unroll
                for (uint32_t o = 0; o < WAVES; o++) {
                    x[o] = o < p.subs ? ml[o * p.units_per_wg + u][n] : f32x4{kLowest, 0.f, 0.f, 0.f};
                    ref = fmaxf(ref, x[o].x);
                }
                sum[0] = own = 0.f;
#pragma unroll
                for (uint32_t o = 0; o < WAVES; o++) {
                    scale[o] = __builtin_amdgcn_exp2f(x[o].x - ref);
                    sum[0] += x[o].y * scale[o];
                    own += x[o].z * scale[o];
                }
            }
            // (times v_scale afterwards: v_scale / total is too small a number sooner than the result)
            const float total = sum[0], inv = total == 0.f ? 0.f : 1.0f / total, v_scale = FP8 ? p.v_scale : 1.0f;
            if (has_row && sub == 0u && kq == 0u) {
                const float l2 = own == 0.f ? -__builtin_inff() : ref + __builtin_amdgcn_logf(own);
                if (!whole) p.part_ml[(uint64_t)slot * p.n_heads + head] = f32x4{ref, total, own, l2};
                if (whole && p.lse) p.lse[(uint64_t)now.s * p.n_heads + head] = l2 * 0.693147180559945309f;
                if (whole && p.granules) p.lse2[(uint64_t)now.s * p.n_heads + head] = l2;
            }
            if (p.subs == 1u) {
                if (has_row && whole) {
#pragma unroll
                    for (int c = 0; c < NV; c++) {
#pragma unroll
                        for (int r = 0; r < 4; r++) {
                            const uint32_t d = (uint32_t)c * 128u + (kq * 4u + (uint32_t)r) * VW;
                            const f32x4 *a = acc + c * VW;
                            uint32_t w[VW / 2];
#pragma unroll
                            for (int i = 0; i < VW / 2; i++) w[i] = X::pack(a[2 * i][r] * inv * v_scale, a[2 * i + 1][r] * inv * v_scale);
                            if (WHOLE || d < p.dim)
                                *reinterpret_cast<typename Raw<2 * VW>::type *>(out + (uint64_t)head * p.out_head + d * 2u) =
                                    __builtin_bit_cast(typename Raw<2 * VW>::type, w);
                        }
                    }
                } else if (has_row) {
#pragma unroll
                    for (int i = 0; i < ACC; i++) part[((uint32_t)i * 4u + kq) * p.part_rows + n] = acc[i];
                }
            } else {
                const uint32_t u = wave % p.units_per_wg;
                for (uint32_t i0 = sub * 2u; i0 < ACC; i0 += p.subs * 2u) {
                    f32x4 a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (uint32_t o = 0; o < WAVES; o++) {
                        if (o >= p.subs) break;
                        a[0] += joined[o * p.units_per_wg + u][i0][lane] * scale[o];
                        a[1] += joined[o * p.units_per_wg + u][i0 + 1u][lane] * scale[o];
                    }
                    if (has_row && whole) {
                        // two dimensions at a time
#pragma unroll
                        for (int r = 0; r < 4; r++) {
                            const uint32_t d = i0 / 8u * 128u + (kq * 4u + (uint32_t)r) * VW + i0 % 8u;
                            if (WHOLE || d < p.dim)
                                *reinterpret_cast<uint32_t *>(out + (uint64_t)head * p.out_head + d * 2u) =
                                    X::pack(a[0][r] * inv * v_scale, a[1][r] * inv * v_scale);
                        }
                    } else if (has_row) {
                        part[(i0 * 4u + kq) * p.part_rows + n] = a[0];
                        part[((i0 + 1u) * 4u + kq) * p.part_rows + n] = a[1];
                    }
                }
                if (next.here) __syncthreads();
            }
        }
        if (!next.here) break;
        at += next.here;
        now = next;
        next = part_at(now.s + 1u, 0u, at);
    }
}

constexpr uint32_t kMaxGroups = 256;    // ranges of a call

// Joins what several ranges left of one request: out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.  Bound by the
// launch itself: behind a kernel that has filled the caches one that returns at once takes 4.7 us, this one 5.4 (4
// requests in 65 ranges each, 8.5 MB of parts), 6.5 (one request in 256), 7.8 with the weights of 32 requests' blocks.
struct Joined {
    float top, sum, own;  // reference, sum of weights as they met the values, as they were
    f32x4 all[4];
    __device__ __forceinline__ void none()
    {
        top = kLowest;
        sum = own = 0.f;
#pragma unroll
        for (int i = 0; i < 4; i++) all[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void add(const f32x4 &x, const f32x4 (&o)[4])
    {
        const float next = fmaxf(top, x.x), f = __builtin_amdgcn_exp2f(top - next), g = __builtin_amdgcn_exp2f(x.x - next);
        top = next;
        sum = sum * f + x.y * g;
        own = own * f + x.z * g;
#pragma unroll
        for (int i = 0; i < 4; i++) all[i] = all[i] * f + o[i] * g;
    }
    // with what the lanes `step` away hold
    __device__ __forceinline__ void add_lanes(int step)
    {
        const f32x4 x = {__shfl_xor(top, step, 64), __shfl_xor(sum, step, 64), __shfl_xor(own, step, 64), 0.f};
        f32x4 o[4];
#pragma unroll
        for (int i = 0; i < 16; i++) o[i / 4][i & 3] = __shfl_xor(all[i / 4][i & 3], step, 64);
        add(x, o);
    }
};

// A lane has four vectors of a range's part that follow one another along i, 4 x 4 dimensions, so
// that it has 4 dimensions to store at a time.  8 lanes take a range; a wave takes up to 8 ranges
// at once, or, of a request in fewer, as many more places; of a request in more, where that
// takes fewer turns, the four waves of a workgroup take a quarter of the ranges each.
template <typename X>
__device__ __forceinline__ void join(const AttendParams &p, uint32_t s, uint32_t wg, uint32_t wgs, uint32_t n_parts, uint32_t g0)
{
    __shared__ f32x4 ml[4][8];
    __shared__ f32x4 rest[4][4][8];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, u = lane & 7u, q = lane >> 3;
    const uint32_t vecs = p.units * p.part_vecs, items = vecs / 4u, lines = (items + 7u) / 8u;
    const uint32_t bits = n_parts <= 1u ? 0u : n_parts <= 2u ? 1u : n_parts <= 4u ? 2u : 3u;
    auto turns = [](uint32_t n, uint32_t each) { return (n + each - 1u) / each; };
    const bool wide = n_parts > 8u && turns(lines, wgs) * turns(n_parts, 64u) < turns(lines, wgs * 4u) * turns(n_parts, 16u);
    const uint32_t at_once = wide ? 32u : 1u << bits, c = wide ? wave * 8u + q : q & (at_once - 1u);  // ranges
    const uint32_t first = wide ? wg : (wg * 4u + wave) << (3u - bits), step = wide ? wgs : wgs * 4u << (3u - bits);
    for (uint32_t line0 = first; line0 < lines; line0 += step) {
        const uint32_t item = (line0 + (wide ? 0u : q >> bits)) * 8u + u;
        const uint32_t unit = p.by_items.quotient(item), in_unit = item - unit * (p.part_vecs / 4u);
        const uint32_t row_of_i4 = p.by_rows.quotient(in_unit), i4 = row_of_i4 >> 2, kq = row_of_i4 & 3u;
        const uint32_t kv_head = p.by_head_tiles.quotient(unit);
        const uint32_t in_group = (unit - kv_head * p.head_tiles) * 16u + in_unit - row_of_i4 * p.part_rows;
        const uint32_t head = kv_head * p.group_heads + in_group;
        const bool here = item < items && in_group < p.group_heads;
        const uint32_t vec = unit * p.part_vecs + (i4 * 16u + kq) * p.part_rows + in_unit - row_of_i4 * p.part_rows;
        Joined j;
        j.none();
        for (uint32_t base = 0; base < n_parts; base += 2u * at_once) {
            f32x4 x[2], o[2][4];
#pragma unroll
            for (uint32_t k = 0; k < 2; k++) {
                const uint32_t i = base + c + at_once * k;
                const uint64_t slot = (g0 + i) * 2u + (i == 0u ? 1u : 0u);
                x[k] = f32x4{kLowest, 0.f, 0.f, 0.f};
#pragma unroll
                for (uint32_t m = 0; m < 4; m++) o[k][m] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (i < n_parts && here) {
                    x[k] = p.part_ml[slot * p.n_heads + head];
#pragma unroll
                    for (uint32_t m = 0; m < 4; m++) o[k][m] = p.part[slot * vecs + vec + m * 4u * p.part_rows];
                }
            }
#pragma unroll
            for (uint32_t k = 0; k < 2; k++) j.add(x[k], o[k]);
        }
        for (uint32_t m = 8; m < 8u * min(at_once, 8u); m <<= 1) j.add_lanes((int)m);
        if (wide) {
            __syncthreads();
            if (q == 0u) {
                ml[wave][u] = f32x4{j.top, j.sum, j.own, 0.f};
#pragma unroll
                for (int i = 0; i < 4; i++) rest[wave][i][u] = j.all[i];
            }
            __syncthreads();
            if (threadIdx.x < 8u) {
                for (int w = 1; w < 4; w++) {
                    const f32x4 o[4] = {rest[w][0][u], rest[w][1][u], rest[w][2][u], rest[w][3][u]};
                    j.add(ml[w][u], o);
                }
            }
        }
        if (!here || c != 0u) continue;
        const float inv = j.sum == 0.f ? 0.f : 1.0f / j.sum;
        const uint32_t vw = p.dim <= 64u ? 4u : 8u;
        uint8_t *const to = p.out + (uint64_t)s * p.out_row + (uint64_t)head * p.out_head;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const uint32_t d = i4 / 2u * 128u + (kq * 4u + (uint32_t)r) * vw + (i4 & 1u) * 4u;
            if (d < p.dim)
                *reinterpret_cast<w32x2 *>(to + d * 2u) = w32x2{X::pack(j.all[0][r] * inv * p.v_scale, j.all[1][r] * inv * p.v_scale),
                                                                X::pack(j.all[2][r] * inv * p.v_scale, j.all[3][r] * inv * p.v_scale)};
        }
        if (p.lse && row_of_i4 == 0u)
            p.lse[(uint64_t)s * p.n_heads + head] =
                j.own == 0.f ? -__builtin_inff() : (j.top + __builtin_amdgcn_logf(j.own)) * 0.693147180559945309f;
    }
}

// Blocks of a workgroup that adds up weights, two for the same lanes.
__host__ __device__ __forceinline__ uint32_t mass_blocks(uint32_t mass_bits) { return 512u >> mass_bits; }

// What each block received: 4, 8 or 16 lanes a block add up 2^(granule - lse) over its granules and all query heads, in
// a fixed order (20 requests of 65381 tokens, 4 heads, blocks of 8: 11.4 us with 4 lanes, 26.7 with 16).  The heads'
// lse are joined once more here, for all blocks of a workgroup at a time, so that this need not wait for the
// workgroups that join.
__device__ __forceinline__ void add_mass(const AttendParams &p, uint32_t s, uint32_t first_block, uint32_t tokens, uint32_t g0, uint32_t g1)
{
    __shared__ float lse[1024];
    __shared__ float2 some[256];
    const uint32_t tid = threadIdx.x, lanes = 1u << p.mass_bits, part = tid & (lanes - 1u), apart = 256u >> p.mass_bits;
    // the first granules of a lane are under way while the heads' lse are found
    constexpr uint32_t kAhead = 4;
    const uint32_t per_block = p.block_size >> p.granule_bits, n_gran = (tokens + p.granule - 1u) >> p.granule_bits;
    const float *from[2];
    uint32_t n[2];
    float ahead[2][kAhead];
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const uint32_t j = first_block + apart * (uint32_t)k + (tid >> p.mass_bits), f = min(j * per_block, n_gran), l = min(f + per_block, n_gran);
        from[k] = p.granules + ((uint64_t)s * p.max_granules + f) * p.n_heads;
        n[k] = (l - f) * p.n_heads;
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++) ahead[k][i] = part + lanes * i < n[k] ? from[k][part + lanes * i] : 0.f;
    }
    if (g0 == g1) {
        for (uint32_t h = tid; h < p.n_heads; h += 256u) lse[h] = tokens ? p.lse2[(uint64_t)s * p.n_heads + h] : 0.f;
    } else {
        const uint32_t across = min(p.n_heads, 256u), parts = 256u / across, h0 = tid % across, from = tid / across;
        for (uint32_t h = h0; h - h0 < p.n_heads; h += across) {
            float top = kLowest, sum = 0.f;
            if (h < p.n_heads && from < parts) {
#pragma unroll 8
                for (uint32_t g = g0 + from; g <= g1; g += parts) {
                    const float l2 = p.part_ml[(uint64_t)(g * 2u + (g == g0 ? 1u : 0u)) * p.n_heads + h].w, m = fmaxf(top, l2);
                    sum = sum * __builtin_amdgcn_exp2f(top - m) + __builtin_amdgcn_exp2f(l2 - m);
                    top = m;
                }
            }
            __syncthreads();
            some[tid] = float2{top, sum};
            __syncthreads();
            if (tid < across && h < p.n_heads) {
                for (uint32_t i = 1; i < parts; i++) top = fmaxf(top, some[i * across + tid].x);
                sum = 0.f;
                for (uint32_t i = 0; i < parts; i++) sum += some[i * across + tid].y * __builtin_amdgcn_exp2f(some[i * across + tid].x - top);
                lse[h] = sum == 0.f ? -__builtin_inff() : top + __builtin_amdgcn_logf(sum);
            }
        }
    }
    const uint32_t part_head = part % p.n_heads, step = lanes % p.n_heads;  // heads of a lane's numbers
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; k++) {
        const uint32_t j = first_block + apart * (uint32_t)k + (tid >> p.mass_bits);
        float sum = 0.f;
        uint32_t h = part_head;
        auto add = [&](float granule) {
            sum += lse[h] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(granule - lse[h]);
            h += step;
            h = h < p.n_heads ? h : h - p.n_heads;
        };
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++)
            if (part + lanes * i < n[k]) add(ahead[k][i]);
#pragma unroll 4
        for (uint32_t i = part + lanes * kAhead; i < n[k]; i += lanes) add(from[k][i]);
        for (uint32_t d = lanes / 2u; d > 0u; d >>= 1) sum += __shfl_xor(sum, (int)d, 64);
        if (part == 0u && j < p.max_blocks) {
            const int64_t at = (int64_t)s * p.mass_stride + j;
            p.mass_out[at] = (p.mass ? p.mass[at] : 0.f) + sum;
        }
    }
}

// What is left when all ranges are done: a row of workgroups per request, first those that join, then
// those that add up the blocks' weights.
template <typename X>
__global__ __launch_bounds__(256) void kv_join_kernel(const AttendParams p)
{
    const uint32_t s = blockIdx.y, lane = threadIdx.x & 63u;
    const uint32_t tokens = seq_tokens(p.lens, s, p.max_tokens), n_tiles = tiles_of(tokens);
    const Deal deal(p, lane, s);
    const uint32_t first = deal.before;
    const uint32_t g0 = p.by_request ? 0u : first / deal.per, g1 = p.by_request ? 0u : n_tiles ? (first + n_tiles - 1u) / deal.per : g0;
    if (blockIdx.x >= p.joins) add_mass(p, s, (blockIdx.x - p.joins) * mass_blocks(p.mass_bits), tokens, g0, g1);
    else if (!n_tiles || g0 != g1) join<X>(p, s, blockIdx.x, p.joins, n_tiles ? g1 - g0 + 1u : 0u, g0);
}

// ---- new tokens into the cache ---------------------------------------------------------------

// A scale of an 8-bit cache, part * 2^bits with part from 1/2 up to 1, and 2^-kUp / part.
struct Scale {
    static constexpr int kUp = 40;
    float scale, inv;
    static Scale of(float scale)
    {
        int bits;
        return Scale{scale, __builtin_ldexpf(1.0f / __builtin_frexpf(scale, &bits), -kUp)};
    }
};

// values / scale, at most 448 either way, such that the nearest e4m3 values of q are those of the quotients.  A product with
// 1 / part is within two steps of 32 bits of the quotient, which may be on the other side of the middle between two e4m3
// values, or on it.  So the product's last four bits are rounded off (a middle has 5 digits), and by what is left of the value then, all
// of which 32 bits hold, the result is moved a little up, a little down or not at all.  us, the product alone / so: 2000 rows of
// 12 + 3 + 3 heads of 80 into 8 bits 6.2 / 6.5.
template <int N>
__host__ __device__ __forceinline__ void over(const float (&values)[N], const Scale &s, float (&q)[N])
{
    int bits;
    const float part = __builtin_ldexpf(__builtin_frexpf(s.scale, &bits), Scale::kUp), top = 447.0f * part;  // (447 becomes 448)
#pragma unroll
    for (int i = 0; i < N; i++) {
        float x = __builtin_ldexpf(__builtin_fabsf(values[i]), Scale::kUp - bits);
        x = x > top ? top : x;  // NaN stays
        const float c = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x * s.inv) + 8u) & ~15u);
        const float left = __builtin_fmaf(-c, part, x);
        q[i] = __builtin_copysignf(__builtin_fmaf(c, fminf(fmaxf(left, -0x1p-20f), 0x1p-20f), c), values[i]);
    }
}

struct PutParams {
    uint8_t *k, *v;
    const int32_t *table, *lens, *starts;
    const uint8_t *ks, *vs, *qs;
    uint8_t *qd;
    const float *inv_freq;
    const int32_t *positions;
    uint64_t k_row, k_head, v_row, v_head, q_row, q_head, qd_row, qd_head;  // bytes
    int64_t table_stride, position_stride;
    uint32_t n_seqs, n_rows, n_heads, n_kv_heads, max_blocks;
    uint32_t dim, token_bytes, head_bytes, block_size, cells_per_block, n_blocks;
    uint32_t rot, interleaved, section0, section01;  // pairs of the first axis, of the first two
    Divide by_steps, by_vecs;  // by a rotated head's steps, and by a head's vectors
    Scale k_scale, v_scale;
    // normed heads, 4 bits
    const float *q_norm, *k_norm;
    float eps, inv_dim;
    uint32_t exponents;  // from a token's first byte to its heads' bytes
};

// The nearest e4m3 values of four numbers up to 448.  (The conversion has no bounds of its own: beyond, it gives NaN.)
__device__ __forceinline__ uint32_t to_fp8(float a, float b, float c, float d)
{
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// The nearest 16-bit or 8-bit values of N numbers.
template <typename X, bool FP8, int N>
__device__ __forceinline__ void store_row(uint8_t *to, uint32_t d, const float (&x)[N], const Scale &s)
{
    if constexpr (FP8) {
        uint32_t w[N / 4];
        float q[N];
        over(x, s, q);
#pragma unroll
        for (int i = 0; i < N / 4; i++) w[i] = to_fp8(q[4 * i], q[4 * i + 1], q[4 * i + 2], q[4 * i + 3]);
        __builtin_nontemporal_store(__builtin_bit_cast(typename Raw<N>::type, w), reinterpret_cast<typename Raw<N>::type *>(to + d));
    } else {
        uint32_t w[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; i++) w[i] = X::pack(x[2 * i], x[2 * i + 1]);
        __builtin_nontemporal_store(__builtin_bit_cast(typename Raw<2 * N>::type, w), reinterpret_cast<typename Raw<2 * N>::type *>(to + d * 2u));
    }
}

// A workgroup has a row.  A thread's first place (N dimensions, or where the halves of pairs lie apart N of each half)
// is asked for first; while it arrives, the angles are found, one pair a thread, and left in LDS for all
// heads, and the row's page is looked up.  Rows are short: what counts is how many of them a CU has under way, so
// a thread holds one place at a time (8192 rows of 32 + 8 + 8 heads of 128, us: four places in flight 41.8, two
// 35.7, one 33.0; loads that stay in the caches 39.1 with two; stores that do not 32.5 with one.  168 MB in
// 32.5 us are 5.2 TB/s in and out, what a large copy reaches is 5.0).
template <typename X, bool FP8, int N>
__global__ __launch_bounds__(512) void kv_put_kernel(const PutParams p)
{
    typedef typename Raw<2 * N>::type raw;
    __shared__ float2 turn[128];
    const uint32_t row = blockIdx.x, tid = threadIdx.x, lane = tid & 63u;
    // the request whose row this is: as many as begin behind the first, up to it
    uint32_t s = row, start = row, next = row + 1u;
    if (p.starts) {
        s = 0;
        for (uint32_t base = 1; base <= p.n_seqs; base += 64u)
            s += (uint32_t)__popcll(__ballot(base + lane <= p.n_seqs && p.starts[base + lane] <= (int32_t)row));
        if (s >= p.n_seqs || (int32_t)row < p.starts[0]) return;
        start = (uint32_t)p.starts[s];
        next = (uint32_t)p.starts[s + 1u];
    }
    const uint32_t vecs = p.dim / N, apart = p.interleaved ? 0u : p.rot / (2u * N);  // steps of the lower halves
    const uint32_t steps = vecs - apart;                                             // steps of a rotated head
    const uint32_t n_q = p.qs ? p.n_heads * steps : 0u, n_k = n_q + p.n_kv_heads * steps, n_all = n_k + p.n_kv_heads * vecs;
    const uint32_t pairs = p.rot / 2u;
    bool page = false;
    uint8_t *kc = nullptr, *vc = nullptr;
    for (uint32_t first = 0; first < n_all; first += blockDim.x) {
        raw a, b;
        clear(a);
        clear(b);
        const uint32_t i = first + tid;
        uint32_t head = 0, d = 0;
        bool two = false;
        if (i < n_all) {
            const uint32_t in = i < n_q ? i : i < n_k ? i - n_q : i - n_k;
            head = i < n_k ? p.by_steps.quotient(in) : p.by_vecs.quotient(in);
            const uint32_t step = in - head * (i < n_k ? steps : vecs);
            const uint8_t *const src = i < n_q ? p.qs + row * p.q_row + head * p.q_head
                                       : i < n_k ? p.ks + row * p.k_row + head * p.k_head
                                                 : p.vs + row * p.v_row + head * p.v_head;
            two = i < n_k && step < apart;
            d = (i < n_k && !two ? step + apart : step) * N;
            a = __builtin_nontemporal_load(reinterpret_cast<const raw *>(src + d * 2u));
            if (two) b = __builtin_nontemporal_load(reinterpret_cast<const raw *>(src + (d + pairs) * 2u));
        }
        if (first == 0u) {
            const int64_t token = (int64_t)p.lens[s] - (int64_t)(next - start) + (int64_t)(row - start);
            for (uint32_t i = tid; i < pairs; i += blockDim.x) {
                const uint32_t axis = i < p.section0 ? 0u : i < p.section01 ? 1u : 2u;
                const double pos = p.positions ? (double)p.positions[(int64_t)axis * p.position_stride + row] : (double)token;
                // in 64 bits: whole turns, and what is left of them; the rest as half turns
                const double turns = pos * (double)p.inv_freq[i] * 0.15915494309189533577;
                float sn, cs;
                sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
                turn[i] = float2{cs, sn};
            }
            page = token >= 0 && token < (int64_t)p.max_blocks * p.block_size;
            uint32_t cell = kNoCell;
            if (page) {
                const uint32_t entry = (uint32_t)token / p.block_size;
                cell = cell_in((uint32_t)p.table[(int64_t)s * p.table_stride + entry], p.n_blocks, p.cells_per_block,
                               (uint32_t)token - entry * p.block_size);
                page = cell != kNoCell;
            }
            kc = p.k + (uint64_t)cell * p.token_bytes;  // not looked at without a page
            vc = p.v + (uint64_t)cell * p.token_bytes;
            __syncthreads();
        }
        if (i >= n_all || (i >= n_q && !page)) continue;
        const uint32_t *const wa = reinterpret_cast<const uint32_t *>(&a), *const wb = reinterpret_cast<const uint32_t *>(&b);
        float x[N], y[N];
#pragma unroll
        for (int e = 0; e < N / 2; e++) {
            x[2 * e] = X::lo(wa[e]);
            x[2 * e + 1] = X::hi(wa[e]);
            y[2 * e] = X::lo(wb[e]);
            y[2 * e + 1] = X::hi(wb[e]);
        }
        if (two) {
#pragma unroll
            for (int e = 0; e < N; e++) {
                const float2 c = turn[d + e];
                const float u = x[e] * c.x - y[e] * c.y, w = y[e] * c.x + x[e] * c.y;
                x[e] = u;
                y[e] = w;
            }
        } else if (i < n_k && d < p.rot) {
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const float2 c = turn[(d + e) / 2u];
                const float u = x[e] * c.x - x[e + 1] * c.y, w = x[e + 1] * c.x + x[e] * c.y;
                x[e] = u;
                x[e + 1] = w;
            }
        }
        if (i < n_q) {
            uint8_t *const to = p.qd + row * p.qd_row + head * p.qd_head;
            store_row<X, false>(to, d, x, p.k_scale);
            if (two) store_row<X, false>(to, d + pairs, y, p.k_scale);
        } else {
            uint8_t *const to = (i < n_k ? kc : vc) + head * p.head_bytes;
            const Scale scale = {i < n_k ? p.k_scale.scale : p.v_scale.scale, i < n_k ? p.k_scale.inv : p.v_scale.inv};
            store_row<X, FP8>(to, d, x, scale);
            if (two) store_row<X, FP8>(to, d + pairs, y, scale);
        }
    }
}

// What another of 16 lanes holds, by a lane pattern that needs no LDS: 0xB1 and 0x4E the lane 1 and 2 away of four, 0x141 and
// 0x140 the one as far from the end of 8 and of 16, 0x128 the one 8 away.
template <int CONTROL>
__device__ __forceinline__ float lanes_of(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}

// New tokens whose heads are normed first, or go into 4 bits.  A thread has 8 dimensions of a head, one behind the other,
// and a head lies in 1 to 32 lanes of a wave (a power of 2): the sum of its squares is a sum over lanes, so is
// the largest of 32 dimensions over four, and the other numbers of pairs come from the lanes that have them.
//   y = x / sqrt(mean x^2 + eps) * weight, then the rotation, all in 32 bits, rounded once.
// Bound by vector instructions and by how many rows are under way: 6853 rows of 32 + 8 + 8 heads of 128 into 4 bits (148 MB), us: with sums by
// shuffles through LDS 53.5, over lanes 51, without a choice for each dimension 45, with the row's request in one round of loads 43, of 128 threads
// 39 (3.8 TB/s); 64 rows into 16 bits 4.6.
// 4 bits: the power of 2 is the one that brings the largest of 32 dimensions to 4 and more, under 8, and numbers are the nearest
// of those there are (6 the largest); infinity or NaN among them makes all 32 NaN.
// WHOLE: the lanes of a head all of whose dimensions turn, halves apart, and are so many times 8; 0: any others.
template <typename X, int KIND, int WHOLE>
__global__ __launch_bounds__(512) void kv_put_heads_kernel(const PutParams p, const uint32_t lane_bits)
{
    __shared__ float2 turn[128];
    const uint32_t row = blockIdx.x, tid = threadIdx.x, lane = tid & 63u;
    const uint32_t pairs = p.rot / 2u;
    // asked for before the row's request is known: its position, and what it is multiplied with
    const uint32_t axis = tid < p.section0 ? 0u : tid < p.section01 ? 1u : 2u;
    const int32_t pos0 = tid < pairs && p.positions ? p.positions[(int64_t)axis * p.position_stride + row] : 0;
    const float freq0 = tid < pairs ? p.inv_freq[tid] : 0.f;
    uint32_t s = row, start = row, next = row + 1u;
    int32_t len;
    if (p.starts && p.n_seqs <= 64u) {
        // so few requests that every lane has one: their ends, and their lengths at once
        const int32_t begin = p.starts[0], ends = lane < p.n_seqs ? p.starts[lane + 1u] : 0x7FFFFFFF, lens = lane < p.n_seqs ? p.lens[lane] : 0;
        s = (uint32_t)__popcll(__ballot(ends <= (int32_t)row));
        if (s >= p.n_seqs || (int32_t)row < begin) return;
        start = (uint32_t)(s ? __builtin_amdgcn_readlane(ends, (int)s - 1) : begin);
        next = (uint32_t)__builtin_amdgcn_readlane(ends, (int)s);
        len = __builtin_amdgcn_readlane(lens, (int)s);
    } else if (p.starts) {
        s = 0;
        for (uint32_t base = 1; base <= p.n_seqs; base += 64u)
            s += (uint32_t)__popcll(__ballot(base + lane <= p.n_seqs && p.starts[base + lane] <= (int32_t)row));
        if (s >= p.n_seqs || (int32_t)row < p.starts[0]) return;
        start = (uint32_t)p.starts[s];
        next = (uint32_t)p.starts[s + 1u];
        len = p.lens[s];
    } else {
        len = p.lens[s];
    }
    const uint32_t n_q = p.qs ? p.n_heads : 0u, n_k = n_q + p.n_kv_heads, n_all = n_k + p.n_kv_heads;
    const uint32_t lanes = WHOLE ? (uint32_t)WHOLE : 1u << lane_bits, in = tid & (lanes - 1u), d = in * 8u, at_once = blockDim.x >> lane_bits;
    bool page = false;
    uint8_t *kc = nullptr, *vc = nullptr;
    const uint32_t mine = tid >> lane_bits;
    auto load = [&](uint32_t i) {
        const uint32_t head = i < n_q ? i : i < n_k ? i - n_q : i - n_k;
        w32x4 raw;
        clear(raw);
        if (i < n_all && d < p.dim) {
            const uint8_t *const src = i < n_q ? p.qs + row * p.q_row + head * p.q_head
                                       : i < n_k ? p.ks + row * p.k_row + head * p.k_head
                                                 : p.vs + row * p.v_row + head * p.v_head;
            raw = __builtin_nontemporal_load(reinterpret_cast<const w32x4 *>(src + d * 2u));
        }
        return raw;
    };
    w32x4 next_raw = load(mine);
    for (uint32_t first = 0; first < n_all; first += at_once) {
        const uint32_t i = first + mine, head = i < n_q ? i : i < n_k ? i - n_q : i - n_k;
        const bool here = i < n_all && d < p.dim;
        const w32x4 raw = next_raw;
        next_raw = load(i + at_once);  // a turn ahead
        if (first == 0u) {
            const int64_t token = (int64_t)len - (int64_t)(next - start) + (int64_t)(row - start);
            for (uint32_t i = tid; i < pairs; i += blockDim.x) {
                const uint32_t axis = i < p.section0 ? 0u : i < p.section01 ? 1u : 2u;
                const int32_t at = i == tid || !p.positions ? pos0 : p.positions[(int64_t)axis * p.position_stride + row];
                const double pos = p.positions ? (double)at : (double)token;
                // in 64 bits: whole turns, and what is left of them; the sine of that in half turns
                const double turns = pos * (double)(i == tid ? freq0 : p.inv_freq[i]) * 0.15915494309189533577;
                const double half_turns = 2.0 * (turns - rint(turns));
                float sn, cs;
                sincospif((float)half_turns, &sn, &cs);
                // and by what its nearest 32-bit number is off
                const float off = (float)(half_turns - (double)(float)half_turns) * 3.14159265f;
                turn[i] = float2{__builtin_fmaf(-sn, off, cs), __builtin_fmaf(cs, off, sn)};
            }
            page = token >= 0 && token < (int64_t)p.max_blocks * p.block_size;
            uint32_t cell = kNoCell;
            if (page) {
                const uint32_t entry = (uint32_t)token / p.block_size;
                cell = cell_in((uint32_t)p.table[(int64_t)s * p.table_stride + entry], p.n_blocks, p.cells_per_block,
                               (uint32_t)token - entry * p.block_size);
                page = cell != kNoCell;
            }
            kc = p.k + (uint64_t)cell * p.token_bytes;  // not looked at without a page
            vc = p.v + (uint64_t)cell * p.token_bytes;
            __syncthreads();
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            x[2 * e] = X::lo(raw[e]);
            x[2 * e + 1] = X::hi(raw[e]);
        }
        // (lanes of a head take part together, those behind its dimensions with zeros)
        const float *const weight = i < n_q ? p.q_norm : i < n_k ? p.k_norm : nullptr;
        if (weight) {
            // Small heads and next to no eps: again, of 2^76 times as much.  (The squares of numbers as small as 2^-64 are no normal
            // numbers, of which the root's instruction makes infinity.)
            float mean, eps = p.eps;
            for (bool again = p.eps < 0x1p-90f;; again = false) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; e++) sum = __builtin_fmaf(x[e], x[e], sum);
                // over the head's lanes: neighbours, pairs, then each four, eight and sixteen with its mirror image
                if (lanes > 1u) sum += lanes_of<0xB1>(sum);
                if (lanes > 2u) sum += lanes_of<0x4E>(sum);
                if (lanes > 4u) sum += lanes_of<0x141>(sum);
                if (lanes > 8u) sum += lanes_of<0x140>(sum);
                if (lanes > 16u) sum += __shfl_xor(sum, 16, 64);
                mean = __builtin_fmaf(sum, p.inv_dim, eps);
                if (!again || !__any(mean < 0x1p-90f)) break;
                const float up = mean < 0x1p-90f ? 0x1p76f : 1.0f;
                eps = eps * up * up;
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] *= up;
            }
            // the root's reciprocal to its last bit, a step behind what the instruction gives
            const float r0 = __builtin_amdgcn_rsqf(mean);
            const float left = __builtin_fmaf(-mean * r0, r0, 1.0f), r = left > -1.0f && left < 1.0f ? __builtin_fmaf(r0 * 0.5f, left, r0) : r0;
            if (here) {
                const f32x4 w0 = *reinterpret_cast<const f32x4 *>(weight + d), w1 = *reinterpret_cast<const f32x4 *>(weight + d + 4u);
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = x[e] * r * (e < 4 ? w0[e & 3] : w1[e & 3]);
            }
        }
        if (WHOLE && i < n_k) {
            // each number of a lower half with the one half the lanes away
            const bool lower = in < lanes / 2u;
            const uint32_t at = d & (pairs - 1u);
#pragma unroll
            for (uint32_t e = 0; e < 8; e++) {
                const float other = WHOLE == 16 ? lanes_of<0x128>(x[e]) : __shfl_xor(x[e], WHOLE / 2, 64);
                const float2 c = turn[at + e];
                x[e] = __builtin_fmaf(lower ? -other : other, c.y, x[e] * c.x);
            }
        } else if (p.interleaved && i < n_k && d < p.rot) {
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float2 c = turn[(d + e) / 2u];
                const float u = x[e] * c.x - x[e + 1] * c.y, w = x[e + 1] * c.x + x[e] * c.y;
                x[e] = u;
                x[e + 1] = w;
            }
        } else if (!p.interleaved && p.rot && i < n_k) {
            // four dimensions at a time: those of a thread may be of both halves
            float other[8];
            const uint32_t fours = pairs / 4u, base = lane & ~(lanes - 1u);
#pragma unroll
            for (uint32_t f = 0; f < 2; f++) {
                const uint32_t at = in * 2u + f, from = at < fours ? at + fours : at < 2u * fours ? at - fours : at;
                const int src = (int)(base + from / 2u);
#pragma unroll
                for (uint32_t e = 0; e < 4; e++) {
                    if (fours & 1u) {
                        const float a = __shfl(x[e], src, 64), b = __shfl(x[4 + e], src, 64);
                        other[4 * f + e] = from & 1u ? b : a;
                    } else {
                        other[4 * f + e] = __shfl(x[4 * f + e], src, 64);
                    }
                }
            }
#pragma unroll
            for (uint32_t e = 0; e < 8; e++) {
                const uint32_t at = d + e;
                if (at >= p.rot) continue;
                const bool lower = at < pairs;
                const float2 c = turn[lower ? at : at - pairs];
                x[e] = lower ? x[e] * c.x - other[e] * c.y : x[e] * c.x + other[e] * c.y;
            }
        }
        uint32_t largest = 0;
        if constexpr (KIND == kBits4) {
#pragma unroll
            for (int e = 0; e < 8; e++) largest = max(largest, __builtin_bit_cast(uint32_t, x[e]) & 0x7FFFFFFFu);
            largest = max(largest, __builtin_bit_cast(uint32_t, lanes_of<0xB1>(__builtin_bit_cast(float, largest))));
            largest = max(largest, __builtin_bit_cast(uint32_t, lanes_of<0x4E>(__builtin_bit_cast(float, largest))));
        }
        if (!here || (i >= n_q && !page)) continue;
        if (i < n_q) {
            store_row<X, false>(p.qd + row * p.qd_row + head * p.qd_head, d, x, p.k_scale);
            continue;
        }
        uint8_t *const to = i < n_k ? kc : vc;
        if constexpr (KIND == kBits4) {
            const bool odd = largest >= 0x7F800000u;
            const int byte = min(max((int)(largest >> 23) - 2, X::kLowPower + 127), X::kHighPower + 127);
            const float power = __builtin_bit_cast(float, (uint32_t)byte << 23);
            uint32_t w = 0;
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], power, 0);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], power, 1);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], power, 2);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], power, 3);
            *reinterpret_cast<w32_any *>(to + head * p.head_bytes + d / 2u) = odd ? 0u : w;
            if ((in & 3u) == 0u) to[p.exponents + head * (p.dim / 32u) + d / 32u] = odd ? (uint8_t)255 : (uint8_t)byte;
        } else {
            const Scale scale = {i < n_k ? p.k_scale.scale : p.v_scale.scale, i < n_k ? p.k_scale.inv : p.v_scale.inv};
            store_row<X, KIND == kBits8>(to + head * p.head_bytes, d, x, scale);
        }
    }
}

// ---- eviction --------------------------------------------------------------------------------
struct EvictParams {
    const int32_t *table, *lens;
    int32_t *table_out, *lens_out;
    const float *mass;
    float *mass_out;
    int32_t *ids, *at, *count;
    int64_t table_stride, mass_stride;
    uint32_t max_blocks, block_size, budget, n_first, n_last, max_evict;
};

// Weights as whole numbers of the same order: lightest first, NaN last, -0 as 0.
__host__ __device__ __forceinline__ uint32_t weight_key(float x)
{
    if (x != x) return ~0u;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// One workgroup per request.  A thread holds EACH entries, THREADS apart, of those that are looked at together; a
// row of no more than EACH x THREADS is read once.  The key of the last block to go is found digit by digit, counted
// in LDS, by three of 11 bits and less: the first has 4 steps per power of two, so that few lanes of many meet in
// one count.  Where as a rule few enough entries then begin with it, they are compared with one another instead of
// counted twice more.  Then the row is closed up: a block moves down by the number of those before it that went.
// All that is written lies before all that is read later, so a row may be its own output.
//
// Bound by its own chain of barriers, not by memory: a row of 512 is 4 KB.  Measured, rows of random weights, a
// quarter kept: 64 rows of 512 in 4.3 us (5.1 with counts alone; 5.4 with 256 threads of two entries and 8-bit
// digits), 64 of 2048 entries 6.2 (6.8; 8.9), 64 of 4096 8.9 (11.4 with eight entries a thread), 8 of 8192 entries 11.8; from four
// entries a thread on the comparison costs 1.3 us more than it saves.
template <uint32_t THREADS, uint32_t EACH, uint32_t DIGIT>
__global__ __launch_bounds__(THREADS) void kv_evict_kernel(const EvictParams p)
{
    constexpr uint32_t kWaves = THREADS / 64, kEach = EACH, kAtOnce = kEach * THREADS, kBins = 1u << DIGIT, kOwn = kBins / THREADS;
    const uint32_t s = blockIdx.x, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    __shared__ uint32_t bins[kBins];
    __shared__ uint32_t sums[kWaves];
    __shared__ uint32_t chosen[3];
    __shared__ uint2 counts[kEach * kWaves];
    constexpr bool kCompare = EACH <= 2u;
    constexpr uint32_t kFew = kCompare ? 256u : 1u;
    __shared__ uint2 few[kFew], ranks[kFew];
    __shared__ uint32_t placed;
    if (tid == 0u) placed = 0u;
    const uint32_t tokens = seq_tokens(p.lens, s, p.max_blocks * p.block_size);
    const uint32_t held = (tokens + p.block_size - 1u) / p.block_size;
    const int32_t *const table = p.table + (int64_t)s * p.table_stride;
    const float *const mass = p.mass + (int64_t)s * p.mass_stride;
    int32_t *const table_out = p.table_out + (int64_t)s * p.table_stride;
    float *const mass_out = p.mass_out + (int64_t)s * p.mass_stride;
    int32_t *const ids = p.ids + (int64_t)s * p.max_evict, *const ats = p.at + (int64_t)s * p.max_evict;
    const uint32_t from = min(p.n_first, held), to = held > p.n_last ? max(held - p.n_last, from) : from;  // may go
    const uint32_t go = min(min(held > p.budget ? held - p.budget : 0u, to - from), p.max_evict);
    const bool resident = held <= kAtOnce;
    float m[kEach];
    int32_t id[kEach];
    auto load = [&](uint32_t base, bool with_ids) {
#pragma unroll
        for (uint32_t e = 0; e < kEach; e++) {
            const uint32_t j = base + e * THREADS + tid;
            m[e] = j < held ? mass[j] : 0.f;
            if (with_ids) id[e] = j < held ? table[j] : -1;
        }
    };
    if (resident) load(0u, true);
    // the largest key that goes, and how many of that key do
    uint32_t prefix = 0, known = 0, left = go;
#pragma unroll 1
    for (uint32_t low = 32; low > 0u && go;) {
        const uint32_t bits = min(DIGIT, low), shift = low - bits, digit = (1u << bits) - 1u;
        low = shift;
#pragma unroll
        for (uint32_t i = 0; i < kOwn; i++) bins[kOwn * tid + i] = 0u;
        __syncthreads();
        for (uint32_t base = 0; base < to; base += kAtOnce) {
            if (!resident) load(base, false);
#pragma unroll
            for (uint32_t e = 0; e < kEach; e++) {
                const uint32_t j = base + e * THREADS + tid, key = weight_key(m[e]);
                if (j >= from && j < to && (key & known) == prefix) atomicAdd(&bins[key >> shift & digit], 1u);
            }
        }
        __syncthreads();
        uint32_t own[kOwn], all = 0;
#pragma unroll
        for (uint32_t i = 0; i < kOwn; i++) all += own[i] = bins[kOwn * tid + i];
        const uint32_t upto = wave_scan(all);
        if (lane == 63u) sums[wave] = upto;
        __syncthreads();
        uint32_t before = upto - all;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; w++) before += w < wave ? sums[w] : 0u;
#pragma unroll
        for (uint32_t i = 0; i < kOwn; i++) {
            if (before < left && left <= before + own[i]) {
                chosen[0] = kOwn * tid + i;
                chosen[1] = left - before;
                chosen[2] = own[i];
            }
            before += own[i];
        }
        __syncthreads();
        prefix |= chosen[0] << shift;
        known |= digit << shift;
        left = chosen[1];
        const uint32_t n = chosen[2];
        if (left == n) {  // all that begin so go
            prefix |= ~known;
            break;
        }
        if (kCompare && low > 0u && resident && n <= kFew) {
            // few begin so: each is compared with all, and the one that `left - 1` others go before is the last to go
            if (tid < kFew) ranks[tid] = uint2{0u, 0u};
#pragma unroll
            for (uint32_t e = 0; e < kEach; e++) {
                const uint32_t j = e * THREADS + tid, key = weight_key(m[e]);
                if (j >= from && j < to && (key & known) == prefix) few[atomicAdd(&placed, 1u)] = uint2{key, j};
            }
            __syncthreads();
            const uint32_t c = tid % kFew;
            const uint2 mine = few[c];
            if (c < n) {
                uint32_t less = 0, before = 0;
                for (uint32_t i = tid / kFew; i < n; i += THREADS / kFew) {
                    const uint2 other = few[i];
                    less += other.x < mine.x ? 1u : 0u;
                    before += other.x == mine.x && other.y < mine.y ? 1u : 0u;
                }
                atomicAdd(&ranks[c].x, less);
                atomicAdd(&ranks[c].y, before);
            }
            __syncthreads();
            if (tid < n && ranks[tid].x + ranks[tid].y == left - 1u) {
                chosen[0] = mine.x;
                chosen[1] = left - ranks[tid].x;
            }
            __syncthreads();
            prefix = chosen[0];
            left = chosen[1];
            break;
        }
    }
    const uint64_t below = (1ull << lane) - 1u;
    uint32_t less_base = 0, tie_base = 0;  // of the entries looked at before
    for (uint32_t base = 0; base < held; base += kAtOnce) {
        if (!resident) load(base, true);
        uint32_t less = 0, tie = 0;  // bit e
        uint64_t bl[kEach], bt[kEach];
#pragma unroll
        for (uint32_t e = 0; e < kEach; e++) {
            const uint32_t j = base + e * THREADS + tid, key = weight_key(m[e]);
            const bool may = go && j >= from && j < to;
            less |= may && key < prefix ? 1u << e : 0u;
            tie |= may && key == prefix ? 1u << e : 0u;
            bl[e] = __ballot(less >> e & 1u);
            bt[e] = __ballot(tie >> e & 1u);
            if (lane == 0u) counts[e * kWaves + wave] = uint2{(uint32_t)__popcll(bl[e]), (uint32_t)__popcll(bt[e])};
        }
        __syncthreads();
        if (wave == 0u) {  // sums of those before each, in the order of the entries
            constexpr uint32_t kPer = (kEach * kWaves + 63u) / 64u;
            uint2 c[kPer], sum = {0u, 0u};
#pragma unroll
            for (uint32_t i = 0; i < kPer; i++) {
                c[i] = kPer * lane + i < kEach * kWaves ? counts[kPer * lane + i] : uint2{0u, 0u};
                sum.x += c[i].x;
                sum.y += c[i].y;
            }
            const uint32_t l = wave_scan(sum.x), t = wave_scan(sum.y);
            uint2 first = {l - sum.x, t - sum.y};
#pragma unroll
            for (uint32_t i = 0; i < kPer; i++) {
                if (kPer * lane + i < kEach * kWaves) counts[kPer * lane + i] = first;
                first.x += c[i].x;
                first.y += c[i].y;
            }
            if (lane == 63u) {
                chosen[0] = l;
                chosen[1] = t;
            }
        }
        __syncthreads();
#pragma unroll
        for (uint32_t e = 0; e < kEach; e++) {
            const uint32_t j = base + e * THREADS + tid;
            if (j >= held) continue;
            const uint2 c = counts[e * kWaves + wave];
            const uint32_t tie_before = tie_base + c.y + (uint32_t)__popcll(bt[e] & below);
            const uint32_t gone = less_base + c.x + (uint32_t)__popcll(bl[e] & below) + min(tie_before, left);
            if (less >> e & 1u || (tie >> e & 1u && tie_before < left)) {
                ids[gone] = id[e];
                ats[gone] = (int32_t)j;
            } else {
                table_out[j - gone] = id[e];
                mass_out[j - gone] = m[e];
            }
        }
        less_base += chosen[0];
        tie_base += chosen[1];
        __syncthreads();
    }
    for (uint32_t j = held - go + tid; j < p.max_blocks; j += THREADS) {
        table_out[j] = -1;
        mass_out[j] = 0.f;
    }
    for (uint32_t j = go + tid; j < p.max_evict; j += THREADS) ids[j] = ats[j] = -1;
    if (tid == 0) {
        p.count[s] = (int32_t)go;
        p.lens_out[s] = (int32_t)(tokens - go * p.block_size);
    }
}

}  // namespace dkv
