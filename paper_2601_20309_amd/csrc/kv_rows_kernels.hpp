// Device kernels of attention of many rows per request over the paged cache (gfx950, wave64).
#pragma once
#include "kv_decode_kernels.hpp"

namespace dkv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

// ---- attention of many rows -------------------------------------------------------------------
//
// Row i of a request's m rows sees the tokens before u_i: u_i = length - m + i + 1, or the whole length. Over those in
// present pages: scores s_t = c q.k_t, weights w_t = 2^(s_t - reference), out = sum w_t v_t / sum w_t, one pass over the
// tokens with a running reference.  The query heads of a KV head are rows, too: heads of a row lie one
// behind the other, so that few rows of many heads fill a tile, and all of them share the keys that are brought.
//
// A workgroup has 128 or 256 rows of one KV head, 32 a wave, and goes over the tokens 64 at a time (32 above 128 dimensions), or, where
// requests have few rows, 32 rows, and its waves take turns at the tokens.  These go into LDS, two tiles in
// turn: in 16 bits whatever the cache holds, so that the products are the same for every type of cache.  Both products are taken
// transposed, tokens x rows and dimensions x rows, as in kv_attend: a lane has one row, its reference and its sums, and
// weights come out as the second product's operand.  Values are read from LDS transposed, four tokens of a dimension at a time.
//
// Scores, references and both sums are held in 32 bits.  A weight meets the values as the nearest number of their type: X, fp16 beside 8
// bits (here products bound the time, and two numbers for a weight would make it half as many again); out is divided by the sum of the weights as they were,
// so that lse has 32 bits.  Errors against 64 bits, root of the mean square, 1e-4, of 300 to 5000
// tokens / of the outputs' own rounding: bf16 22 / 16.6, fp16 2.7 / 2.05, bf16 beside 8 bits 16.7 / 16.6 (a bf16 number for a weight 22).
//
// What bounds it: LDS.  Of 64 tokens a wave reads 32 KB for 32 products of 32 x 32 x 16, and a CU's eight waves that much each.  1024
// rows of 64 heads over 8 of 128 at 31000 tokens take 925 us (1110 TFLOP/s), of 256 rows to a workgroup.  What that is made of, of 128 rows to
// one, which took 1050: without loads 854, without reads of LDS 932, without exponentials 988, the products alone 524.  Beside
// 945 two waves' halves of a step in alternation, with a barrier between them, took 1012; beside 1050 64 rows a wave and one wave to a SIMD,
// which halve the reads, 1227.
// 16-bit rows go from memory into LDS directly: 4 prompts of 2048 tokens 489 us through registers, 194 so.

struct RowsParams {
    const uint8_t *k, *v;
    const int32_t *table, *lens, *starts;
    const uint8_t *q;
    uint8_t *out;
    float *lse;
    const uint8_t *zeros;  // 16 bytes
    f32x4 *part;      // [slot][32 rows][vector][lane]: sums of a part of the tokens, as they lie in registers
    float2 *part_ml;  // [slot][row]: reference, sum of weights
    uint64_t q_row, q_head, out_row, out_head;  // bytes
    int64_t table_stride;
    uint32_t n_seqs, n_rows, n_heads, n_kv_heads, max_tokens;
    uint32_t dim, token_bytes, head_bytes, block_size, cells_per_block, n_blocks;
    uint32_t exponents;  // 4 bits: from a token's first byte to its exponents
    uint32_t group_heads, causal;
    // Parts of the tokens, `least` tiles of tokens and more each: splits of a tile of rows, slots [tile][split][KV head]; or, of
    // tiles of 32 rows, `groups` ranges of all (0: none), slots [range][its last request, or one that begins in it][KV head]
    uint32_t splits, least, groups;
    uint32_t n_tiles, row_bits;                   // tiles of rows of a KV head, empty ones among them; log2 of the rows of one
    Divide by_block, by_group;
    uint32_t negative;  // the scale is: keys meet -q
    float qk_scale;     // to base 2, not negative
    float v_scale;
    float bias;         // beside bf16: of Weights
};

template <typename X>
__device__ __forceinline__ Weights weights(const RowsParams &p)
{
    if constexpr (std::is_same_v<X, Fp16>) return {X::kBias, X::kSlack};
    else return {p.bias, kBf16Slack};
}

// Which rows a tile has.  Request s's tiles are floor(starts[s] * group / rows of one) + s on: as many as it needs, or
// some more, which are empty.  So no sums over requests are needed to find one.
struct RowTile {
    uint32_t s, first;      // request; its rows' heads before this tile
    int32_t start, m;       // the request's first row, and its number of rows
    int32_t len;            // its tokens
    bool here;
};

// Up to 64 requests: every lane has one, so that finding one takes one round of loads.
struct Requests {
    int32_t start, next, len;
    __device__ __forceinline__ Requests(const RowsParams &p, uint32_t lane) : start(0x7FFFFFFF), next(0x7FFFFFFF), len(0)
    {
        if (p.n_seqs > 64u || lane >= p.n_seqs) return;
        start = p.starts ? p.starts[lane] : (int32_t)lane;
        next = p.starts ? p.starts[lane + 1u] : (int32_t)lane + 1;
        len = p.lens[lane];
    }
    // Request s's, from a lane or from memory.
    __device__ __forceinline__ void of(const RowsParams &p, uint32_t s, int32_t &first, int32_t &last, int32_t &tokens) const
    {
        if (p.n_seqs <= 64u) {
            first = __builtin_amdgcn_readlane(start, (int)s);
            last = __builtin_amdgcn_readlane(next, (int)s);
            tokens = __builtin_amdgcn_readlane(len, (int)s);
        } else {
            first = p.starts ? p.starts[s] : (int32_t)s;
            last = p.starts ? p.starts[s + 1u] : (int32_t)s + 1;
            tokens = p.lens[s];
        }
    }
};

__device__ __forceinline__ uint32_t first_tile(const RowsParams &p, uint32_t s, int32_t start)
{
    return (uint32_t)((uint64_t)(uint32_t)max(start, 0) * p.group_heads >> p.row_bits) + s;
}

__device__ __forceinline__ int32_t rows_of(const RowsParams &p, int32_t start, int32_t next)
{
    return start < 0 ? 0 : (int32_t)min(max((int64_t)next - start, (int64_t)0), (int64_t)p.n_rows);
}

__device__ __forceinline__ RowTile row_tile(const RowsParams &p, const Requests &requests, uint32_t lane, uint32_t tile)
{
    RowTile t;
    // the last request whose first tile is not behind this one, 64 candidates at a time
    uint32_t lo = 0;
    if (p.n_seqs <= 64u) {
        const uint64_t before = __ballot(lane < p.n_seqs && first_tile(p, lane, requests.start) <= tile);
        lo = before ? 63u - (uint32_t)__builtin_clzll(before) : 0u;
    } else {
        for (uint32_t range = p.n_seqs; range > 1u;) {
            const uint32_t step = (range + 63u) / 64u, at = lo + lane * step;
            const uint64_t before = __ballot(lane * step < range && first_tile(p, at, p.starts ? p.starts[at] : (int32_t)at) <= tile);
            const uint32_t n = before ? 63u - (uint32_t)__builtin_clzll(before) : 0u;
            range = min(step, range - n * step);
            lo += n * step;
        }
    }
    t.s = __builtin_amdgcn_readfirstlane(lo);
    int32_t next;
    requests.of(p, t.s, t.start, next, t.len);
    t.m = rows_of(p, t.start, next);
    const uint32_t base = first_tile(p, t.s, t.start);
    const uint64_t first = (uint64_t)(tile - base) << p.row_bits;
    t.here = tile >= base && first < (uint64_t)t.m * p.group_heads;
    t.first = (uint32_t)first;
    return t;
}

// Tokens before which row i of the request looks.
__device__ __forceinline__ int32_t row_sees(const RowsParams &p, const RowTile &t, uint32_t row)
{
    const int64_t upto = p.causal ? (int64_t)t.len - t.m + (int64_t)row + 1 : (int64_t)t.len;
    return (int32_t)min(max(upto, (int64_t)0), (int64_t)p.max_tokens);
}

// Tiles of tokens that a tile of rows looks at, and how many of its splits have any.
struct Spread {
    uint32_t tiles, per, active;
    __device__ __forceinline__ Spread(const RowsParams &p, uint32_t upto, uint32_t tokens)
    {
        tiles = (upto + tokens - 1u) / tokens;
        per = max((tiles + p.splits - 1u) / p.splits, p.least);
        active = (tiles + per - 1u) / per;
    }
};

// Ranges: the tiles of tokens of all tiles of 32 rows, one behind the other, are dealt to p.groups equal ranges, whatever
// requests' lengths and rows.  Every wave finds out for itself, 64 requests at a time.
struct RowDeal {
    uint32_t total, per, before;  // tiles of tokens; of a range; of the requests before the one asked for
    uint32_t mine, upto;          // of request (n_seqs - 1) / 64 * 64 + lane; of its 64 up to and with it
    // Tiles of tokens of a request, the same for each of its tiles of rows, and those in all.
    static __device__ __forceinline__ uint32_t tokens_of(const RowsParams &p, int32_t len) { return ((uint32_t)min(max(len, 0), (int32_t)p.max_tokens) + 31u) / 32u; }
    static __device__ __forceinline__ uint32_t work(const RowsParams &p, const Requests &requests, uint32_t s)
    {
        if (s >= p.n_seqs) return 0u;
        int32_t start = requests.start, next = requests.next, len = requests.len;
        if (p.n_seqs > 64u) requests.of(p, s, start, next, len);
        return ((uint32_t)rows_of(p, start, next) * p.group_heads + 31u) / 32u * tokens_of(p, len);
    }
    __device__ __forceinline__ RowDeal(const RowsParams &p, const Requests &requests, uint32_t lane, uint32_t asked) : total(0), per(1), before(0), mine(0), upto(0)
    {
        if (!p.groups) return;
        for (uint32_t base = 0; base < p.n_seqs; base += 64u) {
            mine = work(p, requests, base + lane);
            upto = wave_scan(mine);
            if (asked >= base && asked - base < 64u) before = total + (uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), (int)(asked - base));
            total += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        per = max((total + p.groups - 1u) / p.groups, p.least);
    }
    // The request that tile `at` is of, and how many of its tiles come before.
    __device__ __forceinline__ bool find(const RowsParams &p, const Requests &requests, uint32_t lane, uint32_t at, uint32_t &s, uint32_t &t) const
    {
        uint32_t m = mine, u = upto, first = 0;
        for (uint32_t base = 0; base < p.n_seqs; base += 64u) {
            if (p.n_seqs > 64u) {
                m = work(p, requests, base + lane);
                u = wave_scan(m);
            }
            const uint64_t beyond = __ballot(first + u > at);
            if (beyond) {
                const uint32_t l = (uint32_t)__builtin_ctzll(beyond);
                s = base + l;
                t = at - first - (uint32_t)__builtin_amdgcn_readlane((int)(u - m), (int)l);
                return true;
            }
            first += (uint32_t)__builtin_amdgcn_readlane((int)u, 63);
        }
        return false;  // (starts that fall)
    }
};

template <typename X>
__device__ __forceinline__ f32x16 mma32(w32x4 a, w32x4 b, f32x16 c)
{
    if constexpr (std::is_same_v<X, Fp16>)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(typename X::x8, a), __builtin_bit_cast(typename X::x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(typename X::x8, a), __builtin_bit_cast(typename X::x8, b), c, 0, 0, 0);
}

// A mean of numbers of X that its weights' roundings have put above the largest of them is that one.
template <typename X, bool OF_X>
__device__ __forceinline__ float mean(float x)
{
    return OF_X && __builtin_fabsf(x) < __builtin_inff() ? fminf(fmaxf(x, -X::kMost), X::kMost) : x;
}

// ROWS 128 and 256: four or eight waves have 32 rows each, and share tiles of tokens.  ROWS 32: all waves have the same rows, and take turns at the
// tiles of tokens, each with LDS of its own, so that nothing waits for the others.
constexpr int kManyRowsDims = 128;  // 256 rows: eight waves have no more than 256 registers each
template <int DP, int ROWS>
struct RowStep {
    static constexpr bool TURNS = ROWS == 32;
    static constexpr int TOKENS = TURNS || DP > 128 ? 32 : 64;
    static constexpr int WAVES = TURNS ? (DP > 128 ? 2 : 4) : ROWS / 32;
    static constexpr int PITCH = DP <= 64 ? 64 : DP <= 128 ? 128 : 256;  // of a token in LDS, in numbers
    static constexpr int CHUNKS = PITCH / 8;
    static constexpr int NB = DP / 32, KS = DP / 16, TB = TOKENS / 32;
    // Where 8 numbers lie: keys are read 16 bytes a lane, 32 tokens at once, values 32 dimensions of 8 tokens at once.
    static __device__ __forceinline__ uint32_t key_turn(uint32_t token) { return PITCH == 64 ? token >> 1 & 7u : token & 15u; }
    static __device__ __forceinline__ uint32_t value_turn(uint32_t token) { return (PITCH == 64 ? token >> 1 & 1u : token & 3u) << 2; }
    static __device__ __forceinline__ uint32_t key_at(uint32_t token, uint32_t chunk) { return (token * CHUNKS + (chunk ^ key_turn(token))) * 8u; }
    static __device__ __forceinline__ uint32_t value_at(uint32_t token, uint32_t chunk) { return (token * CHUNKS + (chunk ^ value_turn(token))) * 8u; }
};

// As much of a row of the cache as a thread takes at once, and what it becomes.
template <typename X, int KIND>
struct Piece;
template <typename X>
struct Piece<X, kBits16> {
    static constexpr int N = 8;
    w32x4 raw;
    __device__ __forceinline__ void load(const uint8_t *row, uint32_t d, uint32_t) { raw = *reinterpret_cast<const w32x4 *>(row + d * 2u); }
    __device__ __forceinline__ void none() { clear(raw); }
    __device__ __forceinline__ w32x4 out(int) const { return raw; }
};
template <typename X>
struct Piece<X, kBits8> {
    static constexpr int N = 8;
    w32x2 raw;
    __device__ __forceinline__ void load(const uint8_t *row, uint32_t d, uint32_t) { raw = *reinterpret_cast<const w32x2 *>(row + d); }
    __device__ __forceinline__ void none() { clear(raw); }
    __device__ __forceinline__ w32x4 out(int) const
    {
        return w32x4{X::template from_fp8<false>(raw[0]), X::template from_fp8<true>(raw[0]), X::template from_fp8<false>(raw[1]),
                     X::template from_fp8<true>(raw[1])};
    }
};
template <typename X>
struct Piece<X, kBits4> {
    static constexpr int N = 32;
    w32x4 raw;
    uint32_t exponent;
    __device__ __forceinline__ void load(const uint8_t *row, uint32_t d, uint32_t powers)
    {
        raw = *reinterpret_cast<const w32x4_any *>(row + d / 2u);
        exponent = row[powers + d / 32u];
    }
    __device__ __forceinline__ void none() { clear(raw); exponent = 0u; }
    __device__ __forceinline__ w32x4 out(int i) const
    {
        const float scale = __builtin_bit_cast(float, exponent << 23);
        return w32x4{X::template from_fp4<0>(raw[i], scale), X::template from_fp4<1>(raw[i], scale), X::template from_fp4<2>(raw[i], scale),
                     X::template from_fp4<3>(raw[i], scale)};
    }
};

// 16 bytes a lane from global memory into LDS, one lane's behind the other's from `to` on.  In assembly, since beside the
// builtin the compiler waits for all reads of LDS where some would do, as long as one of these is under way.  Whoever looks at
// what came waits for it first (loaded_lds), and then for the other waves.  (m0 is a register that the compiler sets where it
// needs it, and would warn that nobody else's value in it is kept: none is.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(const uint8_t *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_address(const uint16_t *p)
{
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p);
}
__device__ __forceinline__ void loaded_lds() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// N products of which each reads LDS READS times: the reads are AHEAD products ahead, those of the first ones done.
template <int N, int READS, int AHEAD>
__device__ __forceinline__ void pipeline()
{
    constexpr int kMma = 0x008, kRead = 0x100;
#pragma unroll
    for (int i = 0; i < N - AHEAD; i++) {
        __builtin_amdgcn_sched_group_barrier(kMma, 1, 0);
        __builtin_amdgcn_sched_group_barrier(kRead, READS, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMma, AHEAD, 0);
}

// What a workgroup keeps in LDS, and the waves of a SIMD that leaves room for: no more than two, which have 256 registers each.
template <int KIND, int DP, int ROWS>
struct RowLds {
    using T = RowStep<DP, ROWS>;
    // Numbers that go through registers are stored when the tile before them has been read: of a wave's own tiles one is enough.
    static constexpr uint32_t BUFS = T::TURNS && KIND != kBits16 ? 1 : 2;
    static constexpr uint32_t PLANE = T::TOKENS * T::PITCH, TILE = 2 * PLANE;
    static constexpr uint32_t NUMBERS = BUFS * TILE * (T::TURNS ? T::WAVES : 1), SUMS = T::TURNS ? T::WAVES * 32 : 1, MARKS = ROWS * T::NB * 2;
    static constexpr uint32_t BYTES = NUMBERS * 2 + SUMS * 8 + MARKS * 4 + 4;
    static constexpr int AT_ONCE = (int)(160 * 1024 / BYTES) * T::WAVES / 4;
    // Above 192 dimensions what passes through registers has one wave to a SIMD, too.  (us, one / two with scratch memory, prompts as at
    // READY: 8 bits 146 / 172, 4 bits 147 / 148; in 16 bits 131 / 120, without.)
    static constexpr int WAVES_OF_SIMD = AT_ONCE < 2 || (DP > 192 && KIND != kBits16) ? 1 : 2;
};

template <typename X, int KIND, int DP, int ROWS>
__global__ __launch_bounds__((64 * RowStep<DP, ROWS>::WAVES), (RowLds<KIND, DP, ROWS>::WAVES_OF_SIMD)) void kv_rows_kernel(const RowsParams p)
{
    using T = RowStep<DP, ROWS>;
    // The type of the second product: beside 8 bits fp16, which holds the values exactly, and of a weight as much as one number can.
    using Y = std::conditional_t<KIND == kBits8, Fp16, X>;
    using P = Piece<X, KIND>;  // of keys
    constexpr int TOKENS = T::TOKENS, NB = T::NB, KS = T::KS, TB = T::TB, WAVES = T::WAVES;
    constexpr bool DIRECT = KIND == kBits16, TURNS = T::TURNS;
    constexpr uint32_t SHARING = TURNS ? 1 : WAVES, STEP = TURNS ? WAVES : 1;  // waves of a tile of tokens; tiles of a turn
    constexpr uint32_t UNITS = TOKENS * DP / P::N, ROW_UNITS = DP / P::N;      // pieces of a tile, of a token
    constexpr uint32_t LANES = 64 * SHARING;
    // Operands that are ready before the first product: of 256 dimensions no more than the registers hold.  (us, two / six, which then wait in
    // scratch memory, two prompts of 2048 tokens, 16 heads over 4 of 256: 120 / 135.)
    constexpr int READY = DP > 192 ? 2 : KS * TB < 6 ? KS * TB : 6;
    constexpr int EACH = DIRECT ? 1 : (UNITS + LANES - 1) / LANES;
    using L = RowLds<KIND, DP, ROWS>;
    constexpr uint32_t BUFS = L::BUFS, PLANE = L::PLANE, TILE = L::TILE, VECS = NB * 4;
    // of each wave (or all): tiles of keys and values; at the end sums
    __shared__ __attribute__((aligned(16))) uint16_t lds[L::NUMBERS];
    __shared__ float2 ml[L::SUMS];
    // of each row and dimension: whether it sees infinities or NaN that were taken out, of either sign
    __shared__ uint32_t marks[L::MARKS];
    __shared__ uint32_t any;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t n = lane & 31u, h = lane >> 5;
    // KV heads first, so that those of one request's tiles meet in one die's cache
    const uint32_t kv_head = blockIdx.x % p.n_kv_heads, rest = blockIdx.x / p.n_kv_heads;
    const uint8_t *const kb = p.k + (uint64_t)kv_head * p.head_bytes;
    const uint8_t *const vb = p.v + (uint64_t)kv_head * p.head_bytes;
    uint16_t *const tiles = lds + (TURNS ? wave * BUFS * TILE : 0u);
    const uint32_t tiles_at = lds_address(tiles + (TURNS ? 0u : wave * (512u / T::PITCH) * T::PITCH));  // where this wave's loads go
    // Tiles of tokens `first` to `stop` of a tile of rows, a part of them or all.
    auto run = [&](const RowTile &rt, uint32_t first_tokens, uint32_t stop, bool parts, uint64_t slot) {
    const uint32_t last_flat = min(rt.first + ROWS, (uint32_t)rt.m * p.group_heads) - 1u;
    const uint32_t most = (uint32_t)row_sees(p, rt, p.by_group.quotient(last_flat));
    const uint32_t fewest = (uint32_t)row_sees(p, rt, p.by_group.quotient(rt.first));
    const uint32_t begin = first_tokens + (TURNS ? wave : 0u), end = min(stop, (most + TOKENS - 1u) / TOKENS);
    const uint32_t flat = rt.first + (TURNS ? 0u : wave * 32u) + n, row = p.by_group.quotient(flat), head = kv_head * p.group_heads + flat - row * p.group_heads;
    const uint32_t at_row = (uint32_t)rt.start + row;
    const bool has_row = row < (uint32_t)rt.m && at_row < p.n_rows;
    const uint32_t sees = has_row ? (uint32_t)row_sees(p, rt, row) : 0u;
    // 4 bits: from a token's numbers of this head to the head's powers of 2
    const uint32_t powers = KIND == kBits4 ? p.exponents + kv_head * (p.dim / 32u) - kv_head * p.head_bytes : 0u;
    const int32_t *const pages = p.table + (int64_t)rt.s * p.table_stride;

    for (uint32_t i = tid; i < ROWS * NB * 2; i += 64u * WAVES) marks[i] = 0u;
    if (tid == 0u) any = 0u;
    if constexpr (TURNS) __syncthreads();  // (otherwise: the one of the first tile)
    uint32_t half = h;
    asm volatile("" : "+v"(half));  // (what goes by it is found anew for every tile of rows: kept, it does not fit the registers)
    w32x4 qf[KS];
#pragma unroll
    for (int j = 0; j < KS; j++) {
        const uint32_t d = (uint32_t)j * 16u + half * 8u;
        clear(qf[j]);
        if (has_row && d < p.dim) qf[j] = *reinterpret_cast<const w32x4 *>(p.q + (uint64_t)at_row * p.q_row + (uint64_t)head * p.q_head + d * 2u);
        if (p.negative) qf[j] ^= 0x80008000u;
    }
    // Of a tile every wave has a lane for each token: its page, then the row of the cache.
    auto page_of = [&](uint32_t tile) {
        const uint32_t token = tile * TOKENS + lane % TOKENS;
        return token < most ? (uint32_t)pages[p.by_block.quotient(token)] : kNoCell;
    };
    auto cell_of = [&](uint32_t tile, uint32_t page) {
        const uint32_t token = tile * TOKENS + lane % TOKENS;
        return cell_in(page, p.n_blocks, p.cells_per_block, token - p.by_block.quotient(token) * p.block_size);
    };
    P kp[EACH];
    Piece<Y, KIND> vp[EACH];
    auto load = [&](auto buf, uint32_t cell) {
        if constexpr (DIRECT) {
            // a wave brings 512 numbers at once, whole tokens, each lane the 8 that belong where its lane's go
            // (turns of token + EVERY i are those of either, one with the other: they have no bit in common)
            constexpr uint32_t AT_ONCE = 512 / T::PITCH, EVERY = AT_ONCE * SHARING;
            uint32_t l = lane;
            uint32_t to = __builtin_amdgcn_readfirstlane(tiles_at);
            asm volatile("" : "+v"(l), "+s"(to));  // (found anew for every tile: kept, these are what does not fit the registers)
            to += buf() * TILE * 2u;
            const uint32_t mine = TURNS ? 0u : wave * AT_ONCE, token = mine + l / T::CHUNKS, slot = l % T::CHUNKS;
            const uint32_t ck = slot ^ T::key_turn(token), cv = slot ^ T::value_turn(token);
            const uint64_t off = (uint64_t)cell * p.token_bytes;
            const bool whole = p.dim == T::PITCH && !__any(cell == kNoCell);
#pragma unroll
            for (uint32_t i = 0; i < TOKENS / EVERY; i++) {
                const int from = (int)((token + i * EVERY) * 4u);
                const uint32_t lo = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(uint32_t)off), hi = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(off >> 32));
                const uint64_t at = (uint64_t)hi << 32 | lo;
                const uint32_t dk = (ck ^ T::key_turn(i * EVERY)) * 8u, dv = (cv ^ T::value_turn(i * EVERY)) * 8u;
                const uint8_t *k = kb + dk * 2u + at, *v = vb + dv * 2u + at;
                if (!whole) {
                    const bool here = __builtin_amdgcn_ds_bpermute(from, (int)cell) != (int)kNoCell;
                    if (!here || dk >= p.dim) k = p.zeros;
                    if (!here || dv >= p.dim) v = p.zeros;
                }
                load_lds(k, to + i * EVERY * T::PITCH * 2u);
                load_lds(v, to + PLANE * 2u + i * EVERY * T::PITCH * 2u);
            }
        } else {
            uint32_t first = tid % LANES;
            asm volatile("" : "+v"(first));
#pragma unroll
            for (int i = 0; i < EACH; i++) {
                const uint32_t u = first + LANES * (uint32_t)i, token = u / ROW_UNITS, d = u % ROW_UNITS * P::N;
                const uint32_t c = (uint32_t)__shfl((int)cell, (int)(token % TOKENS), 64);
                kp[i].none();
                vp[i].none();
                if ((UNITS % LANES == 0u || u < UNITS) && c != kNoCell && d < p.dim) {
                    const uint64_t off = (uint64_t)c * p.token_bytes;
                    kp[i].load(kb + off, d, powers);
                    vp[i].load(vb + off, d, powers);
                }
            }
        }
    };
    auto store = [&](auto buf) {
        if constexpr (!DIRECT) {
            uint16_t *const keys = tiles + (BUFS > 1 ? buf() : 0) * TILE, *const values = keys + PLANE;
            uint32_t first = tid % LANES;
            asm volatile("" : "+v"(first));
#pragma unroll
            for (int i = 0; i < EACH; i++) {
                const uint32_t u = first + LANES * (uint32_t)i, token = u / ROW_UNITS, chunk = u % ROW_UNITS * (P::N / 8);
                if (UNITS % LANES != 0u && u >= UNITS) break;
#pragma unroll
                for (int e = 0; e < P::N / 8; e++) {
                    *reinterpret_cast<w32x4 *>(keys + T::key_at(token, chunk + e)) = kp[i].out(e);
                    *reinterpret_cast<w32x4 *>(values + T::value_at(token, chunk + e)) = vp[i].out(e);
                }
            }
        }
    };

    f32x16 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; b++)
#pragma unroll
        for (int i = 0; i < 16; i++) acc[b][i] = 0.f;
    const Weights largest = weights<Y>(p);
    float ref = kLowest, own = 0.f;
    uint64_t next_present = 0;
    uint32_t page = kNoCell;
    typedef std::integral_constant<int, 0> Zero;
    typedef std::integral_constant<int, 1> One;
    if (begin < end) {
        const uint32_t cell = cell_of(begin, page_of(begin));
        next_present = __ballot(cell != kNoCell);
        load(Zero{}, cell);
        if (begin + STEP < end) page = page_of(begin + STEP);
        store(Zero{});
    }
    auto step = [&](auto buf, auto other, uint32_t t) {
        uint16_t *const keys = tiles + (BUFS > 1 ? buf() : 0) * TILE, *const values = keys + PLANE;
        const uint64_t present = next_present;
        if constexpr (DIRECT) loaded_lds();
        if constexpr (!TURNS) __syncthreads();
        // The first operands of either product are asked for before what comes between: the next tile's places, the weights.
        // (chunk 2 j + h of a token begins at key_at(token, h), bits of 2 j turned round)
        auto key = [&](int i) {
            return *reinterpret_cast<const w32x4 *>(keys + (uint32_t)(i % TB) * 32u * T::PITCH + (T::key_at(n, h) ^ (uint32_t)(i / TB) * 16u));
        };
        w32x4 ready[READY];
#pragma unroll
        for (int i = 0; i < READY; i++) ready[i] = key(i);
        if (t + STEP < end) {
            const uint32_t cell = cell_of(t + STEP, page);
            next_present = __ballot(cell != kNoCell);
            load(other, cell);
            if (t + 2u * STEP < end) page = page_of(t + 2u * STEP);
        }
        const bool border = (t + 1u) * TOKENS > fewest;
        f32x16 s[TB];
#pragma unroll
        for (int b = 0; b < TB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) s[b][i] = 0.f;
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < KS * TB; i++) s[i % TB] = mma32<X>(i < READY ? ready[i] : key(i), qf[i / TB], s[i % TB]);
        pipeline<KS * TB, 1, READY>();
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        // register i of block b: token b * 32 + i / 4 * 8 + h * 4 + i % 4
        const uint64_t all = TOKENS == 64 ? ~0ull : 0xFFFFFFFFull;
        if (border || (present & all) != all) {
            const int32_t left = (int32_t)sees - (int32_t)(t * TOKENS + h * 4u);
            const uint64_t there = present >> (h * 4u);
#pragma unroll
            for (int b = 0; b < TB; b++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int token = b * 32 + i / 4 * 8 + i % 4;
                    s[b][i] = token < left && (there >> token & 1u) ? s[b][i] : -__builtin_inff();
                }
        }
        if (border) {
            // A weight of 0 does not make up for a value of infinity or NaN.  Where not all rows see all tokens, those become 0 here, and
            // what they make of the rows that see them is noted.
            for (uint32_t u = tid % LANES; u < TOKENS * (DP / 8u); u += LANES) {
                const uint32_t token = u / (DP / 8u), chunk = u - token * (DP / 8u);
                w32x4 *const at = reinterpret_cast<w32x4 *>(values + T::value_at(token, chunk));
                w32x4 v = *at;
                if (!(Y::odd(v[0]) | Y::odd(v[1]) | Y::odd(v[2]) | Y::odd(v[3]))) continue;
                for (uint32_t e = 0; e < 8; e++) {
                    const uint32_t word = e / 2 == 0u ? v[0] : e / 2 == 1u ? v[1] : e / 2 == 2u ? v[2] : v[3], x = e & 1u ? word >> 16 : word & 0xFFFFu;
                    if (!Y::odd(x)) continue;
                    const bool nan = Y::nan(x);
                    reinterpret_cast<uint16_t *>(at)[e] = 0;
                    for (uint32_t r = 0; r < ROWS; r++) {
                        const uint32_t row = p.by_group.quotient(rt.first + r);
                        if (row >= (uint32_t)rt.m || (uint32_t)row_sees(p, rt, row) <= t * TOKENS + token) continue;
                        uint32_t *const m = marks + (r * NB + chunk / 4u) * 2u;
                        const uint32_t bit = 1u << (chunk % 4u * 8u + e);
                        if (nan || !(x & 0x8000u)) atomicOr(m, bit);
                        if (nan || x & 0x8000u) atomicOr(m + 1, bit);
                    }
                    any = 1u;
                }
            }
            if constexpr (!TURNS) __syncthreads();
        }
        // 16 lanes bring 4 tokens of 16 dimensions, and have 4 tokens of a dimension each
        auto value = [&](int i) {
            const int k = i / NB, b = i % NB;
            const uint32_t token = h * 4u + (lane & 15u) / 4u, d = (lane & 16u) + (lane & 3u) * 4u;
            const uint32_t at = (T::value_at(token, d / 8u) + (d & 4u)) ^ (uint32_t)b * 32u;
            w32x4 a;
#pragma unroll
            for (uint32_t half = 0; half < 2; half++) {
                const uint16_t *from = values + ((uint32_t)k * 16u + half * 8u) * T::PITCH + at;
                const w32x2 x = __builtin_bit_cast(w32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)from));
                a[half * 2u] = x[0];
                a[half * 2u + 1u] = x[1];
            }
            return a;
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < READY; i++) ready[i] = value(i);
        __builtin_amdgcn_sched_barrier(0);
        float top = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < TB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) top = fmaxf(top, s[b][i]);
        top *= p.qk_scale;
        if (__any(top > ref + (largest.bias + largest.slack))) {
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float higher = fmaxf(ref, top - largest.bias), shrink = __builtin_amdgcn_exp2f(ref - higher);
            ref = higher;
            own *= shrink;
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
                for (int i = 0; i < 16; i++) acc[b][i] *= shrink;
        }
        w32x4 w[2 * TB];
#pragma unroll
        for (int b = 0; b < TB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], p.qk_scale, -ref));
                own += s[b][i];
                if (i & 1) w[b * 2 + i / 8][i % 8 / 2] = Y::pack(s[b][i - 1], s[b][i]);
            }
        asm volatile("" : "+v"(own));  // (added up here, not behind the products, where all of the weights would have to be kept)
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < 2 * TB * NB; i++) acc[i % NB] = mma32<Y>(i < READY ? ready[i] : value(i), w[i / NB], acc[i % NB]);
        pipeline<2 * TB * NB, 2, READY>();
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        if (t + STEP < end) store(other);
    };
    for (uint32_t t = begin; t < end; t += 2u * STEP) {
        step(Zero{}, One{}, t);
        if (t + STEP < end) step(One{}, Zero{}, t + STEP);
    }
    own += __shfl_xor(own, 32, 64);
    // vector v of a lane: 4 dimensions, 32 (v / 4) + 8 (v % 4) + 4 h on
    f32x4 *const part = p.part + (slot * (ROWS / 32) + (TURNS ? 0u : wave)) * VECS * 64u + lane;
    uint8_t *const out = p.out + (uint64_t)at_row * p.out_row + (uint64_t)head * p.out_head;
    auto put = [&](uint32_t v, f32x4 a, float inv) {
        const uint32_t d = v / 4u * 32u + v % 4u * 8u + half * 4u;
        // (without a tile of tokens there was no barrier behind the one who cleared these, and nothing to note)
        if ((TURNS || begin < end) && any) {
            const uint32_t *const m = marks + (((TURNS ? 0u : wave * 32u) + n) * NB + v / 4u) * 2u;
            const uint32_t up = m[0] >> (d & 31u), down = m[1] >> (d & 31u);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                a[e] += up >> e & 1u ? __builtin_inff() : 0.f;
                a[e] -= down >> e & 1u ? __builtin_inff() : 0.f;
            }
        }
        if (parts) {
            part[v * 64u] = a;
        } else if (has_row && d < p.dim) {
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] = mean<X, KIND == kBits16>(a[e] * inv) * p.v_scale;
            *reinterpret_cast<w32x2 *>(out + d * 2u) = w32x2{X::pack(o[0], o[1]), X::pack(o[2], o[3])};
        }
    };
    if constexpr (TURNS) {
        // what each wave has goes into LDS, and each joins its share of the dimensions
        f32x4 *const sums = reinterpret_cast<f32x4 *>(lds);
        static_assert(sizeof lds >= WAVES * VECS * 64u * 16u, "room for the sums");
        __syncthreads();
#pragma unroll
        for (uint32_t v = 0; v < VECS; v++) sums[(wave * VECS + v) * 64u + lane] = f32x4{acc[v / 4][v % 4 * 4], acc[v / 4][v % 4 * 4 + 1], acc[v / 4][v % 4 * 4 + 2], acc[v / 4][v % 4 * 4 + 3]};
        if (h == 0u) ml[wave * 32u + n] = float2{ref, own};
        __syncthreads();
        float scale[WAVES];
        float2 x[WAVES];
#pragma unroll
        for (uint32_t o = 0; o < WAVES; o++) {
            x[o] = ml[o * 32u + n];
            ref = fmaxf(ref, x[o].x);
        }
        own = 0.f;
#pragma unroll
        for (uint32_t o = 0; o < WAVES; o++) {
            scale[o] = __builtin_amdgcn_exp2f(x[o].x - ref);
            own += x[o].y * scale[o];
        }
        const float inv = own == 0.f ? 0.f : 1.0f / own;
#pragma unroll
        for (uint32_t i = 0; i < VECS / WAVES; i++) {
            const uint32_t v = wave * (VECS / WAVES) + i;
            f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t o = 0; o < WAVES; o++) a += sums[(o * VECS + v) * 64u + lane] * scale[o];
            put(v, a, inv);
        }
        __syncthreads();
        if (wave != 0u) return;
    } else {
        const float inv = own == 0.f ? 0.f : 1.0f / own;
#pragma unroll
        for (uint32_t v = 0; v < VECS; v++) put(v, f32x4{acc[v / 4][v % 4 * 4], acc[v / 4][v % 4 * 4 + 1], acc[v / 4][v % 4 * 4 + 2], acc[v / 4][v % 4 * 4 + 3]}, inv);
    }
    if (h != 0u) return;
    if (parts) p.part_ml[slot * ROWS + (TURNS ? 0u : wave * 32u) + n] = float2{ref, own};
    else if (has_row && p.lse) p.lse[(uint64_t)at_row * p.n_heads + head] = own == 0.f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(own)) * 0.693147180559945309f;
    };
    const Requests requests(p, lane);
    RowTile rt;
    if constexpr (TURNS) {
        // (run() once in the code, whether the workgroup has a range or a tile)
        const RowDeal deal(p, requests, lane, 0u);
        uint32_t at = p.groups ? rest * deal.per : 0u, here = 1u;
        const uint32_t stop = p.groups ? min(at + deal.per, deal.total) : 1u;
        for (; at < stop; at += here) {
            uint32_t first = 0, last = ~0u;
            uint64_t slot = 0;
            bool parts = false;
            if (p.groups) {
                uint32_t t;
                int32_t next;
                if (!deal.find(p, requests, lane, at, rt.s, t)) return;
                requests.of(p, rt.s, rt.start, next, rt.len);
                rt.m = rows_of(p, rt.start, next);
                const uint32_t tokens = RowDeal::tokens_of(p, rt.len), tile = t / tokens;
                first = t - tile * tokens;
                here = min(tokens - first, stop - at);
                last = first + here;
                parts = here < tokens;
                slot = (uint64_t)(rest * 2u + (first ? 0u : 1u)) * p.n_kv_heads + kv_head;
                rt.first = tile * 32u;
            } else {
                rt = row_tile(p, requests, lane, rest);
                if (!rt.here) return;
            }
            run(rt, first, last, parts, slot);
        }
    } else {
        // last rows, which see most, first
        const uint32_t split = rest % p.splits, tile = p.n_tiles - 1u - rest / p.splits;
        rt = row_tile(p, requests, lane, tile);
        if (!rt.here) return;
        const uint32_t last_flat = min(rt.first + ROWS, (uint32_t)rt.m * p.group_heads) - 1u;
        const Spread spread(p, (uint32_t)row_sees(p, rt, p.by_group.quotient(last_flat)), TOKENS);
        if (split >= max(spread.active, 1u)) return;
        run(rt, split * spread.per, split * spread.per + spread.per, spread.active > 1u, ((uint64_t)tile * p.splits + split) * p.n_kv_heads + kv_head);
    }
}

// Joins the parts of a tile: a wave has 32 rows and 32 dimensions of them, and four parts at a time.  WIDE: so has a workgroup, and its
// waves every fourth part each.  (us, wide / not: 9 requests of 150 rows in four splits 7.8 / 6.0; 16 requests of up to 8005 tokens, 5 rows
// of 40 heads over 8, in 64 ranges a KV head 5.6 / 7.2.)
template <typename X, bool BITS16, bool WIDE>
__global__ __launch_bounds__(256) void kv_rows_join_kernel(const RowsParams p, uint32_t blocks, uint32_t tokens)
{
    constexpr uint32_t WAVES = WIDE ? 4 : 1;
    __shared__ f32x4 sums[WAVES][4][64];
    __shared__ float2 refs[WAVES][64];
    const uint32_t lane = threadIdx.x & 63u, n = lane & 31u, h = lane >> 5, own_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t quarter = WIDE ? own_wave : 0u, item = WIDE ? blockIdx.x : blockIdx.x * 4u + own_wave;
    const uint32_t of_tile = blocks << (p.row_bits - 5u);  // items of a tile
    const uint32_t rest = item / of_tile, in = item - rest * of_tile;
    const uint32_t b = in % blocks, wave = in / blocks, kv_head = rest % p.n_kv_heads, tile = rest / p.n_kv_heads;
    if (tile >= p.n_tiles) return;
    const Requests requests(p, lane);
    const RowTile rt = row_tile(p, requests, lane, tile);
    if (!rt.here) return;
    uint32_t parts, g0 = 0;
    if (p.groups) {
        const uint32_t n_tokens = RowDeal::tokens_of(p, rt.len);
        const RowDeal deal(p, requests, lane, rt.s);
        const uint32_t first = deal.before + rt.first / 32u * n_tokens;
        g0 = first / deal.per;
        parts = n_tokens ? min((first + n_tokens - 1u) / deal.per, p.groups - 1u) - g0 + 1u : 0u;
        if (parts == 1u) return;  // (none: no range has a request without tokens)
    } else {
        const uint32_t last_flat = min(rt.first + (1u << p.row_bits), (uint32_t)rt.m * p.group_heads) - 1u;
        parts = Spread(p, (uint32_t)row_sees(p, rt, p.by_group.quotient(last_flat)), tokens).active;
        if (parts <= 1u) return;
    }
    const uint32_t flat = rt.first + wave * 32u + n, row = p.by_group.quotient(flat), head = kv_head * p.group_heads + flat - row * p.group_heads;
    const uint32_t at_row = (uint32_t)rt.start + row;
    const bool has_row = row < (uint32_t)rt.m && at_row < p.n_rows;
    float ref = kLowest, own = 0.f;
    f32x4 all[4];
#pragma unroll
    for (int i = 0; i < 4; i++) all[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr uint32_t AT_ONCE = 4;
    auto add = [&](const float2 &ml, const f32x4 (&part)[4]) {
        const float next = fmaxf(ref, ml.x), f = __builtin_amdgcn_exp2f(ref - next), g = __builtin_amdgcn_exp2f(ml.x - next);
        ref = next;
        own = own * f + ml.y * g;
#pragma unroll
        for (int i = 0; i < 4; i++) all[i] = all[i] * f + part[i] * g;
    };
    for (uint32_t first = quarter; first < parts; first += WAVES * AT_ONCE) {
        float2 ml[AT_ONCE];
        f32x4 part[AT_ONCE][4];
#pragma unroll
        for (uint32_t o = 0; o < AT_ONCE; o++) {
            const uint32_t i = min(first + WAVES * o, parts - 1u);
            const uint64_t slot = (p.groups ? (uint64_t)(g0 + i) * 2u + (i ? 0u : 1u) : (uint64_t)tile * p.splits + i) * p.n_kv_heads + kv_head;
            ml[o] = p.part_ml[(slot << p.row_bits) + wave * 32u + n];
#pragma unroll
            for (int j = 0; j < 4; j++) part[o][j] = p.part[(((slot << (p.row_bits - 5u)) + wave) * (blocks * 4u) + b * 4u + j) * 64u + lane];
        }
#pragma unroll
        for (uint32_t o = 0; o < AT_ONCE; o++)
            if (first + WAVES * o < parts) add(ml[o], part[o]);
    }
    if constexpr (WIDE) {
        refs[quarter][lane] = float2{ref, own};
#pragma unroll
        for (int i = 0; i < 4; i++) sums[quarter][i][lane] = all[i];
        __syncthreads();
        if (quarter) return;
        for (uint32_t o = 1; o < min(parts, 4u); o++) {
            const f32x4 part[4] = {sums[o][0][lane], sums[o][1][lane], sums[o][2][lane], sums[o][3][lane]};
            add(refs[o][lane], part);
        }
    }
    if (!has_row) return;
    const float inv = own == 0.f ? 0.f : 1.0f / own;
    uint8_t *const out = p.out + (uint64_t)at_row * p.out_row + (uint64_t)head * p.out_head;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t d = b * 32u + (uint32_t)i * 8u + h * 4u;
        if (d >= p.dim) continue;
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] = mean<X, BITS16>(all[i][e] * inv) * p.v_scale;
        *reinterpret_cast<w32x2 *>(out + d * 2u) = w32x2{X::pack(o[0], o[1]), X::pack(o[2], o[3])};
    }
    if (p.lse && h == 0u && b == 0u)
        p.lse[(uint64_t)at_row * p.n_heads + head] = own == 0.f ? -__builtin_inff() : (ref + __builtin_amdgcn_logf(own)) * 0.693147180559945309f;
}

}  // namespace dkv
