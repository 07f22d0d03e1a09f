// Device kernels of a decode step over the paged cache (gfx950, wave64): new
// tokens into their pages, attention of one new token per request, eviction of
// blocks by the weight attention gave them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dkv {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t w32x2 __attribute__((ext_vector_type(2)));

// The 16-bit types of q, k, v and the outputs.
struct Bf16 {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x2 __attribute__((ext_vector_type(2)));
    // Weights are exp2(score - reference): the reference is at most kSlack below the largest score.
    static constexpr float kBias = 0.0f, kSlack = 8.0f;
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
    static constexpr uint32_t kOnes = 0x3F803F80u;
};

struct Fp16 {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x2 __attribute__((ext_vector_type(2)));
    // fp16 has normal numbers from 2^-14 to 2^15: the largest weights lie between 2^8 and 2^15,
    // which leaves 22 powers of two below them before a weight loses digits.
    static constexpr float kBias = 8.0f, kSlack = 7.0f;
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
    static constexpr uint32_t kOnes = 0x3C003C00u;
};

// ---- attention of one new token --------------------------------------------------------------
//
// scores s_t = q.k_t, weights w_t = exp2(c s_t - m), out = sum w_t v_t / sum w_t with a running
// reference m.  Every key and value is read once, so HBM bounds it: a matrix instruction per
// 16 x 16 x 32 products does what the vector units could not beside the loads.
//
// Work is cut into tiles of 32 tokens of one request.  The tiles of all requests, one behind
// the other, are dealt to `groups` equal ranges, whatever the requests' lengths; a range
// belongs to one workgroup (or several that share the KV heads).  A wave has one KV head and up
// to 16 of its query heads (a unit); where there are fewer units than waves, several
// waves take turns at the tiles of a range and join in LDS.  A request that lies in one
// range is finished there; others leave sum, reference and unnormalised output per range, and
// kv_join_kernel joins them.
//
// No operand passes through LDS.  The products are taken transposed, tokens x heads and
// dimensions x heads, so that the weights come out where the second product wants
// them: lane (n, kq) = (lane % 16, lane / 16) holds of head n the tokens kq * 4 + r and
// 16 + kq * 4 + r (r < 4), which are the eight its operand takes if the values are
// brought in the same order (the order of a contraction is free).  For the values it loads
// 8 dimensions of each of those eight tokens, 16 lanes a row, whole rows of 256 bytes, and puts
// the pairs of tokens that a dimension's operand is made of together with byte permutes.
struct AttendParams {
    const uint8_t *k, *v;      // the layer's planes
    const int32_t *table, *lens;
    const uint8_t *q;
    uint8_t *out;
    float *lse;                // nullptr: not wanted
    float *part;               // [groups * 2][n_heads][dim], unnormalised
    f32x4 *part_ml;            // [groups * 2][n_heads]: reference, sum of rounded weights, sum of weights, -
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
    uint32_t groups, wgs_per_group, units, units_per_wg, subs, group_heads, head_tiles;
    uint32_t granule, max_granules;
    float qk_scale;            // to base 2
    float v_scale;
};

constexpr uint32_t kTile = 32;
constexpr uint32_t kNoCell = ~0u;

__device__ __forceinline__ uint32_t seq_tokens(const int32_t *lens, uint32_t s, uint32_t most)
{
    return (uint32_t)min(max(lens[s], 0), (int32_t)most);
}

__device__ __forceinline__ uint32_t tiles_of(uint32_t tokens) { return (tokens + kTile - 1u) / kTile; }

__device__ __forceinline__ uint32_t wave_scan(uint32_t v, uint32_t lane)  // inclusive
{
#pragma unroll
    for (uint32_t d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)v, d, 64);
        v += lane >= d ? o : 0u;
    }
    return v;
}

// Where the tiles of all requests go.  Every wave finds out for itself.
struct Deal {
    uint32_t total, per;  // tiles, and tiles of a range
    __device__ __forceinline__ Deal(const AttendParams &p, uint32_t lane)
    {
        uint32_t sum = 0;
        for (uint32_t base = 0; base < p.n_seqs; base += 64) {
            const uint32_t s = base + lane;
            sum += s < p.n_seqs ? tiles_of(seq_tokens(p.lens, s, p.max_tokens)) : 0u;
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) sum += (uint32_t)__shfl_xor((int)sum, d, 64);
        total = __builtin_amdgcn_readfirstlane(sum);
        per = max((total + p.groups - 1u) / p.groups, 1u);
        per = (per + p.subs - 1u) / p.subs * p.subs;
    }
};

// Tiles of the requests before `s`.
__device__ __forceinline__ uint32_t tiles_before(const AttendParams &p, uint32_t s, uint32_t lane)
{
    uint32_t sum = 0;
    for (uint32_t at = lane; at < s; at += 64) sum += tiles_of(seq_tokens(p.lens, at, p.max_tokens));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += (uint32_t)__shfl_xor((int)sum, d, 64);
    return __builtin_amdgcn_readfirstlane(sum);
}

template <typename X, bool FP8, int DP>
struct Tile {
    static constexpr int KJ = DP / 32;              // steps of 32 dimensions of q.k
    static constexpr int VW = DP == 64 ? 4 : 8;     // dimensions of a row that a lane loads at once,
    static constexpr int NV = DP == 64 ? 1 : DP / 128;  // and how often
    static constexpr int ACC = VW * NV;
};

template <int BYTES>
struct Raw;
template <>
struct Raw<16> { typedef w32x4 type; };
template <>
struct Raw<8> { typedef w32x2 type; };
template <>
struct Raw<4> { typedef uint32_t type; };

template <typename X, bool FP8, int DP>
__global__ __launch_bounds__(512) void kv_attend_kernel(const AttendParams p)
{
    using T = Tile<X, FP8, DP>;
    constexpr int KJ = T::KJ, VW = T::VW, NV = T::NV, ACC = T::ACC;
    typedef typename Raw<FP8 ? 8 : 16>::type kraw;
    typedef typename Raw<(FP8 ? 1 : 2) * VW>::type vraw;
    __shared__ float joined[4][ACC * 4][64];
    __shared__ f32x4 ml[8][16];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n = lane & 15u, kq = lane >> 4;
    const uint32_t group = blockIdx.x / p.wgs_per_group;
    const uint32_t unit = (blockIdx.x - group * p.wgs_per_group) * p.units_per_wg + wave % p.units_per_wg;
    const uint32_t sub = wave / p.units_per_wg;
    const bool active = unit < p.units;
    const Deal deal(p, lane);
    uint32_t at = group * deal.per;
    const uint32_t end = min(at + deal.per, deal.total);
    if (at >= end) return;
    // the request that tile `at` is one of, and which of its tiles
    uint32_t s = 0, t = 0;
    {
        uint32_t before = 0;
        for (uint32_t base = 0; base < p.n_seqs; base += 64) {
            const uint32_t mine = base + lane < p.n_seqs ? tiles_of(seq_tokens(p.lens, base + lane, p.max_tokens)) : 0u;
            const uint32_t upto = wave_scan(mine, lane);
            const uint64_t beyond = __ballot(before + upto > at);
            if (beyond) {
                const uint32_t first = (uint32_t)__builtin_ctzll(beyond);
                s = base + first;
                t = at - before - (uint32_t)__shfl((int)(upto - mine), (int)first, 64);
                break;
            }
            before += (uint32_t)__shfl((int)upto, 63, 64);
        }
        s = __builtin_amdgcn_readfirstlane(s);
        t = __builtin_amdgcn_readfirstlane(t);
    }
    const uint32_t kv_head = active ? unit / p.head_tiles : 0u, ht = active ? unit - kv_head * p.head_tiles : 0u;
    const uint32_t rows = min(16u, p.group_heads - ht * 16u);      // query heads of this wave
    const uint32_t head = kv_head * p.group_heads + ht * 16u + n;  // this lane's
    const bool has_row = active && n < rows;
    const uint8_t *const kb = p.k + (uint64_t)kv_head * p.head_bytes;
    const uint8_t *const vb = p.v + (uint64_t)kv_head * p.head_bytes;
    constexpr uint32_t elem = FP8 ? 1u : 2u;

    while (at < end && s < p.n_seqs) {
        const uint32_t tokens = seq_tokens(p.lens, s, p.max_tokens), n_tiles = tiles_of(tokens);
        if (n_tiles == 0) {
            s++;
            t = 0;
            continue;
        }
        const uint32_t here = min(n_tiles - t, end - at);
        const int32_t *const row = p.table + (int64_t)s * p.table_stride;
        w32x4 qf[KJ];
#pragma unroll
        for (int j = 0; j < KJ; j++) {
            const uint32_t d = (uint32_t)j * 32u + kq * 8u;
            qf[j] = w32x4{0u, 0u, 0u, 0u};
            if (has_row && d < p.dim)
                qf[j] = *reinterpret_cast<const w32x4 *>(p.q + (uint64_t)s * p.q_row + (uint64_t)head * p.q_head + d * 2u);
        }
        f32x4 acc[ACC], sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ACC; i++) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        float ref = -1e30f;  // finite, so that a score of -inf has weight 0 from the start
        float own = 0.f;     // this lane's part of the sum of weights as they are, before they are rounded

        // The row of the cache that token (half, n) of tile `tt` lies in.
        auto cell_of = [&](uint32_t tt, uint32_t half) {
            const uint32_t token = tt * kTile + half * 16u + n;
            uint32_t cell = kNoCell;
            if (token < tokens) {
                const uint32_t entry = token / p.block_size;
                const uint32_t id = (uint32_t)row[entry];
                if (id < p.n_blocks) cell = id * p.cells_per_block + (token - entry * p.block_size);
            }
            return cell;
        };
        for (uint32_t tt = t + sub; tt < t + here && active; tt += p.subs) {
            uint32_t cell[2];
            cell[0] = cell_of(tt, 0);
            cell[1] = cell_of(tt, 1);
            kraw kr[2][KJ];
            vraw vr[8][NV];
            uint32_t vcell[8];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uint64_t off = (uint64_t)(cell[h] == kNoCell ? 0u : cell[h]) * p.token_bytes;
#pragma unroll
                for (int j = 0; j < KJ; j++) {
                    const uint32_t d = (uint32_t)j * 32u + kq * 8u;
                    kr[h][j] = *reinterpret_cast<const kraw *>(kb + off + (d < p.dim ? d : 0u) * elem);
                }
            }
#pragma unroll
            for (int r = 0; r < 8; r++) {
                vcell[r] = (uint32_t)__shfl((int)cell[r / 4], (int)(kq * 4u + (r & 3)), 64);
                const uint64_t off = (uint64_t)(vcell[r] == kNoCell ? 0u : vcell[r]) * p.token_bytes;
#pragma unroll
                for (int c = 0; c < NV; c++) {
                    const uint32_t d = (uint32_t)c * 128u + n * VW;
                    vr[r][c] = *reinterpret_cast<const vraw *>(vb + off + (d < p.dim ? d : 0u) * elem);
                }
            }
            // scores: token x head
            f32x4 sc[2];
#pragma unroll
            for (int h = 0; h < 2; h++) {
                sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < KJ; j++) {
                    w32x4 a;
                    if constexpr (FP8) a = w32x4{X::template from_fp8<false>(kr[h][j].x), X::template from_fp8<true>(kr[h][j].x),
                                                 X::template from_fp8<false>(kr[h][j].y), X::template from_fp8<true>(kr[h][j].y)};
                    else a = kr[h][j];
                    // dimensions that are not there meet zeros of q: they must not be NaN
                    if ((uint32_t)j * 32u + 32u > p.dim && (uint32_t)j * 32u + kq * 8u >= p.dim) a = w32x4{0u, 0u, 0u, 0u};
                    sc[h] = X::mma(a, qf[j], sc[h]);
                }
            }
            float w[8], top = -__builtin_inff();
#pragma unroll
            for (int r = 0; r < 8; r++) {
                w[r] = vcell[r] == kNoCell ? -__builtin_inff() : sc[r / 4][r & 3] * p.qk_scale;
                top = fmaxf(top, w[r]);
            }
            if (__any(top > ref + X::kBias + X::kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float next = fmaxf(ref, top - X::kBias), shrink = __builtin_amdgcn_exp2f(ref - next);
                ref = next;
#pragma unroll
                for (int i = 0; i < ACC; i++) acc[i] *= shrink;
                sum *= shrink;
                own *= shrink;
            }
#pragma unroll
            for (int r = 0; r < 8; r++) {
                w[r] = __builtin_amdgcn_exp2f(w[r] - ref);
                own += w[r];
            }
            const w32x4 pw = {X::pack(w[0], w[1]), X::pack(w[2], w[3]), X::pack(w[4], w[5]), X::pack(w[6], w[7])};
            // out is divided by the sum of the weights that it is made of, the rounded ones (rows of
            // ones beside the values); lse and the blocks' weights go by the sum of those that they were.
            sum = X::mma(w32x4{X::kOnes, X::kOnes, X::kOnes, X::kOnes}, pw, sum);
#pragma unroll
            for (int c = 0; c < NV; c++) {
                uint32_t pair[8][VW / 2];  // of each token: dimensions 2i and 2i + 1
#pragma unroll
                for (int r = 0; r < 8; r++) {
#pragma unroll
                    for (int i = 0; i < VW / 2; i++) {
                        if constexpr (FP8 && VW == 8)
                            pair[r][i] = i & 1 ? X::template from_fp8<true>(vr[r][c][i / 2]) : X::template from_fp8<false>(vr[r][c][i / 2]);
                        else if constexpr (FP8)
                            pair[r][i] = i & 1 ? X::template from_fp8<true>(vr[r][c]) : X::template from_fp8<false>(vr[r][c]);
                        else
                            pair[r][i] = vr[r][c][i];
                        // a weight of 0 does not make up for NaN
                        if (vcell[r] == kNoCell) pair[r][i] = 0u;
                    }
                }
#pragma unroll
                for (int i = 0; i < VW / 2; i++) {
                    w32x4 even, odd;
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        even[k] = __builtin_amdgcn_perm(pair[2 * k + 1][i], pair[2 * k][i], 0x05040100u);
                        odd[k] = __builtin_amdgcn_perm(pair[2 * k + 1][i], pair[2 * k][i], 0x07060302u);
                    }
                    acc[c * VW + 2 * i] = X::mma(even, pw, acc[c * VW + 2 * i]);
                    acc[c * VW + 2 * i + 1] = X::mma(odd, pw, acc[c * VW + 2 * i + 1]);
                }
            }
            if (p.granules) {
                // weights of runs of `granule` tokens (1, 2, 4, 8 or 16: it divides a block and a half tile)
                float *const g = p.granules + (uint64_t)s * p.max_granules * p.n_heads;
                const uint32_t n_gran = (tokens + p.granule - 1u) / p.granule;
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const uint32_t first = tt * kTile + (uint32_t)h * 16u + kq * 4u;
                    auto put = [&](uint32_t token, float weight) {
                        const uint32_t i = token / p.granule;
                        if (has_row && i < n_gran) g[(uint64_t)i * p.n_heads + head] = ref + __builtin_amdgcn_logf(weight);
                    };
                    const float *x = w + 4 * h;
                    if (p.granule == 1u) {
                        for (uint32_t r = 0; r < 4; r++) put(first + r, x[r]);
                    } else if (p.granule == 2u) {
                        put(first, x[0] + x[1]);
                        put(first + 2u, x[2] + x[3]);
                    } else {
                        float y = (x[0] + x[1]) + (x[2] + x[3]);
                        if (p.granule >= 8u) y += __shfl_xor(y, 16, 64);
                        if (p.granule == 16u) y += __shfl_xor(y, 32, 64);
                        if ((kq * 4u) % p.granule == 0u) put(first, y);
                    }
                }
            }
        }
        own += __shfl_xor(own, 16, 64);
        own += __shfl_xor(own, 32, 64);
        // waves that took turns at the tiles join
        if (p.subs > 1u) {
            if (kq == 0) ml[wave][n] = f32x4{ref, sum[0], own, 0.f};
            __syncthreads();
            float top = -1e30f, all = 0.f, all_own = 0.f;
            for (uint32_t o = 0; o < p.subs; o++) top = fmaxf(top, ml[o * p.units_per_wg + wave % p.units_per_wg][n].x);
            for (uint32_t o = 0; o < p.subs; o++) {
                const f32x4 x = ml[o * p.units_per_wg + wave % p.units_per_wg][n];
                const float f = __builtin_amdgcn_exp2f(x.x - top);
                all += x.y * f;
                all_own += x.z * f;
            }
            const float shrink = __builtin_amdgcn_exp2f(ref - top);
            ref = top;
            sum[0] = all;
            own = all_own;
#pragma unroll
            for (int i = 0; i < ACC; i++) acc[i] *= shrink;
            for (uint32_t half = p.subs / 2u; half > 0; half >>= 1) {
                const uint32_t slot = wave - half * p.units_per_wg;
                if (sub >= half && sub < 2u * half) {
#pragma unroll
                    for (int i = 0; i < ACC * 4; i++) joined[slot][i][lane] = acc[i / 4][i & 3];
                }
                __syncthreads();
                if (sub < half) {
#pragma unroll
                    for (int i = 0; i < ACC * 4; i++) acc[i / 4][i & 3] += joined[wave][i][lane];
                }
                __syncthreads();
            }
        }
        if (has_row && sub == 0u) {
            const bool whole = here == n_tiles;
            const float total = sum[0];
            const uint32_t slot = group * 2u + (t > 0u ? 0u : 1u);
            const float inv = total == 0.f ? 0.f : p.v_scale / total;
            if (whole && kq == 0u) {
                const float l2 = own == 0.f ? -__builtin_inff() : ref + __builtin_amdgcn_logf(own);
                if (p.lse) p.lse[(uint64_t)s * p.n_heads + head] = l2 * 0.693147180559945309f;
                if (p.granules) p.lse2[(uint64_t)s * p.n_heads + head] = l2;
            }
            if (!whole && kq == 0u) p.part_ml[(uint64_t)slot * p.n_heads + head] = f32x4{ref, total, own, 0.f};
#pragma unroll
            for (int c = 0; c < NV; c++) {
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const uint32_t d = (uint32_t)c * 128u + (kq * 4u + (uint32_t)r) * VW;
                    if (d >= p.dim) continue;
                    if (whole) {
                        uint8_t *const to = p.out + (uint64_t)s * p.out_row + (uint64_t)head * p.out_head + d * 2u;
#pragma unroll
                        for (int i = 0; i < VW / 4; i++) {
                            const f32x4 *a = acc + c * VW + 4 * i;
                            *reinterpret_cast<w32x2 *>(to + 8 * i) =
                                w32x2{X::pack(a[0][r] * inv, a[1][r] * inv), X::pack(a[2][r] * inv, a[3][r] * inv)};
                        }
                    } else {
                        float *const to = p.part + ((uint64_t)slot * p.n_heads + head) * p.dim + d;
#pragma unroll
                        for (int i = 0; i < VW / 4; i++) {
                            const f32x4 *a = acc + c * VW + 4 * i;
                            *reinterpret_cast<f32x4 *>(to + 4 * i) = f32x4{a[0][r], a[1][r], a[2][r], a[3][r]};
                        }
                    }
                }
            }
        }
        at += here;
        t = 0;
        s++;
    }
}

// Joins what several ranges left of one request, a workgroup per request and query head:
// out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i.
template <typename X>
__global__ __launch_bounds__(256) void kv_join_kernel(const AttendParams p)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, head = blockIdx.x, s = blockIdx.y;
    const uint32_t n_tiles = tiles_of(seq_tokens(p.lens, s, p.max_tokens));
    const Deal deal(p, lane);
    const uint32_t first = tiles_before(p, s, lane);
    uint8_t *const to = p.out + (uint64_t)s * p.out_row + (uint64_t)head * p.out_head;
    const uint32_t g0 = first / deal.per, g1 = n_tiles ? (first + n_tiles - 1u) / deal.per : g0;
    if (n_tiles && g0 == g1) return;  // finished where it was computed
    __shared__ f32x4 part[4];
    __shared__ float rest[3][256];
    auto slot_of = [&](uint32_t g) { return (uint64_t)(g * 2u + (g == g0 ? 1u : 0u)) * p.n_heads + head; };
    float top = -1e30f, sum = 0.f, own = 0.f;
    if (n_tiles) {
        for (uint32_t g = g0 + threadIdx.x; g <= g1; g += 256) {
            const f32x4 x = p.part_ml[slot_of(g)];
            const float m = fmaxf(top, x.x), f = __builtin_amdgcn_exp2f(top - m), fx = __builtin_amdgcn_exp2f(x.x - m);
            sum = sum * f + x.y * fx;
            own = own * f + x.z * fx;
            top = m;
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const float m2 = __shfl_xor(top, d, 64), l2 = __shfl_xor(sum, d, 64), o2 = __shfl_xor(own, d, 64), m = fmaxf(top, m2);
        const float f = __builtin_amdgcn_exp2f(top - m), f2 = __builtin_amdgcn_exp2f(m2 - m);
        sum = sum * f + l2 * f2;
        own = own * f + o2 * f2;
        top = m;
    }
    if (lane == 0) part[wave] = f32x4{top, sum, own, 0.f};
    __syncthreads();
    top = fmaxf(fmaxf(part[0].x, part[1].x), fmaxf(part[2].x, part[3].x));
    sum = own = 0.f;
    for (int w = 0; w < 4; w++) {
        const float f = __builtin_amdgcn_exp2f(part[w].x - top);
        sum += part[w].y * f;
        own += part[w].z * f;
    }
    const float inv = sum == 0.f ? 0.f : p.v_scale / sum;
    if (threadIdx.x == 0) {
        const float l2 = own == 0.f ? -__builtin_inff() : top + __builtin_amdgcn_logf(own);
        if (p.lse) p.lse[(uint64_t)s * p.n_heads + head] = l2 * 0.693147180559945309f;
        if (p.granules) p.lse2[(uint64_t)s * p.n_heads + head] = l2;
    }
    // a lane has 4 dimensions, a wave every fourth range
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    const uint32_t d = lane * 4u;
    if (n_tiles && d < p.dim) {
#pragma unroll 4
        for (uint32_t g = g0 + wave; g <= g1; g += 4) {
            const uint64_t at = slot_of(g);
            const float f = __builtin_amdgcn_exp2f(p.part_ml[at].x - top);
            o += *reinterpret_cast<const f32x4 *>(p.part + at * p.dim + d) * f;
        }
    }
    if (wave > 0) *reinterpret_cast<f32x4 *>(&rest[wave - 1][d]) = o;
    __syncthreads();
    if (wave == 0 && d < p.dim) {
        for (int w = 0; w < 3; w++) o += *reinterpret_cast<const f32x4 *>(&rest[w][d]);
        o *= inv;
        *reinterpret_cast<w32x2 *>(to + d * 2u) = w32x2{X::pack(o[0], o[1]), X::pack(o[2], o[3])};
    }
}

// What each block received: 16 lanes a block add up 2^(granule - lse) over its granules and
// all query heads, in a fixed order.
static __global__ __launch_bounds__(256) void kv_mass_kernel(const AttendParams p)
{
    const uint32_t s = blockIdx.y, part = threadIdx.x & 15u, j = blockIdx.x * 16u + (threadIdx.x >> 4);
    const uint32_t tokens = seq_tokens(p.lens, s, p.max_tokens);
    const uint32_t per_block = p.block_size / p.granule, n_gran = (tokens + p.granule - 1u) / p.granule;
    const uint32_t g0 = min(j * per_block, n_gran), g1 = min(g0 + per_block, n_gran);
    const float *const g = p.granules + ((uint64_t)s * p.max_granules + g0) * p.n_heads;
    float sum = 0.f;
    for (uint32_t i = part, h = part % p.n_heads; i < (g1 - g0) * p.n_heads; i += 16u) {
        const float l2 = p.lse2[(uint64_t)s * p.n_heads + h];
        sum += l2 == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(g[i] - l2);
        h += 16u;
        while (h >= p.n_heads) h -= p.n_heads;
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if (part == 0u && j < p.max_blocks) {
        const int64_t at = (int64_t)s * p.mass_stride + j;
        p.mass_out[at] = (p.mass ? p.mass[at] : 0.f) + sum;
    }
}

// ---- new tokens into the cache ---------------------------------------------------------------
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
    float k_inv, v_inv;
};

// The nearest e4m3 values of four numbers.  The conversion has no bounds of its own: beyond 448
// it gives NaN.
__device__ __forceinline__ uint32_t to_fp8(float a, float b, float c, float d, float inv)
{
    auto bound = [inv](float x) {
        x *= inv;
        return x > 448.f ? 448.f : x < -448.f ? -448.f : x;  // NaN stays
    };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(bound(a), bound(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(bound(c), bound(d), w, true);
}

// A workgroup takes a row at a time: its angles into LDS, then q, k and v in steps of 4
// dimensions (two of them where the pairs' halves lie apart).
template <typename X, bool FP8>
__global__ __launch_bounds__(256) void kv_put_kernel(const PutParams p)
{
    __shared__ float2 turn[128];
    const uint32_t row = blockIdx.x, tid = threadIdx.x;
    // the request whose row this is
    uint32_t s = row, start = row, next = row + 1u;
    if (p.starts) {
        uint32_t lo = 0, hi = p.n_seqs;  // starts[lo] <= row, starts[hi] > row
        if (row >= (uint32_t)p.starts[p.n_seqs] || row < (uint32_t)p.starts[0]) return;
        while (hi - lo > 1u) {
            const uint32_t mid = (lo + hi) / 2u;
            if ((uint32_t)p.starts[mid] <= row) lo = mid;
            else hi = mid;
        }
        s = lo;
        start = (uint32_t)p.starts[s];
        next = (uint32_t)p.starts[s + 1u];
    }
    const int64_t cell_token = (int64_t)p.lens[s] - (int64_t)(next - start) + (int64_t)(row - start);
    bool page = cell_token >= 0 && cell_token < (int64_t)p.max_blocks * p.block_size;
    uint64_t cell = 0;
    if (page) {
        const uint32_t entry = (uint32_t)cell_token / p.block_size;
        const uint32_t id = (uint32_t)p.table[(int64_t)s * p.table_stride + entry];
        page = id < p.n_blocks;
        cell = (uint64_t)id * p.cells_per_block + ((uint32_t)cell_token - entry * p.block_size);
    }
    const uint32_t pairs = p.rot / 2u;
    for (uint32_t i = tid; i < pairs; i += 256u) {
        const uint32_t axis = i < p.section0 ? 0u : i < p.section01 ? 1u : 2u;
        const double pos = p.positions ? (double)p.positions[(int64_t)axis * p.position_stride + row] : (double)cell_token;
        // in 64 bits: half turns, and of those what is left of whole turns
        const double turns = pos * (double)p.inv_freq[i] * 0.15915494309189533577;
        const float half = 2.0f * (float)(turns - rint(turns));
        float sn, cs;
        sincospif(half, &sn, &cs);
        turn[i] = float2{cs, sn};
    }
    __syncthreads();
    const uint32_t v4 = p.dim / 4u, r4 = p.rot / 4u;
    const uint32_t apart = p.interleaved ? 0u : r4 / 2u;   // steps of the lower halves
    const uint32_t steps = v4 - apart;                     // steps of a rotated head
    const uint32_t n_q = p.qs ? p.n_heads * steps : 0u, n_k = p.n_kv_heads * steps, n_v = p.n_kv_heads * v4;
    uint8_t *const kc = p.k + cell * p.token_bytes, *const vc = p.v + cell * p.token_bytes;
    auto rotated = [&](uint32_t step, const uint8_t *src, auto &&store) {
        if (step < apart) {
            const uint32_t d = step * 4u, d2 = d + p.rot / 2u;
            const w32x2 a = *reinterpret_cast<const w32x2 *>(src + d * 2u), b = *reinterpret_cast<const w32x2 *>(src + d2 * 2u);
            const float x[4] = {X::lo(a.x), X::hi(a.x), X::lo(a.y), X::hi(a.y)};
            const float y[4] = {X::lo(b.x), X::hi(b.x), X::lo(b.y), X::hi(b.y)};
            float u[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float2 c = turn[d + i];
                u[i] = x[i] * c.x - y[i] * c.y;
                w[i] = y[i] * c.x + x[i] * c.y;
            }
            store(d, u);
            store(d2, w);
            return;
        }
        const uint32_t d = (step + apart) * 4u;
        const w32x2 a = *reinterpret_cast<const w32x2 *>(src + d * 2u);
        float x[4] = {X::lo(a.x), X::hi(a.x), X::lo(a.y), X::hi(a.y)};
        if (d < p.rot) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const float2 c = turn[(d + i) / 2u];
                const float u = x[i] * c.x - x[i + 1] * c.y, w = x[i + 1] * c.x + x[i] * c.y;
                x[i] = u;
                x[i + 1] = w;
            }
        }
        store(d, x);
    };
    auto into_cache = [&](uint8_t *to, float inv) {
        return [=](uint32_t d, const float(&x)[4]) {
            if constexpr (FP8) *reinterpret_cast<uint32_t *>(to + d) = to_fp8(x[0], x[1], x[2], x[3], inv);
            else *reinterpret_cast<w32x2 *>(to + d * 2u) = w32x2{X::pack(x[0], x[1]), X::pack(x[2], x[3])};
        };
    };
    for (uint32_t i = tid; i < n_q + n_k + n_v; i += 256u) {
        if (i < n_q) {
            const uint32_t h = i / steps, step = i - h * steps;
            uint8_t *const to = p.qd + row * p.qd_row + h * p.qd_head;
            rotated(step, p.qs + row * p.q_row + h * p.q_head, [=](uint32_t d, const float(&x)[4]) {
                *reinterpret_cast<w32x2 *>(to + d * 2u) = w32x2{X::pack(x[0], x[1]), X::pack(x[2], x[3])};
            });
        } else if (!page) {
            break;
        } else if (i < n_q + n_k) {
            const uint32_t h = (i - n_q) / steps, step = i - n_q - h * steps;
            rotated(step, p.ks + row * p.k_row + h * p.k_head, into_cache(kc + h * p.head_bytes, p.k_inv));
        } else {
            const uint32_t j = i - n_q - n_k, h = j / v4, d = (j - h * v4) * 4u;
            const w32x2 a = *reinterpret_cast<const w32x2 *>(p.vs + row * p.v_row + h * p.v_head + d * 2u);
            const float x[4] = {X::lo(a.x), X::hi(a.x), X::lo(a.y), X::hi(a.y)};
            into_cache(vc + h * p.head_bytes, p.v_inv)(d, x);
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

constexpr int kEvictThreads = 1024;

// Weights as whole numbers of the same order: lightest first, NaN last, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float x)
{
    if (x != x) return ~0u;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// One workgroup per request.  The key of the last block to go is found digit by digit (8 bits at a
// time, counted in LDS); then the row is closed up, 1024 entries at a time: what
// is read of a stretch is read before anything is written, and nothing is written behind what has
// been read, so a row may be its own output.
static __global__ __launch_bounds__(kEvictThreads) void kv_evict_kernel(const EvictParams p)
{
    const uint32_t s = blockIdx.x, tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    __shared__ uint32_t bins[256];
    __shared__ uint32_t chosen[2];
    __shared__ uint2 waves[kEvictThreads / 64];
    const uint32_t tokens = seq_tokens(p.lens, s, p.max_blocks * p.block_size);
    const uint32_t held = (tokens + p.block_size - 1u) / p.block_size;
    const int32_t *const table = p.table + (int64_t)s * p.table_stride;
    const float *const mass = p.mass + (int64_t)s * p.mass_stride;
    int32_t *const table_out = p.table_out + (int64_t)s * p.table_stride;
    float *const mass_out = p.mass_out + (int64_t)s * p.mass_stride;
    int32_t *const ids = p.ids + (int64_t)s * p.max_evict, *const ats = p.at + (int64_t)s * p.max_evict;
    const uint32_t from = min(p.n_first, held), to = held > p.n_last ? max(held - p.n_last, from) : from;  // may go
    const uint32_t go = min(min(held > p.budget ? held - p.budget : 0u, to - from), p.max_evict);
    // key of the go-th lightest, and how many of that key go
    uint32_t prefix = 0, left = go;
    for (int shift = 24; shift >= 0 && go; shift -= 8) {
        if (tid < 256u) bins[tid] = 0u;
        __syncthreads();
        for (uint32_t j = from + tid; j < to; j += kEvictThreads) {
            const uint32_t key = weight_key(mass[j]);
            if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[key >> shift & 255u], 1u);
        }
        __syncthreads();
        if (wave == 0) {
            uint32_t mine[4], sum = 0;
            for (int i = 0; i < 4; i++) sum += mine[i] = bins[lane * 4u + i];
            uint32_t before = wave_scan(sum, lane) - sum;
            for (int i = 0; i < 4; i++) {
                if (before < left && left <= before + mine[i]) {
                    chosen[0] = lane * 4u + i;
                    chosen[1] = left - before;
                }
                before += mine[i];
            }
        }
        __syncthreads();
        prefix |= chosen[0] << shift;
        left = chosen[1];
    }
    uint32_t gone = 0, ties = 0;  // in the stretches before
    for (uint32_t base = 0; base < held; base += kEvictThreads) {
        const uint32_t j = base + tid;
        int32_t id = -1;
        float m = 0.f;
        uint32_t key = 0;
        bool less = false, tie = false;
        if (j < held) {
            id = table[j];
            m = mass[j];
            key = weight_key(m);
            const bool may = go && j >= from && j < to;
            less = may && key < prefix;
            tie = may && key == prefix;
        }
        const uint64_t below = (1ull << lane) - 1u, bl = __ballot(less), bt = __ballot(tie);
        if (lane == 0) waves[wave] = uint2{(uint32_t)__popcll(bl), (uint32_t)__popcll(bt)};
        __syncthreads();
        uint32_t less_before = 0, tie_before = ties, less_all = 0, tie_all = 0;
        for (uint32_t w = 0; w < kEvictThreads / 64; w++) {
            const uint2 x = waves[w];
            less_before += w < wave ? x.x : 0u;
            tie_before += w < wave ? x.y : 0u;
            less_all += x.x;
            tie_all += x.y;
        }
        less_before += (uint32_t)__popcll(bl & below);
        tie_before += (uint32_t)__popcll(bt & below);
        const bool goes = less || (tie && tie_before < left);
        // those that went before j: the lighter ones, and of the ties the first `left`
        const uint32_t left_before = gone + less_before + (min(tie_before, left) - min(ties, left));
        if (j < held) {
            if (goes) {
                ids[left_before] = id;
                ats[left_before] = (int32_t)j;
            } else {
                table_out[j - left_before] = id;
                mass_out[j - left_before] = m;
            }
        }
        gone += less_all + (min(ties + tie_all, left) - min(ties, left));
        ties += tie_all;
        __syncthreads();  // the next stretch's counts, and reads of rows that are their own output
    }
    for (uint32_t j = held - go + tid; j < p.max_blocks; j += kEvictThreads) {
        table_out[j] = -1;
        mass_out[j] = 0.f;
    }
    for (uint32_t j = go + tid; j < p.max_evict; j += kEvictThreads) ids[j] = ats[j] = -1;
    if (tid == 0) {
        p.count[s] = (int32_t)go;
        p.lens_out[s] = (int32_t)(tokens - go * p.block_size);
    }
}

}  // namespace dkv
