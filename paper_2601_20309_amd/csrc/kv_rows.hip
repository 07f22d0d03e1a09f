// Host side of attention of many rows per request (see include/duplexkv.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kv_rows.hpp"
#include "kv_rows_kernels.hpp"

namespace {

template <typename X, int KIND>
void launch_rows(dim3 g, hipStream_t s, const dkv::RowsParams &p)
{
    auto launch = [&](auto dims, auto rows) {
        constexpr int DP = decltype(dims)::value, ROWS = decltype(rows)::value;
        using T = dkv::RowStep<DP, ROWS>;
        hipLaunchKernelGGL((dkv::kv_rows_kernel<X, KIND, DP, ROWS>), g, dim3(64 * T::WAVES), 0, s, p);
        const uint64_t joins = (uint64_t)p.n_tiles * p.n_kv_heads * (ROWS / 32) * (DP / 32);
        const auto join = [&](auto wide) {
            constexpr bool WIDE = decltype(wide)::value;
            hipLaunchKernelGGL((dkv::kv_rows_join_kernel<X, KIND == dkv::kBits16, WIDE>), dim3((uint32_t)(WIDE ? joins : (joins + 3) / 4)), dim3(256), 0, s, p,
                               (uint32_t)DP / 32u, (uint32_t)T::TOKENS);
        };
        if (p.groups || p.splits > 8u) join(std::true_type{});
        else if (p.splits > 1u) join(std::false_type{});
    };
    auto go = [&](auto dims) {
        if (p.row_bits == 5u) return launch(dims, std::integral_constant<int, 32>{});
        if constexpr (decltype(dims)::value <= dkv::kManyRowsDims)
            if (p.row_bits == 8u) return launch(dims, std::integral_constant<int, 256>{});
        launch(dims, std::integral_constant<int, 128>{});
    };
    switch (dkv::rows_dims(p.dim)) {
    case 64: go(std::integral_constant<int, 64>{}); break;
    case 96: go(std::integral_constant<int, 96>{}); break;
    case 128: go(std::integral_constant<int, 128>{}); break;
    case 192: go(std::integral_constant<int, 192>{}); break;
    default: go(std::integral_constant<int, 256>{}); break;
    }
}

}  // namespace

extern "C" int kv_attend_rows(kv_decoder *d, const kv_attend_rows_args *a, void *stream)
{
    using namespace dkv;
    if (!d || !a || a->layer < 0 || a->layer >= d->cfg.n_layers || a->n_seqs < 0 || a->n_rows < 0) return KV_EINVAL;
    const float qk_scale = (float)((double)a->scale * 1.4426950408889634074 * (double)d->dc.k_scale);
    if (!std::isfinite(qk_scale)) return KV_EINVAL;
    if (a->n_seqs > d->dc.max_seqs || a->n_rows > d->dc.max_rows) return KV_E2BIG;
    const bool rows_here = a->n_seqs > 0 && a->n_rows > 0;
    if (!a->starts && a->n_rows != a->n_seqs) return KV_EINVAL;
    if (rows_here && (!a->table || !a->lens || !a->q.data || !a->out.data)) return KV_EINVAL;
    if (a->n_seqs > 1 && a->table_stride < d->dc.max_blocks) return KV_EINVAL;
    if (!rows_ok(a->q) || !rows_ok(a->out)) return KV_EINVAL;
    if (!rows_aligned(a->q) || !rows_aligned(a->out)) return KV_EUNSUP;
    if (a->out.data && !apart(a->out, a->n_rows, d->dc.n_heads, d->dim)) return KV_EINVAL;
    if (!rows_here) return KV_OK;
    OnDevice on(d->device);
    if (!on.ok()) return KV_EHIP;
    RowsParams p{};
    p.k = plane(d, a->layer, 0);
    p.v = plane(d, a->layer, 1);
    p.table = a->table;
    p.lens = a->lens;
    p.starts = a->starts;
    p.q = (const uint8_t *)a->q.data;
    p.out = (uint8_t *)const_cast<void *>(a->out.data);
    p.lse = a->lse;
    p.zeros = d->rows_zeros;
    p.part = d->rows_part;
    p.part_ml = d->rows_ml;
    p.q_row = 2ull * (uint64_t)a->q.row;
    p.q_head = 2ull * (uint64_t)a->q.head;
    p.out_row = 2ull * (uint64_t)a->out.row;
    p.out_head = 2ull * (uint64_t)a->out.head;
    p.table_stride = a->table_stride;
    p.n_seqs = (uint32_t)a->n_seqs;
    p.n_rows = (uint32_t)a->n_rows;
    p.n_heads = (uint32_t)d->dc.n_heads;
    p.n_kv_heads = (uint32_t)d->cfg.n_kv_heads;
    p.max_tokens = (uint32_t)d->dc.max_blocks * (uint32_t)d->cfg.block_size;
    p.dim = (uint32_t)d->dim;
    p.token_bytes = d->token_bytes;
    p.head_bytes = d->head_bytes;
    p.exponents = d->exponents;
    p.block_size = (uint32_t)d->cfg.block_size;
    p.cells_per_block = d->cells_per_block;
    p.n_blocks = (uint32_t)d->cfg.n_hbm_blocks;
    p.group_heads = p.n_heads / p.n_kv_heads;
    p.causal = a->causal ? 1u : 0u;
    p.by_block = Divide::by(p.block_size);
    p.by_group = Divide::by(p.group_heads);
    p.negative = qk_scale < 0.f ? 1u : 0u;
    p.qk_scale = std::max(std::fabs(qk_scale), 0x1p-126f);  // (0 times the score of what is masked, -inf, is NaN)
    p.v_scale = d->dc.v_scale;
    p.bias = bf16_bias(p.max_tokens);
    const int kind = (d->dc.x_type == KV_FP16 ? 1 : 0) + (d->dc.kv_type == KV_FP8 ? 2 : d->dc.kv_type == KV_FP4 ? 4 : 0);
    // Few rows to a request: 32 to a tile.  Many, and enough tiles for all compute units: 256, so that half as many bytes
    // go into LDS.  us, 128 rows / 256: 4 prompts of 2048 tokens, 32 heads over 8 of 128, 190 / 178; 1024 tokens at 31000, 64
    // over 8, 1124 / 990; 24 requests of 180 rows of 12 heads of 64 43.9 / 50.4.
    const uint64_t mean = (uint64_t)p.n_rows * p.group_heads / p.n_seqs;
    const bool few = mean <= 48u && row_tiles(p.n_rows, p.group_heads, p.n_seqs, 5) * p.n_kv_heads <= kMostTiles;
    const bool many = mean >= 1024u && p.dim <= (uint32_t)kManyRowsDims && row_tiles(p.n_rows, p.group_heads, 0, 8) * p.n_kv_heads >= (uint64_t)d->n_cus &&
                      row_tiles(p.n_rows, p.group_heads, p.n_seqs, 8) * p.n_kv_heads <= kMostTiles / 2;
    p.row_bits = few ? 5u : many ? 8u : 7u;
    p.n_tiles = (uint32_t)row_tiles(p.n_rows, p.group_heads, p.n_seqs, (int)p.row_bits);
    const uint64_t each = (uint64_t)p.n_tiles * p.n_kv_heads;
    const uint32_t tokens = p.dim > 128u || few ? 32u : 64u, most = (p.max_tokens + tokens - 1u) / tokens;
    p.splits = 1u;
    p.least = 2u;
    uint64_t wgs = each;
    if (few) {
        // Equal ranges for two workgroups a compute unit (one where their tiles fill its LDS); a workgroup for each tile where no
        // request can be longer than four steps of its waves.  A range is two steps at least, so that one long request leaves no
        // more parts than can be joined in a few rounds (us, 3 rows of 4 heads of 96 over 15900 tokens in 4 bits, by one tile / 4 /
        // 8 / 16: 183 / 18.4 / 16.1 / 17.0).
        const uint32_t at_once = (uint32_t)d->n_cus * (kind < 2 && p.dim > 64u ? 1u : 2u);
        if (most > 16u && (uint64_t)p.n_tiles * most <= 0x7FFFFFFFu && each * (rows_dims(p.dim) / 32u) <= kMostTiles) {
            p.least = 8u;
            p.groups = (uint32_t)std::min<uint64_t>(std::max(1u, at_once / p.n_kv_heads), (uint64_t)p.n_tiles * most);
            wgs = (uint64_t)p.groups * p.n_kv_heads;
        }
    } else {
        // Few tiles of rows: the tokens are split, so that every compute unit has two workgroups, or one of 256 rows.  (More
        // splits leave more to join.  us, two / four / six to a compute unit: 24 requests of 180 rows, 12 heads of 64, 42.3 / 42.2 / 48.9;
        // 9 requests of 150 rows, 3 heads of 96 in 4 bits, 25.9 / 28.3 / 29.2.)
        const uint64_t wanted = (uint64_t)d->n_cus * (many ? 1u : 2u);
        p.splits = (uint32_t)std::max<uint64_t>(1u, std::min<uint64_t>(wanted / each, (most + p.least - 1u) / p.least));
        wgs = each * p.splits;
    }
    const dim3 g((uint32_t)wgs);
    hipStream_t s = (hipStream_t)stream;
    switch (kind) {
    case 0: launch_rows<Bf16, kBits16>(g, s, p); break;
    case 1: launch_rows<Fp16, kBits16>(g, s, p); break;
    case 2: launch_rows<Bf16, kBits8>(g, s, p); break;
    case 3: launch_rows<Fp16, kBits8>(g, s, p); break;
    case 4: launch_rows<Bf16, kBits4>(g, s, p); break;
    default: launch_rows<Fp16, kBits4>(g, s, p); break;
    }
    DECTRY(hipGetLastError());
    return KV_OK;
}
