// Host side of the decode step's operators (see include/duplexkv.h): checks,
// launch shapes, and the handle that holds their device memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <new>
#include <numeric>
#include <type_traits>

#include "kv_decoder.hpp"
#include "kv_rows.hpp"

using dkv::OnDevice, dkv::apart, dkv::plane, dkv::rows_aligned, dkv::rows_ok;

namespace {

constexpr uint32_t kFewRequests = 16;
constexpr int32_t kMostRows = 0xFFFFFF;  // of a kv_put: as many workgroups of 256 lanes as a launch can count lanes
// Workgroups that join, over all requests.  us of the joins, with 512 / 1024 / 2048: 32 requests around 1024 tokens 7.0 /
// 6.4 / 6.3, 128 around 500 9.2 / 8.1 / 9.2.
constexpr uint32_t kJoinWgs = 1024;

// How units and waves make up workgroups: up to `most` units each, evenly, and as many waves per unit as then fit.
struct Workgroup {
    uint32_t per_range, units, subs;  // workgroups of a range, units of one, waves of a unit
    Workgroup(uint32_t all, uint32_t most, uint32_t waves)
        : per_range((all + most - 1) / most), units((all + per_range - 1) / per_range), subs(1)
    {
        while (2 * subs * units <= waves) subs *= 2;
    }
};

// ranges: a workgroup per compute unit
uint32_t ranges(const kv_decoder *d, const Workgroup &w)
{
    return std::max(1u, std::min(dkv::kMaxGroups, (uint32_t)d->n_cus / w.per_range));
}

int kinds(const kv_decoder *d, int &dp)
{
    dp = d->dim <= 64 ? 64 : d->dim <= 128 ? 128 : 256;
    return (d->dc.x_type == KV_FP16 ? 1 : 0) + (d->dc.kv_type == KV_FP8 ? 2 : d->dc.kv_type == KV_FP4 ? 4 : 0);
}

template <typename X, bool FP8>
void launch_put(bool eights, uint32_t threads, hipStream_t s, const dkv::PutParams &p)
{
    if (eights) hipLaunchKernelGGL((dkv::kv_put_kernel<X, FP8, 8>), dim3(p.n_rows), dim3(threads), 0, s, p);
    else hipLaunchKernelGGL((dkv::kv_put_kernel<X, FP8, 4>), dim3(p.n_rows), dim3(threads), 0, s, p);
}

// Normed heads, or 4 bits.
template <typename X, int KIND>
void launch_put_heads(hipStream_t s, const dkv::PutParams &p)
{
    uint32_t bits = 0;
    while ((8u << bits) < p.dim) bits++;
    const uint32_t heads = (p.qs ? p.n_heads : 0u) + 2u * p.n_kv_heads;
    // us of 768 lanes a row, by 128 / 256 / 512: 64 rows 7.1 / 5.5 / 4.8, 6853 into 4 bits 40.2 / 43.0 / 52.6.
    const uint32_t most = p.n_rows <= 1024u ? 512u : 128u, lanes = heads << bits, turns = (lanes + most - 1u) / most;
    const uint32_t threads = ((lanes + turns - 1u) / turns + 63u) / 64u * 64u;
    const auto go = [&](auto whole) {
        hipLaunchKernelGGL((dkv::kv_put_heads_kernel<X, KIND, decltype(whole)::value>), dim3(p.n_rows), dim3(threads), 0, s, p, bits);
    };
    const uint32_t whole = p.rot == p.dim && !p.interleaved ? p.dim / 8u : 0u;
    if (whole == 8u) go(std::integral_constant<int, 8>{});
    else if (whole == 16u) go(std::integral_constant<int, 16>{});
    else if (whole == 32u) go(std::integral_constant<int, 32>{});
    else go(std::integral_constant<int, 0>{});
}

template <typename X, int KIND>
void launch_attend(int dp, dim3 g, dim3 b, hipStream_t s, const dkv::AttendParams &p)
{
    auto go = [&](auto dims) {
        constexpr int DP = decltype(dims)::value;
        if ((int)p.dim == DP) hipLaunchKernelGGL((dkv::kv_attend_kernel<X, KIND, DP, true>), g, b, 0, s, p);
        else hipLaunchKernelGGL((dkv::kv_attend_kernel<X, KIND, DP, false>), g, b, 0, s, p);
    };
    if (dp == 64) go(std::integral_constant<int, 64>{});
    else if (dp == 128) go(std::integral_constant<int, 128>{});
    else go(std::integral_constant<int, 256>{});
}

}  // namespace

extern "C" {

int kv_decoder_create(kv_decoder **out, const kv_config *cfg, const kv_decoder_config *dc, void *hbm_cache)
{
    if (!out) return KV_EINVAL;
    *out = nullptr;
    const uint64_t cache_bytes = cfg ? kv_cache_bytes(cfg) : 0;
    if (!cache_bytes || !dc || !hbm_cache) return KV_EINVAL;
    if (dc->n_heads <= 0 || dc->n_heads % cfg->n_kv_heads != 0 || dc->max_seqs <= 0 || dc->max_blocks <= 0) return KV_EINVAL;
    if (dc->x_type != KV_BF16 && dc->x_type != KV_FP16) return KV_EINVAL;
    if (dc->kv_type == KV_FP8 || dc->kv_type == KV_FP4 ? cfg->elem_bytes != 1 : dc->kv_type != dc->x_type || cfg->elem_bytes != 2)
        return KV_EINVAL;
    // 4 bits: 17 bytes of a row are 32 dimensions
    const bool fp4 = dc->kv_type == KV_FP4;
    if (fp4 && cfg->head_dim % 17 != 0) return KV_EINVAL;
    const int64_t dim = fp4 ? (int64_t)cfg->head_dim / 17 * 32 : cfg->head_dim;
    if (dc->max_rows < 0) return KV_EINVAL;
    for (float scale : {dc->k_scale, dc->v_scale})
        if (!(scale > 0.f) || !std::isfinite(scale) || !std::isfinite(1.f / scale) || (dc->kv_type != KV_FP8 && scale != 1.f))
            return KV_EINVAL;
    if (dim > 256 || dim % 8 != 0 || dc->n_heads > 1024 || (uintptr_t)hbm_cache % 16 != 0) return KV_EUNSUP;
    // tokens of a request, tiles of a call and the requests of a launch are counted in 31, 31 and 16 bits
    const int64_t tokens = (int64_t)dc->max_blocks * cfg->block_size;
    if (tokens > 0x7FFFFFC0 || dc->max_seqs > 65535 || (tokens / dkv::kTile + 1) * dc->max_seqs > 0x7FFFFFFF) return KV_EUNSUP;
    const uint64_t token_bytes = (uint64_t)cfg->n_kv_heads * (uint64_t)cfg->head_dim * (uint64_t)cfg->elem_bytes;
    const uint64_t cells = (uint64_t)cfg->block_size * (cfg->hbm_layout == KV_HBM_BLOCK_FIRST ? 2ull * cfg->n_layers : 1ull);
    // granules of a block, over all query heads, are counted in 31 bits, and the lanes that add them up in 32
    if (dc->weigh && ((uint64_t)cfg->block_size * (uint64_t)dc->n_heads > 0x7FFFFFFFull || dc->max_blocks > (1 << 28))) return KV_EUNSUP;
    if (token_bytes >> 31 || cells >> 31 || cells * (uint64_t)cfg->n_hbm_blocks >= 0xFFFFFFFFull) return KV_EUNSUP;
    if (!dkv::rows_fit(cfg->n_kv_heads, dc->n_heads, dc->max_seqs, dc->max_rows)) return KV_EUNSUP;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || ndev <= 0) {
        (void)hipGetLastError();
        fprintf(stderr, "duplexkv: no HIP device is visible\n");
        return KV_EHIP;
    }
    hipPointerAttribute_t at;
    hipDeviceptr_t base = nullptr;
    size_t span = 0;
    if (hipPointerGetAttributes(&at, hbm_cache) != hipSuccess || at.type != hipMemoryTypeDevice ||
        hipMemGetAddressRange(&base, &span, (hipDeviceptr_t)hbm_cache) != hipSuccess ||
        (uintptr_t)hbm_cache + cache_bytes > (uintptr_t)base + span) {
        (void)hipGetLastError();
        fprintf(stderr, "duplexkv: hbm_cache is not a device allocation of the configured size\n");
        return KV_EINVAL;
    }
    kv_decoder *d = new (std::nothrow) kv_decoder;
    if (!d) return KV_ENOMEM;
    d->cfg = *cfg;
    d->dc = *dc;
    d->device = at.device;
    d->hbm = (uint8_t *)hbm_cache;
    d->dim = (int32_t)dim;
    d->head_bytes = fp4 ? (uint32_t)dim / 2u : (uint32_t)(dim * cfg->elem_bytes);
    d->exponents = fp4 ? (uint32_t)cfg->n_kv_heads * d->head_bytes : 0u;
    d->token_bytes = (uint32_t)token_bytes;
    d->cells_per_block = (uint32_t)cells;
    d->plane_bytes = kv_seg_bytes(cfg) * (cfg->hbm_layout == KV_HBM_BLOCK_FIRST ? 1ull : (uint64_t)cfg->n_hbm_blocks);
    const uint32_t group = (uint32_t)(dc->n_heads / cfg->n_kv_heads);
    d->waves = dim <= 64 ? dkv::Step<64>::WAVES : dim <= 128 ? dkv::Step<128>::WAVES : dkv::Step<256>::WAVES;
    d->head_tiles = (group + 15) / 16;
    d->units = (uint32_t)cfg->n_kv_heads * d->head_tiles;
    d->part_rows = std::min(group, 16u);
    d->part_vecs = (dim <= 64 ? 4u : dim <= 128 ? 8u : 16u) * 4u * d->part_rows;
    d->granule = cfg->block_size % 4 ? 1u : std::gcd((uint32_t)cfg->block_size, 16u);
    d->max_granules = (uint32_t)dc->max_blocks * ((uint32_t)cfg->block_size / d->granule);
    OnDevice on(d->device);
    auto fail = [&](int code) {
        delete d;
        return code;
    };
    if (!on.ok() || hipDeviceGetAttribute(&d->n_cus, hipDeviceAttributeMultiprocessorCount, d->device) != hipSuccess)
        return fail(KV_EHIP);
    // ranges: a workgroup per compute unit, no more than there can be turns
    const uint64_t most_tiles = (uint64_t)dc->max_seqs * (((uint64_t)dc->max_blocks * cfg->block_size + dkv::kTile - 1) / dkv::kTile);
    d->max_groups = (uint32_t)std::min<uint64_t>(ranges(d, Workgroup(d->units, d->waves, d->waves)), most_tiles);
    const uint64_t slots = 2ull * d->max_groups;
    const uint64_t n_part = slots * d->units * d->part_vecs * sizeof(dkv::f32x4), n_ml = slots * (uint64_t)dc->n_heads * sizeof(dkv::f32x4),
                   n_lse = ((uint64_t)dc->max_seqs * (uint64_t)dc->n_heads * 4 + 255) / 256 * 256,
                   n_gran = dc->weigh ? (uint64_t)dc->max_seqs * d->max_granules * (uint64_t)dc->n_heads * 4 : 0;
    const uint64_t n_rows_part = dkv::rows_part_bytes(d), n_rows_ml = dkv::rows_ml_bytes(d), n_gran16 = (n_gran + 15) / 16 * 16;
    uint8_t *mem = nullptr;
    if (hipMalloc((void **)&mem, n_part + n_ml + n_lse + n_gran16 + n_rows_part + n_rows_ml + 16) != hipSuccess) {
        (void)hipGetLastError();
        return fail(KV_ENOMEM);
    }
    d->part = (dkv::f32x4 *)mem;
    d->part_ml = (dkv::f32x4 *)(mem + n_part);
    d->lse2 = (float *)(mem + n_part + n_ml);
    d->granules = (float *)(mem + n_part + n_ml + n_lse);
    d->rows_part = (dkv::f32x4 *)(mem + n_part + n_ml + n_lse + n_gran16);
    d->rows_ml = (float2 *)(mem + n_part + n_ml + n_lse + n_gran16 + n_rows_part);
    d->rows_zeros = mem + n_part + n_ml + n_lse + n_gran16 + n_rows_part + n_rows_ml;
    if (dc->max_rows && (hipMemset(d->rows_zeros, 0, 16) != hipSuccess || hipDeviceSynchronize() != hipSuccess)) {
        (void)hipFree(mem);
        return fail(KV_EHIP);
    }
    *out = d;
    return KV_OK;
}

int kv_decoder_destroy(kv_decoder *d)
{
    if (!d) return KV_EINVAL;
    OnDevice on(d->device);
    (void)hipDeviceSynchronize();
    (void)hipFree(d->part);
    delete d;
    return KV_OK;
}

int kv_put(kv_decoder *d, const kv_put_args *a, void *stream)
{
    if (!d || !a || a->layer < 0 || a->layer >= d->cfg.n_layers || a->n_seqs < 0 || a->n_rows < 0) return KV_EINVAL;
    if (a->n_seqs > d->dc.max_seqs) return KV_E2BIG;
    const bool rows_here = a->n_seqs > 0 && a->n_rows > 0;
    if (!a->starts && a->n_rows != a->n_seqs) return KV_EINVAL;
    if (rows_here && (!a->table || !a->lens || !a->k.data || !a->v.data)) return KV_EINVAL;
    if (a->table_stride < d->dc.max_blocks && a->n_seqs > 1) return KV_EINVAL;
    if (!rows_ok(a->k) || !rows_ok(a->v) || !rows_ok(a->q) || !rows_ok(a->q_out)) return KV_EINVAL;
    if ((a->q.data == nullptr) != (a->q_out.data == nullptr)) return KV_EINVAL;
    int32_t pairs = 0;
    if (a->inv_freq) {
        if (a->rot_dim <= 0 || a->rot_dim > d->dim || a->n_axes < 1 || a->n_axes > 3) return KV_EINVAL;
        if (!a->positions && a->n_axes != 1) return KV_EINVAL;
        for (int i = 0; i < a->n_axes; i++) {
            if (a->sections[i] < 0 || a->sections[i] > a->rot_dim) return KV_EINVAL;
            pairs += a->sections[i];
        }
        if (2 * pairs != a->rot_dim) return KV_EINVAL;
        if (a->positions && a->n_axes > 1 && a->position_stride != 0 && a->position_stride < a->n_rows) return KV_EINVAL;
        if (a->rot_dim % 8 != 0) return KV_EUNSUP;
    }
    if ((a->q_norm || a->k_norm) && !(a->norm_eps >= 0.f && std::isfinite(a->norm_eps))) return KV_EINVAL;
    if (a->q_norm && !a->q.data) return KV_EINVAL;
    if ((uintptr_t)a->q_norm % 16 != 0 || (uintptr_t)a->k_norm % 16 != 0) return KV_EUNSUP;
    if (!rows_aligned(a->k) || !rows_aligned(a->v) || !rows_aligned(a->q) || !rows_aligned(a->q_out)) return KV_EUNSUP;
    if (a->q_out.data && !apart(a->q_out, a->n_rows, d->dc.n_heads, d->dim)) return KV_EINVAL;
    if (a->n_rows > kMostRows) return KV_EUNSUP;
    if (!rows_here) return KV_OK;
    OnDevice on(d->device);
    if (!on.ok()) return KV_EHIP;
    dkv::PutParams p{};
    p.k = plane(d, a->layer, 0);
    p.v = plane(d, a->layer, 1);
    p.table = a->table;
    p.lens = a->lens;
    p.starts = a->starts;
    p.ks = (const uint8_t *)a->k.data;
    p.vs = (const uint8_t *)a->v.data;
    p.qs = (const uint8_t *)a->q.data;
    p.qd = (uint8_t *)const_cast<void *>(a->q_out.data);
    p.inv_freq = a->inv_freq;
    p.positions = a->positions;
    p.k_row = 2ull * (uint64_t)a->k.row;
    p.k_head = 2ull * (uint64_t)a->k.head;
    p.v_row = 2ull * (uint64_t)a->v.row;
    p.v_head = 2ull * (uint64_t)a->v.head;
    p.q_row = 2ull * (uint64_t)a->q.row;
    p.q_head = 2ull * (uint64_t)a->q.head;
    p.qd_row = 2ull * (uint64_t)a->q_out.row;
    p.qd_head = 2ull * (uint64_t)a->q_out.head;
    p.table_stride = a->table_stride;
    p.position_stride = a->position_stride;
    p.n_seqs = (uint32_t)a->n_seqs;
    p.n_rows = (uint32_t)a->n_rows;
    p.n_heads = (uint32_t)d->dc.n_heads;
    p.n_kv_heads = (uint32_t)d->cfg.n_kv_heads;
    p.max_blocks = (uint32_t)d->dc.max_blocks;
    p.dim = (uint32_t)d->dim;
    p.token_bytes = d->token_bytes;
    p.head_bytes = d->head_bytes;
    p.exponents = d->exponents;
    p.block_size = (uint32_t)d->cfg.block_size;
    p.cells_per_block = d->cells_per_block;
    p.n_blocks = (uint32_t)d->cfg.n_hbm_blocks;
    p.rot = a->inv_freq ? (uint32_t)a->rot_dim : 0u;
    p.interleaved = a->interleaved ? 1u : 0u;
    p.section0 = a->inv_freq ? (uint32_t)a->sections[0] : 0u;
    p.section01 = p.section0 + (a->inv_freq && a->n_axes > 1 ? (uint32_t)a->sections[1] : 0u);
    p.q_norm = a->q_norm;
    p.k_norm = a->k_norm;
    p.eps = a->norm_eps;
    p.inv_dim = 1.0f / (float)d->dim;
    p.k_scale = dkv::Scale::of(d->dc.k_scale);
    p.v_scale = dkv::Scale::of(d->dc.v_scale);
    hipStream_t s = (hipStream_t)stream;
    int dp;
    const int kind = kinds(d, dp);
    if (a->q_norm || a->k_norm || kind >= 4) {
        switch (kind) {
        case 0: launch_put_heads<dkv::Bf16, dkv::kBits16>(s, p); break;
        case 1: launch_put_heads<dkv::Fp16, dkv::kBits16>(s, p); break;
        case 2: launch_put_heads<dkv::Bf16, dkv::kBits8>(s, p); break;
        case 3: launch_put_heads<dkv::Fp16, dkv::kBits8>(s, p); break;
        case 4: launch_put_heads<dkv::Bf16, dkv::kBits4>(s, p); break;
        default: launch_put_heads<dkv::Fp16, dkv::kBits4>(s, p); break;
        }
        DECTRY(hipGetLastError());
        return KV_OK;
    }
    // 8 dimensions a step, or 4 where the halves of pairs are no multiple of 8 apart
    const bool eights = p.interleaved || p.rot % 16u == 0;
    const uint32_t n = eights ? 8u : 4u;
    p.by_vecs = dkv::Divide::by(p.dim / n);
    const uint32_t steps = p.dim / n - (p.interleaved ? 0u : p.rot / (2u * n));
    p.by_steps = dkv::Divide::by(steps);
    // Few rows: a thread for each place of a row, up to 512.  More rows than the chip has room for at
    // once: workgroups of up to 256, so that more of them are under way, and of equal turns.  us, 448 places a
    // row, by 512 / 128 lanes: 64 rows 3.7 / 5.1, 1000 7.6 / 9.5, 1500 11.2 / 11.3, 8192 38.1 / 32.5; 88 places,
    // 6200 rows 27.6 / 11.0.
    const uint32_t places = (p.n_heads * (p.qs ? 1u : 0u) + p.n_kv_heads) * steps + p.n_kv_heads * (p.dim / n);
    const uint32_t most = p.n_rows <= 1024u ? 512u : 256u, turns = (places + most - 1u) / most;
    const uint32_t threads = ((places + turns - 1u) / turns + 63u) / 64u * 64u;
    switch (kind) {
    case 0: launch_put<dkv::Bf16, false>(eights, threads, s, p); break;
    case 1: launch_put<dkv::Fp16, false>(eights, threads, s, p); break;
    case 2: launch_put<dkv::Bf16, true>(eights, threads, s, p); break;
    default: launch_put<dkv::Fp16, true>(eights, threads, s, p); break;
    }
    DECTRY(hipGetLastError());
    return KV_OK;
}

int kv_attend(kv_decoder *d, const kv_attend_args *a, void *stream)
{
    if (!d || !a || a->layer < 0 || a->layer >= d->cfg.n_layers || a->n_seqs < 0) return KV_EINVAL;
    const float qk_scale = (float)((double)a->scale * 1.4426950408889634074 * (double)d->dc.k_scale);
    if (!std::isfinite(qk_scale)) return KV_EINVAL;
    if (a->n_seqs > d->dc.max_seqs) return KV_E2BIG;
    if (a->n_seqs > 0 && (!a->table || !a->lens || !a->q.data || !a->out.data)) return KV_EINVAL;
    if (!rows_ok(a->q) || !rows_ok(a->out)) return KV_EINVAL;
    if (a->n_seqs > 1 && (a->table_stride < d->dc.max_blocks || (a->mass_out && a->mass_stride < d->dc.max_blocks))) return KV_EINVAL;
    if (a->mass && !a->mass_out) return KV_EINVAL;
    if (a->mass_out && !d->dc.weigh) return KV_EUNSUP;
    if (!rows_aligned(a->q) || !rows_aligned(a->out)) return KV_EUNSUP;
    if (!apart(a->out, a->n_seqs, d->dc.n_heads, d->dim)) return KV_EINVAL;
    if (a->n_seqs == 0) return KV_OK;
    OnDevice on(d->device);
    if (!on.ok()) return KV_EHIP;
    dkv::AttendParams p{};
    p.k = plane(d, a->layer, 0);
    p.v = plane(d, a->layer, 1);
    p.table = a->table;
    p.lens = a->lens;
    p.q = (const uint8_t *)a->q.data;
    p.out = (uint8_t *)const_cast<void *>(a->out.data);
    p.lse = a->lse;
    p.part = d->part;
    p.part_ml = d->part_ml;
    p.lse2 = d->lse2;
    p.granules = a->mass_out ? d->granules : nullptr;
    p.mass = a->mass;
    p.mass_out = a->mass_out;
    p.mass_stride = a->mass_stride;
    p.q_row = 2ull * (uint64_t)a->q.row;
    p.q_head = 2ull * (uint64_t)a->q.head;
    p.out_row = 2ull * (uint64_t)a->out.row;
    p.out_head = 2ull * (uint64_t)a->out.head;
    p.table_stride = a->table_stride;
    p.n_seqs = (uint32_t)a->n_seqs;
    p.n_heads = (uint32_t)d->dc.n_heads;
    p.max_blocks = (uint32_t)d->dc.max_blocks;
    p.max_tokens = p.max_blocks * (uint32_t)d->cfg.block_size;
    p.bias = dkv::bf16_bias(p.max_tokens);
    p.share = dkv::Share::of(p.max_tokens);
    p.dim = (uint32_t)d->dim;
    p.token_bytes = d->token_bytes;
    p.head_bytes = d->head_bytes;
    p.exponents = d->exponents;
    p.block_size = (uint32_t)d->cfg.block_size;
    p.cells_per_block = d->cells_per_block;
    p.n_blocks = (uint32_t)d->cfg.n_hbm_blocks;
    p.units = d->units;
    p.group_heads = (uint32_t)(d->dc.n_heads / d->cfg.n_kv_heads);
    p.head_tiles = d->head_tiles;
    p.part_rows = d->part_rows;
    p.part_vecs = d->part_vecs;
    p.by_items = dkv::Divide::by(p.part_vecs / 4u);
    p.by_rows = dkv::Divide::by(p.part_rows);
    p.by_head_tiles = dkv::Divide::by(p.head_tiles);
    p.granule = d->granule;
    p.granule_bits = (uint32_t)__builtin_ctz(d->granule);
    p.by_block = dkv::Divide::by(p.block_size);
    p.max_granules = d->max_granules;
    // Few numbers a block: four lanes for it, so that a workgroup has more blocks; up to 64, where there are more workgroups
    // than the chip holds at once, eight.  us of the second launch, four / 16 lanes: 63 requests of 1203 blocks of 20
    // numbers 7.9 / 13.7, 32 of 512 of 32 7.9 / 8.2, 2 of 710 of 24 10.6 / 9.7; eight / 16: 118 of 1594 of 40 16.3 / 25.0, 37 of
    // 340 of 45 6.4 / 6.1.
    const uint32_t numbers = p.block_size / p.granule * p.n_heads;
    const uint64_t mass_wgs = (uint64_t)p.n_seqs * p.max_blocks / dkv::mass_blocks(4u);
    p.mass_bits = numbers <= 32u ? 2u : numbers <= 64u && mass_wgs > 8ull * (uint32_t)d->n_cus ? 3u : 4u;
    p.qk_scale = qk_scale;
    p.v_scale = d->dc.v_scale;
    const uint32_t tiles = (p.max_tokens + dkv::kTile - 1) / dkv::kTile;
    // Up to 16 requests: half as many units, and two waves each, to a workgroup, so that ranges are longer and leave half as many
    // parts.  More requests: a wave each, so that ranges meet fewer of their ends.  us, by eight / by four: 4 requests of
    // 32768 tokens (64 query heads) 93.2 / 90.7, one of 8192 17.7 / 16.7; 32 around 1024 43.4 / 45.6.
    Workgroup w(d->units, p.n_seqs <= kFewRequests ? d->waves / 2 : d->waves, d->waves);
    // Where no request can be longer than three steps of its waves, each is a range, and nothing is left to join: with
    // fewer units, and so more waves for each, to a workgroup, as long as two workgroups per compute unit take all requests,
    // and no second launch is needed for block weights anyway.  us, split and joined / a range each: 3 requests of up to
    // 100 tokens 9.6 / 5.9; 32 of 192 15.2 / 10.6, of 512 21.1 / 15.7; 128 of 256 31.0 / 27.6; 3 of 600, three steps, 15.3 /
    // 12.3; 4 of 1000, four steps, 14.0 / 17.6; with weights 16 of up to 512 13.0 / 15.2.
    // Where one range each fills the chip, up to six steps: 300 of up to 128 tokens 25.7 / 24.2, of 8-bit and up to 160 24.3 /
    // 21.1; 1000 of up to 128 65.8 / 61.9; 512 of up to 192 42.9 / 42.0, 300 31.2 / 31.6.
    // More waves for each, up to one a tile, as long as a compute unit has one workgroup: us with as few / as many, 32 requests
    // of 64 tokens 10.5 / 8.4, of 192 10.7 / 9.3, 2 of 256 10.2 / 8.3; with two workgroups a compute unit 64 of 256 14.8 / 19.3.
    for (uint32_t most = d->waves; most > 0 && !p.by_request; most /= 2) {
        const Workgroup x(d->units, most, d->waves);
        const bool full = !p.granules && most == d->waves && p.n_seqs * x.per_range >= (uint32_t)d->n_cus;
        if (tiles > (full ? 6u : 3u) * x.subs) continue;
        if (most < d->waves && (p.n_seqs * x.per_range > 2u * (uint32_t)d->n_cus || p.granules)) continue;
        w = x;
        p.by_request = 1u;
        for (uint32_t fewer = most / 2; fewer > 0 && w.subs < tiles; fewer /= 2) {
            const Workgroup y(d->units, fewer, d->waves);
            if (p.n_seqs * y.per_range > (uint32_t)d->n_cus) break;
            w = y;
        }
    }
    p.wgs_per_group = w.per_range;
    p.units_per_wg = w.units;
    p.subs = w.subs;
    // no more ranges than there is memory for, and than there can be turns in this call
    p.groups = p.by_request ? p.n_seqs
                            : (uint32_t)std::min<uint64_t>(std::min(d->max_groups, ranges(d, w)), (uint64_t)p.n_seqs * tiles);
    hipStream_t s = (hipStream_t)stream;
    const dim3 g(p.groups * p.wgs_per_group), b(64 * p.units_per_wg * p.subs);
    int dp;
    const int kind = kinds(d, dp);
    switch (kind) {
    case 0: launch_attend<dkv::Bf16, dkv::kBits16>(dp, g, b, s, p); break;
    case 1: launch_attend<dkv::Fp16, dkv::kBits16>(dp, g, b, s, p); break;
    case 2: launch_attend<dkv::Bf16, dkv::kBits8>(dp, g, b, s, p); break;
    case 3: launch_attend<dkv::Fp16, dkv::kBits8>(dp, g, b, s, p); break;
    case 4: launch_attend<dkv::Bf16, dkv::kBits4>(dp, g, b, s, p); break;
    default: launch_attend<dkv::Fp16, dkv::kBits4>(dp, g, b, s, p); break;
    }
    DECTRY(hipGetLastError());
    const uint32_t lines = (p.units * p.part_vecs / 4u + 7u) / 8u;
    if (!p.by_request) p.joins = std::min(lines, std::max(1u, kJoinWgs / p.n_seqs));
    const uint32_t mass_blocks = dkv::mass_blocks(p.mass_bits);
    const dim3 gj(p.joins + (p.granules ? (p.max_blocks + mass_blocks - 1u) / mass_blocks : 0u), p.n_seqs);
    if (gj.x == 0u) return KV_OK;
    if (d->dc.x_type == KV_FP16) hipLaunchKernelGGL(dkv::kv_join_kernel<dkv::Fp16>, gj, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(dkv::kv_join_kernel<dkv::Bf16>, gj, dim3(256), 0, s, p);
    DECTRY(hipGetLastError());
    return KV_OK;
}

int kv_evict(kv_decoder *d, const kv_evict_args *a, void *stream)
{
    if (!d || !a || a->n_seqs < 0 || a->budget < 0 || a->n_first < 0 || a->n_last < 1 || a->max_evict < 0) return KV_EINVAL;
    if (a->n_seqs > d->dc.max_seqs) return KV_E2BIG;
    if (a->n_seqs > 1 && (a->table_stride < d->dc.max_blocks || a->mass_stride < d->dc.max_blocks)) return KV_EINVAL;
    if (a->n_seqs == 0) return KV_OK;
    if (!a->table || !a->table_out || !a->lens || !a->lens_out || !a->mass || !a->mass_out || !a->n_evicted ||
        (a->max_evict > 0 && (!a->evicted_ids || !a->evicted_at)))
        return KV_EINVAL;
    OnDevice on(d->device);
    if (!on.ok()) return KV_EHIP;
    dkv::EvictParams p{};
    p.table = a->table;
    p.lens = a->lens;
    p.table_out = a->table_out;
    p.lens_out = a->lens_out;
    p.mass = a->mass;
    p.mass_out = a->mass_out;
    p.ids = a->evicted_ids;
    p.at = a->evicted_at;
    p.count = a->n_evicted;
    p.table_stride = a->table_stride;
    p.mass_stride = a->mass_stride;
    p.max_blocks = (uint32_t)d->dc.max_blocks;
    p.block_size = (uint32_t)d->cfg.block_size;
    p.budget = (uint32_t)a->budget;
    p.n_first = (uint32_t)a->n_first;
    p.n_last = (uint32_t)a->n_last;
    p.max_evict = (uint32_t)a->max_evict;
    const dim3 g((uint32_t)a->n_seqs);
    hipStream_t s = (hipStream_t)stream;
    if (p.max_blocks <= 512u) hipLaunchKernelGGL((dkv::kv_evict_kernel<512, 1, 11>), g, dim3(512), 0, s, p);
    else if (p.max_blocks <= 2048u) hipLaunchKernelGGL((dkv::kv_evict_kernel<1024, 2, 11>), g, dim3(1024), 0, s, p);
    else if (p.max_blocks <= 4096u) hipLaunchKernelGGL((dkv::kv_evict_kernel<1024, 4, 11>), g, dim3(1024), 0, s, p);
    else hipLaunchKernelGGL((dkv::kv_evict_kernel<1024, 8, 11>), g, dim3(1024), 0, s, p);
    DECTRY(hipGetLastError());
    return KV_OK;
}

}  // extern "C"
