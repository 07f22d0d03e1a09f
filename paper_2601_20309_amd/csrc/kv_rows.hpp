// What attention of many rows asks of a decoder: limits, and memory for what splits leave.
#pragma once
#include <algorithm>

#include "kv_decoder.hpp"

namespace dkv {

constexpr uint64_t kMostTiles = 0xFFFFFF;  // as many workgroups of 256 lanes as a launch can count lanes

// Tiles of rows of one KV head, empty ones among them.
inline uint64_t row_tiles(int64_t n_rows, int64_t group, int64_t n_seqs, int bits) { return ((uint64_t)(n_rows * group) >> bits) + (uint64_t)n_seqs; }

// Heads of rows are counted in 31 bits, and the lanes of a launch in 32.
inline bool rows_fit(int64_t n_kv_heads, int64_t n_heads, int64_t n_seqs, int64_t n_rows)
{
    const int64_t group = n_heads / n_kv_heads;
    return n_rows * group <= 0x7FFFFF00 && (n_rows == 0 || row_tiles(n_rows, group, n_seqs, 7) * (uint64_t)n_kv_heads <= kMostTiles);
}

// Dimensions that the kernels are made for.
inline uint32_t rows_dims(uint32_t dim) { return dim <= 64u ? 64u : dim <= 96u ? 96u : dim <= 128u ? 128u : dim <= 192u ? 192u : 256u; }

// Rows that splits and ranges may leave sums of: splits of two workgroups to a compute unit, of 128 rows (or one, of 256), or two parts of 32
// rows of every range, as many ranges, and one of each KV head at least.
inline uint64_t row_sums(const kv_decoder *d) { return std::max(256ull * (uint64_t)d->n_cus, 64ull * (uint64_t)d->cfg.n_kv_heads); }

inline uint64_t rows_part_bytes(const kv_decoder *d) { return d->dc.max_rows ? row_sums(d) * rows_dims((uint32_t)d->dim) * 4u : 0u; }
inline uint64_t rows_ml_bytes(const kv_decoder *d) { return d->dc.max_rows ? row_sums(d) * sizeof(float2) : 0u; }

}  // namespace dkv
