// What attention of many rows asks of a decoder: limits, and memory for what splits leave.
#pragma once
#include <algorithm>

#include "kv_decoder.hpp"

namespace dkv {

// Workgroups of a call that is split: two for each of the most compute units that there are.
constexpr uint64_t kRowSlots = 512;
constexpr uint32_t kRowsOfTile = 128;

// Tiles of rows of one KV head, empty ones among them.
inline uint64_t row_tiles(int64_t n_rows, int64_t group, int64_t n_seqs) { return (uint64_t)(n_rows * group) / kRowsOfTile + (uint64_t)n_seqs; }

// Heads of rows are counted in 31 bits, and the lanes of a launch in 32.
inline bool rows_fit(int64_t n_kv_heads, int64_t n_heads, int64_t n_seqs, int64_t n_rows)
{
    const int64_t group = n_heads / n_kv_heads;
    return n_rows * group <= 0x7FFFFF00 && (n_rows == 0 || row_tiles(n_rows, group, n_seqs) * (uint64_t)n_kv_heads <= 0xFFFFFF);
}

// Dimensions that the kernels are made for.
inline uint32_t rows_dims(uint32_t dim) { return dim <= 64u ? 64u : dim <= 96u ? 96u : dim <= 128u ? 128u : dim <= 192u ? 192u : 256u; }

inline uint64_t rows_part_bytes(const kv_decoder *d) { return d->dc.max_rows ? kRowSlots * kRowsOfTile * (uint64_t)rows_dims(d->dim) * 4u : 0u; }
inline uint64_t rows_ml_bytes(const kv_decoder *d) { return d->dc.max_rows ? kRowSlots * kRowsOfTile * sizeof(float2) : 0u; }

}  // namespace dkv
