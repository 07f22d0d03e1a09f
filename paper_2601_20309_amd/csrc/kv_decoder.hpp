// The decoder's handle and what its calls' host code shares.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>

#include "../../include/duplexkv.h"
#include "kv_decode_kernels.hpp"

struct kv_decoder {
    kv_config cfg;
    kv_decoder_config dc;
    int device = 0, n_cus = 0;
    int32_t dim = 0;           // of a head; cfg.head_dim where the cache has more than 4 bits
    uint32_t head_bytes = 0, exponents = 0;  // of a head's numbers in a token; 4 bits: from its first byte to its heads' powers of 2
    uint8_t *hbm = nullptr;
    uint32_t token_bytes = 0, cells_per_block = 0;
    uint64_t plane_bytes = 0;  // from K to V of a layer, and half the way to the next layer
    // kv_attend: most waves of a workgroup, units (up to 16 query heads of a KV head), and the most ranges that there is memory for
    uint32_t waves = 0, units = 0, head_tiles = 0, max_groups = 0;
    uint32_t part_rows = 0, part_vecs = 0;
    uint32_t granule = 0, max_granules = 0;
    // one allocation, in this order
    dkv::f32x4 *part = nullptr;
    dkv::f32x4 *part_ml = nullptr;
    float *lse2 = nullptr, *granules = nullptr;
    // kv_attend_rows: what splits leave
    dkv::f32x4 *rows_part = nullptr;
    float2 *rows_ml = nullptr;
    uint8_t *rows_zeros = nullptr;  // what lies in pages that are not there: 16 bytes
};

namespace dkv {

#define DECTRY(call)                                                                                            \
    do {                                                                                                        \
        hipError_t err_ = (call);                                                                               \
        if (err_ != hipSuccess) {                                                                               \
            fprintf(stderr, "duplexkv: %s failed: %s (%s:%d)\n", #call, hipGetErrorString(err_), __FILE__, __LINE__); \
            return KV_EHIP;                                                                                     \
        }                                                                                                       \
    } while (0)

// The decoder's device is the current one for as long as this lives.
class OnDevice {
  public:
    explicit OnDevice(int device)
    {
        if (hipGetDevice(&before_) != hipSuccess) return;
        ok_ = before_ == device || hipSetDevice(device) == hipSuccess;
        moved_ = ok_ && before_ != device;
    }
    ~OnDevice()
    {
        if (moved_) (void)hipSetDevice(before_);
    }
    bool ok() const { return ok_; }

  private:
    int before_ = 0;
    bool ok_ = false, moved_ = false;
};

inline bool rows_ok(const kv_rows &r) { return r.row >= 0 && r.head >= 0; }
// 16-bit elements: rows begin on multiples of 16 bytes
inline bool rows_aligned(const kv_rows &r) { return (uintptr_t)r.data % 16 == 0 && r.row % 8 == 0 && r.head % 8 == 0; }

// rows that are written lie apart, token by token or head by head
inline bool apart(const kv_rows &r, int32_t n, int32_t heads, int32_t dim)
{
    const auto spans = [](int64_t outer, int64_t inner, int32_t n_outer, int32_t n_inner, int32_t dim) {
        const __int128 span = (__int128)inner * (n_inner - 1) + dim;
        return (n_inner < 2 || inner >= dim) && (n_outer < 2 || outer >= span);
    };
    return n <= 0 || spans(r.row, r.head, n, heads, dim) || spans(r.head, r.row, heads, n, dim);
}

inline uint8_t *plane(const kv_decoder *d, int32_t layer, int which)
{
    return d->hbm + (2ull * (uint64_t)layer + (uint64_t)which) * d->plane_bytes;
}

}  // namespace dkv
