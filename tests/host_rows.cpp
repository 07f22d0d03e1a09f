// CPU-only checks of the host code of attention of many rows, of decoders over a cache in 4 bits and of normed heads, against
// a stand-in for the HIP runtime that notes every launch and runs none.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "../paper_2601_20309_amd/csrc/kv_decode.hip"
#include "../paper_2601_20309_amd/csrc/kv_rows.hip"

#define CHECK(cond, ...)                                              \
    do {                                                              \
        if (!(cond)) {                                                \
            std::fprintf(stderr, "FAIL %s:%d: ", __FILE__, __LINE__); \
            std::fprintf(stderr, __VA_ARGS__);                        \
            std::fprintf(stderr, "\n");                               \
            std::exit(1);                                             \
        }                                                             \
    } while (0)

namespace {
struct Launch {
    dim3 g, b;
    std::vector<unsigned char> args;
};
std::vector<Launch> launches;
size_t arg_bytes = 0, allocated = 0;
int device_now = 0;
struct {
    dim3 g, b;
    size_t shared;
    hipStream_t s;
} next_launch;
}  // namespace

extern "C" {
uint64_t kv_seg_bytes(const kv_config *c) { return (uint64_t)c->block_size * c->n_kv_heads * c->head_dim * c->elem_bytes; }
uint64_t kv_cache_bytes(const kv_config *c) { return c->n_layers > 0 ? 2ull * c->n_layers * kv_seg_bytes(c) * c->n_hbm_blocks : 0; }
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, unsigned long, int, int) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t shared, hipStream_t s) { next_launch = {g, b, shared, s}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *shared, hipStream_t *s)
{
    *g = next_launch.g; *b = next_launch.b; *shared = next_launch.shared; *s = next_launch.s;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *, dim3 g, dim3 b, void **args, size_t, hipStream_t)
{
    CHECK(device_now == 3, "launched on device %d", device_now);
    CHECK((uint64_t)g.x * b.x <= 0xFFFFFFFFull, "more lanes than a launch counts");
    const auto *a = static_cast<unsigned char *>(args[0]);
    launches.push_back({g, b, {a, a + arg_bytes}});
    return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipGetDevice(int *d) { *d = device_now; return hipSuccess; }
hipError_t hipSetDevice(int d) { device_now = d; return hipSuccess; }
hipError_t hipGetDeviceCount(int *n) { *n = 4; return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "none"; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) { allocated = n; *p = std::calloc(1, 64); return hipSuccess; }
hipError_t hipMemset(void *, int, size_t) { return hipSuccess; }
hipError_t hipMemGetAddressRange(hipDeviceptr_t *base, size_t *n, hipDeviceptr_t) { *base = nullptr; *n = ~(size_t)0; return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *a, const void *)
{
    a->type = hipMemoryTypeDevice;
    a->device = 3;
    return hipSuccess;
}
}

namespace {
kv_config shape(int layers, int heads, int dim, int p, int elem, int blocks)
{
    kv_config c{};
    c.n_layers = layers; c.n_kv_heads = heads; c.head_dim = dim; c.block_size = p; c.elem_bytes = elem;
    c.n_hbm_blocks = blocks; c.n_host_slots = 1; c.hbm_layout = KV_HBM_LAYER_FIRST;
    return c;
}

int create(kv_decoder **d, const kv_config &c, kv_decoder_config dc) { return kv_decoder_create(d, &c, &dc, (void *)0x100000); }
kv_rows rows(int64_t row, int64_t head, uintptr_t at = 0x2000) { return kv_rows{(void *)at, row, head}; }

void creation()
{
    kv_decoder *d = nullptr;
    auto of = [&](int head_dim, int elem, int type, int max_rows = 0, int n_heads = 4, int seqs = 8, int heads = 2, float scale = 1.f) {
        const int rc = create(&d, shape(2, heads, head_dim, 16, elem, 40), {n_heads, KV_BF16, type, seqs, 16, scale, scale, 0, max_rows});
        if (d) kv_decoder_destroy(d);
        return rc;
    };
    CHECK(of(68, 1, KV_FP4) == KV_OK && of(17, 1, KV_FP4) == KV_OK && of(136, 1, KV_FP4) == KV_OK, "4 bits");
    CHECK(of(64, 1, KV_FP4) == KV_EINVAL && of(68, 2, KV_FP4) == KV_EINVAL && of(68, 1, KV_FP4, 0, 4, 8, 2, 2.f) == KV_EINVAL, "4 bits");
    CHECK(of(153, 1, KV_FP4) == KV_EUNSUP && of(68, 1, KV_BF16) == KV_EINVAL && of(68, 1, 4) == KV_EINVAL, "4 bits");
    CHECK(of(64, 2, KV_BF16, -1) == KV_EINVAL && of(64, 2, KV_BF16, 1) == KV_OK, "rows");
    CHECK(of(64, 2, KV_BF16, 0x7FFFFFFF) == KV_EUNSUP && of(64, 2, KV_BF16, 0x3FFFFF00, 4) == KV_EUNSUP, "rows");
    CHECK(of(64, 2, KV_BF16, 0x10000000, 2) == KV_OK, "rows");
    CHECK(create(&d, shape(2, 2, 68, 16, 1, 40), {4, KV_FP16, KV_FP4, 8, 16, 1.f, 1.f, 0, 0}) == KV_OK, "create");
    CHECK(d->dim == 128 && d->head_bytes == 64 && d->exponents == 128 && d->token_bytes == 136, "a row in 4 bits");
    kv_decoder_destroy(d);
}

void refusals()
{
    kv_decoder *d = nullptr;
    CHECK(create(&d, shape(2, 2, 64, 16, 2, 40), {4, KV_BF16, KV_BF16, 8, 16, 1.f, 1.f, 0, 100}) == KV_OK, "create");
    int32_t *const ints = (int32_t *)0x4000;
    const kv_attend_rows_args a0{1, 3, 50, 16, 1, 0.125f, ints, ints, ints, rows(256, 64), rows(256, 64), nullptr};
    auto attend = [&](auto &&f) { kv_attend_rows_args a = a0; f(a); return kv_attend_rows(d, &a, nullptr); };
    arg_bytes = sizeof(int);
    CHECK(attend([](auto &) {}) == KV_OK && !launches.empty() && device_now == 0, "the plain one");
    launches.clear();
    CHECK(kv_attend_rows(nullptr, &a0, nullptr) == KV_EINVAL && kv_attend_rows(d, nullptr, nullptr) == KV_EINVAL, "NULL");
#define EINVALS(...) CHECK(attend([](auto &a) { __VA_ARGS__; }) == KV_EINVAL, #__VA_ARGS__)
#define EUNSUPS(...) CHECK(attend([](auto &a) { __VA_ARGS__; }) == KV_EUNSUP, #__VA_ARGS__)
    EINVALS(a.layer = -1);
    EINVALS(a.layer = 2);
    EINVALS(a.n_seqs = -1);
    EINVALS(a.n_rows = -1);
    EINVALS(a.starts = nullptr);
    EINVALS(a.scale = std::nanf(""));
    EINVALS(a.scale = INFINITY);
    EINVALS(a.scale = 3e38f);
    EINVALS(a.table = nullptr);
    EINVALS(a.lens = nullptr);
    EINVALS(a.q.data = nullptr);
    EINVALS(a.out.data = nullptr);
    EINVALS(a.q.row = -256);
    EINVALS(a.q.head = -64);
    EINVALS(a.out.row = 0);
    EINVALS(a.out.head = 0);
    EINVALS(a.out.row = 248);
    EINVALS(a.table_stride = 15);
    EUNSUPS(a.q.data = (void *)0x2008);
    EUNSUPS(a.q.row = 260);
    EUNSUPS(a.out.head = 68);
    CHECK(attend([](auto &a) { a.n_seqs = 9; }) == KV_E2BIG && attend([](auto &a) { a.n_rows = 101; }) == KV_E2BIG, "too many");
    CHECK(launches.empty(), "something refused was launched");
    CHECK(attend([](auto &a) { a.n_seqs = 0; a.table = nullptr; }) == KV_OK && attend([](auto &a) { a.n_rows = 0; a.q.data = nullptr; }) == KV_OK, "none");
    CHECK(launches.empty(), "nothing to do was launched");
    CHECK(attend([](auto &a) { a.n_seqs = 1; a.table_stride = 0; }) == KV_OK && attend([](auto &a) { a.starts = nullptr; a.n_rows = 3; }) == KV_OK, "fine");
    CHECK(attend([](auto &a) { a.q = rows(0, 0); a.causal = 0; a.scale = 0.f; }) == KV_OK, "fine");

    kv_put_args p0{};
    p0.layer = 1; p0.n_seqs = p0.n_rows = 3; p0.table_stride = 16; p0.table = p0.lens = ints;
    p0.k = p0.v = rows(128, 64); p0.q = p0.q_out = rows(256, 64);
    p0.q_norm = p0.k_norm = (const float *)0x8000; p0.norm_eps = 1e-6f;
    auto put = [&](auto &&f) { kv_put_args a = p0; f(a); return kv_put(d, &a, nullptr); };
    launches.clear();
    CHECK(put([](auto &) {}) == KV_OK && launches.size() == 1, "norms");
    CHECK(put([](auto &a) { a.q.data = a.q_out.data = nullptr; }) == KV_EINVAL && put([](auto &a) { a.norm_eps = -1.f; }) == KV_EINVAL, "norms");
    CHECK(put([](auto &a) { a.norm_eps = INFINITY; }) == KV_EINVAL && put([](auto &a) { a.norm_eps = std::nanf(""); }) == KV_EINVAL, "norms");
    CHECK(put([](auto &a) { a.k_norm = (const float *)0x8008; }) == KV_EUNSUP && launches.size() == 1, "norms");
    CHECK(put([](auto &a) { a.q.data = a.q_out.data = nullptr; a.q_norm = nullptr; a.norm_eps = 0.f; }) == KV_OK, "k alone");
    CHECK(put([](auto &a) { a.q_norm = a.k_norm = nullptr; a.norm_eps = -1.f; }) == KV_OK, "no norm");
    kv_decoder_destroy(d);
}

// Every workgroup has a tile, and what splits leave lies inside what was allocated for it.
void launched()
{
    for (int heads : {1, 2, 3, 8, 9, 40}) {
        for (int group : {1, 4, 5, 24}) {
            for (int dim : {8, 64, 96, 128, 192, 256}) {
                for (int n : {1, 7, 300}) {
                    for (int n_rows : {1, 5, 128, 1000, 70001}) {
                        for (int blocks : {1, 9, 2000}) {
                            kv_decoder *d = nullptr;
                            if (heads * group > 1024) continue;
                            CHECK(create(&d, shape(1, heads, dim, 16, 2, 40), {heads * group, KV_BF16, KV_BF16, n, blocks, 1.f, 1.f, 0, n_rows}) == KV_OK, "create");
                            const char *const end = (const char *)d->part + allocated;
                            const kv_attend_rows_args a{0, n, n_rows, blocks, 1, 1.f, (int32_t *)16, (int32_t *)16, (int32_t *)16,
                                                        rows(heads * group * dim, dim), rows(heads * group * dim, dim), nullptr};
                            launches.clear();
                            arg_bytes = sizeof(dkv::RowsParams);
                            CHECK(kv_attend_rows(d, &a, nullptr) == KV_OK, "launch");
                            dkv::RowsParams x;
                            memcpy((void *)&x, launches[0].args.data(), sizeof x);
                            CHECK(x.splits >= 1 && launches.size() == (x.splits > 1 || x.groups ? 2u : 1u), "launches");
                            CHECK(launches[0].g.x == (x.groups ? x.groups * x.n_kv_heads : x.n_tiles * x.n_kv_heads * x.splits), "grid");
                            CHECK(!x.groups || (x.splits == 1 && x.row_bits == 5), "ranges are of tiles of 32 rows");
                            // the last request's last tile, wherever its rows are, comes before n_tiles
                            CHECK((uint64_t)n_rows * group / (1u << x.row_bits) + n <= x.n_tiles, "tiles");
                            if (x.splits > 1 || x.groups) {
                                const uint64_t slots = (x.groups ? 2ull * x.groups : (uint64_t)x.n_tiles * x.splits) * x.n_kv_heads;
                                const uint64_t vecs = (uint64_t)(1u << x.row_bits) * (dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256) / 4;
                                CHECK((const char *)(x.part + slots * vecs) <= (const char *)x.part_ml, "parts end");
                                CHECK((const char *)(x.part_ml + slots * (1u << x.row_bits)) <= end, "references end");
                            }
                            kv_decoder_destroy(d);
                        }
                    }
                }
            }
        }
    }
}

// As many tiles as a request needs lie between its first and the next one's.
void tiles()
{
    for (uint64_t tile : {32, 64, 128, 256})
        for (uint64_t group : {1, 3, 5, 8, 24, 1024})
            for (uint64_t start : {0ull, 1ull, 7ull, 127ull, 1000ull, 999999ull})
                for (uint64_t m : {0ull, 1ull, 2ull, 31ull, 129ull, 5000ull}) {
                    const uint64_t first = start * group / tile, next = (start + m) * group / tile + 1;
                    CHECK(next - first >= (m * group + tile - 1) / tile, "tiles of %d rows from %d", (int)m, (int)start);
                }
}
}  // namespace

int main()
{
    creation();
    refusals();
    launched();
    tiles();
    std::printf("host rows ok\n");
    return 0;
}
