// CPU-only checks of the decoder's host code against a stand-in for the HIP runtime that notes
// every launch and runs none: what is refused, what is launched, and whether what a launch may
// address lies inside the memory that the decoder holds.
#include <cinttypes>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <random>
#include <vector>

#include "../paper_2601_20309_amd/csrc/kv_decode.hip"

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
size_t arg_bytes = 0;  // of the next launches' one argument
size_t allocated = 0;
int device_now = 0;
bool device_memory = true;
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
hipError_t hipMemGetAddressRange(hipDeviceptr_t *base, size_t *n, hipDeviceptr_t) { *base = nullptr; *n = ~(size_t)0; return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *a, const void *)
{
    a->type = device_memory ? hipMemoryTypeDevice : hipMemoryTypeHost;
    a->device = 3;
    return hipSuccess;
}
}

namespace {
void *const kCache = (void *)0x100000;

kv_config shape(int layers, int heads, int dim, int p, int elem, int blocks, int hbm = KV_HBM_LAYER_FIRST)
{
    kv_config c{};
    c.n_layers = layers; c.n_kv_heads = heads; c.head_dim = dim; c.block_size = p; c.elem_bytes = elem;
    c.n_hbm_blocks = blocks; c.n_host_slots = 1; c.hbm_layout = hbm;
    return c;
}

int create(kv_decoder **d, const kv_config &c, kv_decoder_config dc, void *cache = kCache) { return kv_decoder_create(d, &c, &dc, cache); }

kv_rows rows(int64_t row, int64_t head, uintptr_t at = 0x2000) { return kv_rows{(void *)at, row, head}; }

// Pages, and the rows they make, in all the ways an id can be bad.
void pages()
{
    using dkv::cell_in;
    for (int64_t id : {-1ll, -2ll, (long long)INT32_MIN, 100ll, 101ll, (long long)INT32_MAX})
        CHECK(cell_in((uint32_t)(int32_t)id, 100, 16, 3) == dkv::kNoCell, "id %" PRId64, id);
    CHECK(cell_in(0, 100, 16, 3) == 3 && cell_in(99, 100, 16, 15) == 99 * 16 + 15, "good ids");
    CHECK(cell_in(0x7FFFFFFE, 0x7FFFFFFF, 2, 1) == 0xFFFFFFFD, "the largest");
}

void division()
{
    std::mt19937 rng(1);
    for (uint32_t d : {1u, 2u, 3u, 5u, 7u, 16u, 24u, 31u, 33u, 100u, 4095u, 65537u, 1u << 30, 0x7FFFFFFFu}) {
        const dkv::Divide by = dkv::Divide::by(d);
        for (int i = 0; i < 2000; i++) {
            const uint64_t k = rng() % (0x7FFFFFFFu / d + 1u);
            for (int64_t x : {(int64_t)(rng() >> 1), (int64_t)(k * d), (int64_t)(k * d) - 1, (int64_t)0x7FFFFFFF})
                if (x >= 0 && x <= 0x7FFFFFFF) CHECK(by.quotient((uint32_t)x) == (uint32_t)x / d, "%" PRId64 " / %u", x, d);
        }
    }
}

void weights()
{
    const float inf = std::numeric_limits<float>::infinity();
    const float up[] = {-inf, -3e38f, -1.f, -1e-45f, 0.f, 1e-45f, 1e-38f, 1.f, 3e38f, inf, std::nanf("")};
    for (size_t i = 0; i + 1 < sizeof up / sizeof *up; i++) CHECK(dkv::weight_key(up[i]) < dkv::weight_key(up[i + 1]), "weight %zu", i);
    CHECK(dkv::weight_key(-0.f) == dkv::weight_key(0.f), "zeros");
    CHECK(dkv::weight_key(-std::nanf("")) == dkv::weight_key(std::nanf("")), "NaN");
}

void creation()
{
    kv_decoder *d = nullptr;
    const kv_decoder_config ok{4, KV_BF16, KV_BF16, 8, 16, 1.f, 1.f, 1};
    const kv_config sh = shape(2, 2, 64, 16, 2, 40);
    auto with = [&](auto &&f) { kv_decoder_config x = ok; f(x); return create(&d, sh, x); };
    auto of = [&](const kv_config &c, int n_heads = 4) { kv_decoder_config x = ok; x.n_heads = n_heads; const int rc = create(&d, c, x); if (d) kv_decoder_destroy(d); return rc; };
    CHECK(kv_decoder_create(nullptr, &sh, &ok, kCache) == KV_EINVAL && kv_decoder_create(&d, nullptr, &ok, kCache) == KV_EINVAL, "NULL");
    CHECK(kv_decoder_create(&d, &sh, nullptr, kCache) == KV_EINVAL && create(&d, sh, ok, nullptr) == KV_EINVAL, "NULL");
    CHECK(of(sh) == KV_OK && device_now == 0, "the plain one");
    CHECK(with([](auto &x) { x.n_heads = 3; }) == KV_EINVAL && with([](auto &x) { x.n_heads = 0; }) == KV_EINVAL, "heads");
    CHECK(with([](auto &x) { x.n_heads = -2; }) == KV_EINVAL && with([](auto &x) { x.max_seqs = 0; }) == KV_EINVAL, "counts");
    CHECK(with([](auto &x) { x.max_blocks = -1; }) == KV_EINVAL && with([](auto &x) { x.x_type = KV_FP8; }) == KV_EINVAL, "counts, types");
    CHECK(with([](auto &x) { x.kv_type = KV_FP16; }) == KV_EINVAL && with([](auto &x) { x.kv_type = KV_FP8; }) == KV_EINVAL, "types");
    CHECK(with([](auto &x) { x.k_scale = 2.f; }) == KV_EINVAL && with([](auto &x) { x.v_scale = 0.f; }) == KV_EINVAL, "scales");
    CHECK(with([](auto &x) { x.max_seqs = 65536; }) == KV_EUNSUP && with([](auto &x) { x.max_blocks = 0x7FFFFFF; }) == KV_EUNSUP, "limits");
    CHECK(with([](auto &x) { x.max_seqs = 60000; x.max_blocks = 100000; }) == KV_EUNSUP, "tiles");
    CHECK(of(shape(1, 2, 264, 16, 2, 4)) == KV_EUNSUP && of(shape(1, 2, 60, 16, 2, 4)) == KV_EUNSUP, "dimensions");
    CHECK(of(shape(1, 1, 64, 16, 2, 4), 1025) == KV_EUNSUP && of(shape(1, 1, 64, 16, 2, 4), 1024) == KV_OK, "query heads");
    CHECK(of(shape(1, 1, 8, 16, 2, 0x10000000)) == KV_EUNSUP && of(shape(1, 1, 8, 16, 2, 0xFFFFFFF)) == KV_OK, "rows");
    CHECK(of(shape(0, 1, 8, 16, 2, 4)) == KV_EINVAL, "layers");
    CHECK(of(shape(1, 1, 8, 0x200000, 2, 4), 1024) == KV_EUNSUP && of(shape(1, 1, 8, 0x100000, 2, 4), 1024) == KV_OK, "granules of a block");
    CHECK(create(&d, sh, ok, (void *)0x100008) == KV_EUNSUP, "alignment");
    device_memory = false;
    CHECK(create(&d, sh, ok) == KV_EINVAL && d == nullptr, "host memory");
    device_memory = true;
    CHECK(kv_decoder_destroy(nullptr) == KV_EINVAL, "destroy");
}

void refusals()
{
    kv_decoder *d = nullptr;
    CHECK(create(&d, shape(2, 2, 64, 16, 2, 40), {4, KV_BF16, KV_BF16, 8, 16, 1.f, 1.f, 0}) == KV_OK, "create");
    int32_t *const ints = (int32_t *)0x4000;
    float *const floats = (float *)0x8000;
    const kv_attend_args a0{1, 3, 16, 0.125f, ints, ints, rows(256, 64), rows(256, 64), nullptr, nullptr, nullptr, 0};
    auto attend = [&](auto &&f) { kv_attend_args a = a0; f(a); return kv_attend(d, &a, nullptr); };
    kv_put_args p0{};
    p0.layer = 1; p0.n_seqs = p0.n_rows = 3; p0.table_stride = 16; p0.table = p0.lens = ints;
    p0.k = p0.v = rows(128, 64); p0.q = p0.q_out = rows(256, 64);
    p0.inv_freq = floats; p0.rot_dim = 64; p0.n_axes = 1; p0.sections[0] = 32;
    auto put = [&](auto &&f) { kv_put_args a = p0; f(a); return kv_put(d, &a, nullptr); };
    const kv_evict_args e0{3, 4, 1, 1, 5, 16, 16, ints, ints, ints, ints, floats, floats, ints, ints, ints};
    auto evict = [&](auto &&f) { kv_evict_args a = e0; f(a); return kv_evict(d, &a, nullptr); };
    auto nothing = [](auto &) {};
    arg_bytes = sizeof(int);
    CHECK(attend(nothing) == KV_OK && put(nothing) == KV_OK && evict(nothing) == KV_OK, "the plain ones");
    CHECK(!launches.empty() && device_now == 0, "launched, and the device as before");
    launches.clear();
    CHECK(kv_attend(nullptr, &a0, nullptr) == KV_EINVAL && kv_attend(d, nullptr, nullptr) == KV_EINVAL, "NULL");
    CHECK(kv_put(nullptr, &p0, nullptr) == KV_EINVAL && kv_evict(d, nullptr, nullptr) == KV_EINVAL, "NULL");
#define EINVALS(call, ...) CHECK(call([](auto &a) { __VA_ARGS__; }) == KV_EINVAL, #call ": " #__VA_ARGS__)
#define EUNSUPS(call, ...) CHECK(call([](auto &a) { __VA_ARGS__; }) == KV_EUNSUP, #call ": " #__VA_ARGS__)
    EINVALS(attend, a.layer = -1);
    EINVALS(attend, a.layer = 2);
    EINVALS(attend, a.n_seqs = -1);
    EINVALS(attend, a.scale = std::nanf(""));
    EINVALS(attend, a.scale = INFINITY);
    EINVALS(attend, a.table = nullptr);
    EINVALS(attend, a.lens = nullptr);
    EINVALS(attend, a.q.data = nullptr);
    EINVALS(attend, a.out.data = nullptr);
    EINVALS(attend, a.q.row = -256);
    EINVALS(attend, a.out.row = 0);
    EINVALS(attend, a.out.head = 0);
    EINVALS(attend, a.table_stride = 15);
    EINVALS(attend, a.mass = (float *)16);
    EUNSUPS(attend, a.mass_out = (float *)16; a.mass_stride = 16);
    EUNSUPS(attend, a.q.data = (void *)0x2008);
    EUNSUPS(attend, a.q.row = 260);
    EUNSUPS(attend, a.out.head = 68);
    CHECK(attend([](auto &a) { a.n_seqs = 9; }) == KV_E2BIG && put([](auto &a) { a.n_seqs = a.n_rows = 9; }) == KV_E2BIG, "requests");
    CHECK(evict([](auto &a) { a.n_seqs = 9; }) == KV_E2BIG, "requests");
    EINVALS(put, a.layer = 2);
    EINVALS(put, a.n_rows = -1);
    EINVALS(put, a.n_rows = 4);
    EINVALS(put, a.k.data = nullptr);
    EINVALS(put, a.v.data = nullptr);
    EINVALS(put, a.q.data = nullptr);
    EINVALS(put, a.q_out.data = nullptr);
    EINVALS(put, a.q_out.row = 0);
    EINVALS(put, a.lens = nullptr);
    EINVALS(put, a.table_stride = 3);
    EINVALS(put, a.rot_dim = 0);
    EINVALS(put, a.rot_dim = 72; a.sections[0] = 36);
    EINVALS(put, a.sections[0] = 31);
    EINVALS(put, a.sections[0] = -1);
    EINVALS(put, a.n_axes = 0);
    EINVALS(put, a.n_axes = 4);
    EINVALS(put, a.n_axes = 2; a.sections[0] = a.sections[1] = 16);                                     // two axes want positions
    EINVALS(put, a.n_axes = 2; a.sections[0] = a.sections[1] = 16; a.positions = (int32_t *)16; a.position_stride = 2);
    EINVALS(put, a.n_axes = 2; a.sections[0] = a.sections[1] = 16; a.positions = (int32_t *)16; a.position_stride = -3);
    // rows that are written into one another: neither token by token nor head by head
    EINVALS(put, a.q_out.row = 248);
    EINVALS(put, a.q_out.head = 56);
    EINVALS(attend, a.out.row = 128);
    EINVALS(attend, a.out = rows(64, 184));
    EINVALS(attend, a.out = rows(0x4000000000000000, 56));
    EUNSUPS(put, a.n_rows = 0x1000000; a.starts = (int32_t *)16);
    EUNSUPS(put, a.rot_dim = 12; a.sections[0] = 6);
    EUNSUPS(put, a.k.data = (void *)0x2004);
    EUNSUPS(put, a.v.row = 132);
    EINVALS(evict, a.n_seqs = -1);
    EINVALS(evict, a.budget = -1);
    EINVALS(evict, a.n_first = -1);
    EINVALS(evict, a.n_last = 0);
    EINVALS(evict, a.max_evict = -1);
    EINVALS(evict, a.table_stride = 15);
    EINVALS(evict, a.mass_stride = 15);
    EINVALS(evict, a.table_out = nullptr);
    EINVALS(evict, a.lens_out = nullptr);
    EINVALS(evict, a.mass = nullptr);
    EINVALS(evict, a.n_evicted = nullptr);
    EINVALS(evict, a.evicted_at = nullptr);
    CHECK(launches.empty(), "something refused was launched");
    CHECK(attend([](auto &a) { a.out = rows(64, 192); }) == KV_OK && put([](auto &a) { a.q_out = rows(64, 192); }) == KV_OK, "head by head");
    CHECK(attend([](auto &a) { a.n_seqs = 1; a.out = rows(0, 64); }) == KV_OK, "one row");
    CHECK(attend([](auto &a) { a.q = rows(0, 0); }) == KV_OK && put([](auto &a) { a.k = a.v = a.q = rows(0, 0); }) == KV_OK, "read several times");
    CHECK(put([](auto &a) { a.n_axes = 2; a.sections[0] = a.sections[1] = 16; a.positions = (int32_t *)16; }) == KV_OK, "one axis' positions");
    CHECK(put([](auto &a) { a.n_rows = 0xFFFFFF; a.starts = (int32_t *)16; }) == KV_OK && launches.back().b.x <= 256, "rows");
    launches.clear();
    // nothing to do is done without a launch, whatever the pointers
    CHECK(attend([](auto &a) { a.n_seqs = 0; a.table = nullptr; }) == KV_OK && evict([](auto &a) { a.n_seqs = 0; a.mass = nullptr; }) == KV_OK, "none");
    CHECK(put([](auto &a) { a.n_rows = 0; a.starts = (int32_t *)16; a.k.data = nullptr; }) == KV_OK && launches.empty(), "none");
    kv_decoder_destroy(d);
}

// Every range's parts, and every request's granules, lie inside what was allocated; every unit has a wave; a
// range's workgroups are no more than the chip has compute units for.
void attend_launches()
{
    for (int heads : {1, 2, 3, 5, 8, 9, 16, 40}) {
        for (int group : {1, 4, 8, 16, 24, 25}) {
            for (int dim : {8, 64, 72, 128, 192, 256}) {
                for (int p : {1, 5, 16, 24}) {
                    for (int n : {1, 7, 300}) {
                        for (int blocks : {1, 9, 2000}) {
                            kv_decoder *d = nullptr;
                            if (heads * group > 1024) continue;
                            CHECK(create(&d, shape(1, heads, dim, p, 2, 40), {heads * group, KV_BF16, KV_BF16, n, blocks, 1.f, 1.f, 1}) == KV_OK, "create");
                            const kv_attend_args a{0, n, blocks, 1.f, (int32_t *)16, (int32_t *)16, rows(heads * group * dim, dim), rows(heads * group * dim, dim),
                                                   nullptr, nullptr, (float *)16, blocks};
                            launches.clear();
                            arg_bytes = sizeof(dkv::AttendParams);
                            CHECK(kv_attend(d, &a, nullptr) == KV_OK && launches.size() == 2, "launches");
                            dkv::AttendParams x;
                            memcpy((void *)&x, launches[1].args.data(), sizeof x);
                            const uint64_t waves = launches[0].b.x / 64, tiles = ((uint64_t)blocks * p + 31) / 32;
                            CHECK(waves >= 1 && waves <= 8 && launches[0].b.x % 64 == 0 && waves == x.units_per_wg * x.subs, "waves");
                            CHECK((uint64_t)x.units == (uint64_t)heads * ((group + 15) / 16), "units");
                            CHECK((uint64_t)x.units_per_wg * x.wgs_per_group >= x.units && x.units_per_wg * (x.wgs_per_group - 1) < x.units, "every unit once");
                            CHECK(launches[0].g.x == x.groups * x.wgs_per_group, "grid");
                            if (x.by_request) {
                                CHECK(x.groups == (uint32_t)n && tiles <= (a.mass_out ? 3 : 6) * x.subs && x.joins == 0, "a range per request");
                            } else {
                                CHECK(x.groups >= 1 && x.groups <= dkv::kMaxGroups && x.groups * x.wgs_per_group <= 256 + x.wgs_per_group, "ranges");
                                CHECK(x.groups <= d->max_groups && x.joins >= 1, "memory for ranges");
                            }
                            const uint64_t slots = 2ull * d->max_groups;
                            CHECK(x.part_vecs % 4 == 0 && x.part_rows == (uint32_t)std::min(group, 16), "parts");
                            const char *const base = (const char *)x.part, *const end = base + allocated;
                            CHECK((const char *)(x.part + slots * x.units * x.part_vecs) <= (const char *)x.part_ml, "parts end");
                            CHECK((const char *)(x.part_ml + slots * x.n_heads) <= (const char *)x.lse2, "references end");
                            CHECK((const char *)(x.lse2 + (uint64_t)n * x.n_heads) <= (const char *)x.granules, "lse end");
                            CHECK((const char *)(x.granules + (uint64_t)n * x.max_granules * x.n_heads) <= end, "granules end");
                            CHECK(p % x.granule == 0 && 16 % x.granule == 0 && x.granule == 1u << x.granule_bits, "granule");
                            CHECK((uint64_t)x.max_granules * x.granule == (uint64_t)blocks * p, "granules");
                            CHECK(launches[1].g.y == (uint32_t)n && launches[1].g.x == x.joins + (blocks + dkv::mass_blocks(x.mass_bits) - 1) / dkv::mass_blocks(x.mass_bits), "join grid");
                            kv_decoder_destroy(d);
                        }
                    }
                }
            }
        }
    }
}
}  // namespace

int main()
{
    pages();
    division();
    weights();
    creation();
    refusals();
    attend_launches();
    std::printf("host decode ok\n");
    return 0;
}
