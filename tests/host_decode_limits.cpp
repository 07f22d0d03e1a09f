// CPU-only checks of the decoder's limits: scales that 32 bits do not hold to base 2, and grids beyond what a launch counts.
#define main host_decode_main
#include "host_decode.cpp"
#undef main

namespace {
void scales()
{
    kv_decoder *d = nullptr;
    for (float k_scale : {1.f, 1e20f}) {
        const bool eight = k_scale != 1.f;
        CHECK(create(&d, shape(1, 2, 64, 16, eight ? 1 : 2, 40), {4, KV_BF16, eight ? KV_FP8 : KV_BF16, 2, 2, k_scale, 1.f, 0}) == KV_OK, "create");
        const kv_attend_args a0{0, 2, 2, 1.f, (int32_t *)16, (int32_t *)16, rows(256, 64), rows(256, 64), nullptr, nullptr, nullptr, 0};
        arg_bytes = sizeof(dkv::AttendParams);
        for (float scale : {0.f, -1.f, 1e-30f, 2.3e38f, -2.3e38f, 2.4e38f, -2.4e38f, 3e38f, 2.3e18f, 2.4e18f}) {
            launches.clear();
            kv_attend_args a = a0;
            a.scale = scale;
            const bool holds = std::fabs((double)scale * (double)k_scale * 1.4426950408889634074) < 3.4028235e38;
            CHECK(kv_attend(d, &a, nullptr) == (holds ? KV_OK : KV_EINVAL) && launches.empty() == !holds, "scale %g * %g", scale, k_scale);
        }
        kv_decoder_destroy(d);
    }
}

// A launch counts its lanes in 32 bits along an axis.
void grids()
{
    for (int heads : {1, 4, 65, 1024}) {
        for (int p : {1, 5, 16}) {
            for (int64_t blocks = 1 << 20; blocks * p <= 0x7FFFFFC0; blocks *= 2) {
                for (int weigh : {0, 1}) {
                    kv_decoder *d = nullptr;
                    const int rc = create(&d, shape(1, 1, 8, p, 2, 40), {heads, KV_BF16, KV_BF16, 1, (int)blocks, 1.f, 1.f, weigh});
                    if (rc != KV_OK) {
                        CHECK(rc == KV_EUNSUP && weigh && blocks > (1 << 28), "%d heads, %d tokens, %" PRId64 " blocks", heads, p, blocks);
                        continue;
                    }
                    kv_attend_args a{0, 1, (int)blocks, 1.f, (int32_t *)16, (int32_t *)16, rows(heads * 8, 8), rows(heads * 8, 8), nullptr, nullptr, nullptr, 0};
                    if (weigh) a.mass_out = (float *)16;
                    launches.clear();
                    arg_bytes = sizeof(dkv::AttendParams);
                    CHECK(kv_attend(d, &a, nullptr) == KV_OK, "attend");
                    for (const Launch &l : launches)
                        CHECK((uint64_t)l.g.x * l.b.x < 1ull << 32 && l.g.y <= 65535, "%d heads, %d tokens, %" PRId64 " blocks: %u workgroups", heads, p, blocks, l.g.x);
                    kv_decoder_destroy(d);
                }
            }
        }
    }
    // the most requests of the most heads
    kv_decoder *d = nullptr;
    CHECK(create(&d, shape(1, 1024, 8, 1, 2, 40), {1024, KV_BF16, KV_BF16, 65535, 1, 1.f, 1.f, 1}) == KV_OK, "create");
    for (int n : {1, 300, 65535}) {
        kv_attend_args a{0, n, 1, 1.f, (int32_t *)16, (int32_t *)16, rows(8192, 8), rows(8192, 8), nullptr, nullptr, (float *)16, 1};
        launches.clear();
        CHECK(kv_attend(d, &a, nullptr) == KV_OK, "attend");
        for (const Launch &l : launches) CHECK((uint64_t)l.g.x * l.b.x < 1ull << 32 && l.g.y <= 65535, "%d requests: %u workgroups", n, l.g.x);
    }
    kv_decoder_destroy(d);
}
}  // namespace

int main(int argc, char **argv)
{
    if (argc > 1 && !std::strcmp(argv[1], "scales")) scales();
    else grids();
    std::printf("host decode limits ok\n");
    return 0;
}
