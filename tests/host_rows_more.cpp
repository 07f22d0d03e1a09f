// CPU-only checks of what the host code of the decoder's calls hands to kernels.
#define main host_rows_main
#include "host_rows.cpp"
#undef main

#include <cstddef>

namespace {
// What only 4 bits and normed heads have lies behind what every kernel reads: in between, it costs the others' loads of arguments.
void arguments()
{
    CHECK(offsetof(dkv::AttendParams, exponents) > offsetof(dkv::AttendParams, v_scale), "kv_attend");
    for (size_t at : {offsetof(dkv::PutParams, q_norm), offsetof(dkv::PutParams, k_norm), offsetof(dkv::PutParams, eps),
                      offsetof(dkv::PutParams, inv_dim), offsetof(dkv::PutParams, exponents)})
        CHECK(at > offsetof(dkv::PutParams, v_scale), "kv_put");
}

// The largest weights of all tokens that there may be add up to a half at most, and no more is given away than that takes.
void largest_weights()
{
    for (uint32_t tokens : {1u, 16u, 4095u, 4096u, 4097u, 8192u, 70001u, 1u << 20, (1u << 28) + 1u, 0x7FFFFFC0u}) {
        const double most = std::exp2((double)dkv::bf16_bias(tokens) + (double)dkv::kBf16Slack);
        CHECK(most * tokens <= 0.5 && most * std::max(tokens, 4096u) > 0.25, "%u tokens: weights up to %g", tokens, most);
        const dkv::Share share = dkv::Share::of(tokens);
        CHECK(0x1p-8 * share.part * std::min(tokens, 1u << 28) <= 1.0 && (share.part == 1.0f || 0x1p-8 * share.part * tokens > 0.25), "%u tokens: %g of weights", tokens, (double)share.part);
        CHECK(share.exponents == (uint32_t)-std::ilogb(share.part) * 0x800080u && share.part >= 0x1p-20f, "%u tokens", tokens);
    }
}

// What parts of the tokens leave: no more memory than the most of them take, and room for it where there are most KV heads.
void memory()
{
    for (int heads : {1, 2, 40, 300, 1024})
        for (int dim : {8, 64, 72, 96, 128, 136, 256}) {
            kv_decoder *d = nullptr;
            const auto made = [&](int max_rows) {
                CHECK(create(&d, shape(1, heads, dim, 16, 2, 40), {heads, KV_BF16, KV_BF16, 70, 3000, 1.f, 1.f, 0, max_rows}) == KV_OK, "create");
                return allocated;
            };
            const size_t without = made(0);
            kv_decoder_destroy(d);
            const size_t dims = dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256, with = made(300);
            CHECK(with - without == 65536 * (dims * 4 + 8), "%d heads of %d: %zu bytes", heads, dim, with - without);
            for (int n : {1, 3, 70}) {
                const kv_attend_rows_args a{0, n, 300, 3000, 1, 1.f, (int32_t *)16, (int32_t *)16, (int32_t *)16, rows(heads * dim, dim), rows(heads * dim, dim), nullptr};
                launches.clear();
                arg_bytes = sizeof(dkv::RowsParams);
                CHECK(kv_attend_rows(d, &a, nullptr) == KV_OK, "launch");
                dkv::RowsParams x;
                memcpy((void *)&x, launches[0].args.data(), sizeof x);
                const uint64_t slots = (x.groups ? 2ull * x.groups : x.splits > 1 ? (uint64_t)x.n_tiles * x.splits : 0ull) * x.n_kv_heads;
                CHECK(slots << x.row_bits <= 65536, "%d heads of %d, %d requests: %d slots", heads, dim, n, (int)slots);
            }
            kv_decoder_destroy(d);
        }
}
}  // namespace

int main()
{
    arguments();
    largest_weights();
    memory();
    std::printf("host rows more ok\n");
    return 0;
}
