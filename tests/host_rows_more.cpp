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
    }
}
}  // namespace

int main()
{
    arguments();
    largest_weights();
    std::printf("host rows more ok\n");
    return 0;
}
