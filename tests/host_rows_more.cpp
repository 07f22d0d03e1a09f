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
}  // namespace

int main()
{
    arguments();
    std::printf("host rows more ok\n");
    return 0;
}
