// CPU-only check of kv_table_drop: long random sequences of the block table's calls beside a plain
// list of what each request holds.  The engine's transfers are a stand-in that moves nothing.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <set>
#include <vector>

#include "../paper_2601_20309_amd/csrc/kv_engine.hpp"

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
int drains = 0, fail_drain = KV_OK;
}
extern "C" int kv_rotate(kv_engine *, const int32_t *, const int32_t *, int32_t, const int32_t *, const int32_t *, int32_t) { return KV_OK; }
extern "C" int kv_swap_out(kv_engine *, const int32_t *, const int32_t *, int32_t) { return KV_OK; }
int dkv::drain(kv_engine *e)
{
    if (fail_drain != KV_OK) return fail_drain;
    drains++;
    e->idle_epoch++;
    return KV_OK;
}

namespace {
struct Request {
    bool used = false, resident = false;
    int32_t len = 0;
    std::vector<int32_t> ids, slots, states;
};

Request look(kv_table *t, int32_t q)
{
    Request r;
    int32_t ids[512], slots[512], states[512], n = 0, info[2] = {0, 0};
    if (kv_table_blocks(t, q, ids, slots, states, 512, &n, info) != KV_OK) return r;
    r.used = true;
    r.resident = info[1] != 0;
    r.len = info[0];
    r.ids.assign(ids, ids + n);
    r.slots.assign(slots, slots + n);
    r.states.assign(states, states + n);
    return r;
}

void whole(kv_table *t, int32_t requests, int32_t nb, int32_t ns, int32_t P)
{
    std::set<int32_t> ids, slots;
    for (int32_t q = 0; q < requests; q++) {
        const Request r = look(t, q);
        if (!r.used) continue;
        CHECK((int32_t)r.ids.size() == (r.len + P - 1) / P, "request %d: %zu blocks of %d tokens", q, r.ids.size(), r.len);
        for (int32_t b : r.ids) CHECK(b < 0 ? !r.resident : ids.insert(b).second, "block %d", b);
        for (int32_t s : r.slots) CHECK(s < 0 || slots.insert(s).second, "slot %d twice", s);
        for (size_t i = 0; i < r.states.size(); i++) {
            const bool full = (int32_t)(i + 1) * P <= r.len;
            CHECK(!r.resident || full == (r.states[i] != KV_BLOCK_DIRTY) || r.states[i] == KV_BLOCK_SYNCED, "state %d of block %zu", r.states[i], i);
        }
    }
    kv_table_counts c{};
    CHECK(kv_table_get_counts(t, &c) == KV_OK, "counts");
    CHECK(c.free_hbm_blocks == nb - (int64_t)ids.size() && c.free_host_slots == ns - (int64_t)slots.size(), "free blocks and slots");
}

void run(uint64_t seed, int steps)
{
    std::mt19937_64 rng(seed);
    const int32_t nb = 60, ns = 80, P = 1 + (int32_t)(seed % 5), requests = 6;
    kv_engine e{};
    e.cfg.n_layers = e.cfg.n_kv_heads = 1; e.cfg.head_dim = 8; e.cfg.block_size = P; e.cfg.elem_bytes = 2;
    e.cfg.n_hbm_blocks = nb; e.cfg.n_host_slots = ns; e.cfg.path = KV_PATH_FUSED;
    kv_table *t = nullptr;
    CHECK(kv_table_create(&t, &e, requests) == KV_OK, "create");
    int dropped = 0, refused = 0;
    for (int step = 0; step < steps; step++) {
        const int32_t q = (int32_t)(rng() % requests);
        const Request before = look(t, q);
        switch (rng() % 7) {
        case 0: case 1: (void)kv_table_append(t, q, (int32_t)(rng() % (4 * P)), nullptr, 0, nullptr); break;
        case 2: { int32_t n; (void)kv_table_eager(t, (int32_t)(rng() % 5), &n); break; }
        case 3:
            if (before.used && before.resident) (void)kv_table_rotate(t, &q, 1, nullptr, 0);
            else if (before.used) (void)kv_table_rotate(t, nullptr, 0, &q, 1);
            break;
        case 4: if (rng() % 8 == 0 && before.used) CHECK(kv_table_finish(t, q) == KV_OK, "finish"); break;
        case 5: e.idle_epoch++; break;      // kv_wait
        default: {
            const int32_t full = before.len / P;
            std::vector<int32_t> at;
            for (int32_t i = 0; i < (int32_t)before.ids.size(); i++)
                if (rng() % 3 == 0) at.push_back(i);
            const bool bad = rng() % 4 == 0 && !at.empty();
            if (bad) {
                switch (rng() % 4) {
                case 0: at.back() = (int32_t)before.ids.size(); break;
                case 1: at.push_back(at.back()); break;
                case 2: at.front() = -1; break;
                default: std::reverse(at.begin(), at.end()); break;
                }
            }
            const bool fits = before.used && before.resident && std::is_sorted(at.begin(), at.end()) &&
                              std::adjacent_find(at.begin(), at.end()) == at.end() && (at.empty() || (at.front() >= 0 && at.back() < full));
            const int rc = kv_table_drop(t, q, at.data(), (int32_t)at.size());
            CHECK(rc == (fits ? KV_OK : KV_EINVAL), "step %d: drop returned %d", step, rc);
            const Request after = look(t, q);
            Request want = before;
            if (fits) {
                for (size_t i = at.size(); i-- > 0;) {
                    want.ids.erase(want.ids.begin() + at[i]);
                    want.slots.erase(want.slots.begin() + at[i]);
                    want.states.erase(want.states.begin() + at[i]);
                }
                want.len -= P * (int32_t)at.size();
                dropped += (int)at.size();
            } else {
                refused++;
            }
            CHECK(after.ids == want.ids && after.slots == want.slots && after.states == want.states && after.len == want.len &&
                      after.resident == want.resident && after.used == want.used, "step %d: what is left", step);
        }
        }
        whole(t, requests, nb, ns, P);
    }
    CHECK(dropped > steps / 40 && refused > steps / 100, "%d dropped, %d refused", dropped, refused);
    // a copy of its blocks may be under way: waited for, and a failure changes nothing
    for (int32_t q = 0; q < requests; q++)
        if (look(t, q).used) CHECK(kv_table_finish(t, q) == KV_OK, "finish");
    int32_t n = 0, first = 0;
    e.idle_epoch++;
    CHECK(kv_table_append(t, 0, 4 * P, nullptr, 0, nullptr) == KV_OK, "append");
    drains = 0;
    CHECK(kv_table_drop(t, 0, &first, 1) == KV_OK && drains == 0, "nothing under way");
    CHECK(kv_table_eager(t, 1, &n) == KV_OK && n == 1, "eager");
    fail_drain = KV_EHIP;
    const Request r = look(t, 0);
    CHECK(kv_table_drop(t, 0, &first, 1) == KV_EHIP && look(t, 0).ids == r.ids, "failed wait");
    fail_drain = KV_OK;
    CHECK(kv_table_drop(t, 0, &first, 1) == KV_OK && drains == 1 && look(t, 0).len == 2 * P, "waited");
    CHECK(kv_table_drop(nullptr, 0, &first, 1) == KV_EINVAL && kv_table_drop(t, -1, &first, 1) == KV_EINVAL &&
              kv_table_drop(t, requests, &first, 1) == KV_EINVAL && kv_table_drop(t, 5, nullptr, 0) == KV_EINVAL &&
              kv_table_drop(t, 0, nullptr, 1) == KV_EINVAL && kv_table_drop(t, 0, &first, -1) == KV_EINVAL, "arguments");
    CHECK(kv_table_drop(t, 0, nullptr, 0) == KV_OK, "none");
    // all of a request may go; it grows again
    const int32_t both[2] = {0, 1};
    CHECK(kv_table_drop(t, 0, both, 2) == KV_OK && look(t, 0).used && look(t, 0).len == 0, "all");
    CHECK(kv_table_append(t, 0, 1, nullptr, 0, &n) == KV_OK && n == 1 && look(t, 0).len == 1, "again");
    CHECK(kv_table_destroy(t) == KV_OK, "destroy");
}
}  // namespace

int main()
{
    for (uint64_t seed = 1; seed <= 10; seed++) run(seed, 4000);
    std::printf("host drop ok\n");
    return 0;
}
