// Host-side paths of the serving entry points exercised without a GPU, built with csrc/api_serving.hip under
// -fsanitize=address,undefined by tests/test_serving_abi.py.  Every call below must return before any kernel launch.
#include "../include/atp.h"

#include <climits>
#include <cstdio>
#include <vector>

static int failures = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) { std::printf("FAILED line %d: %s\n", __LINE__, #cond); ++failures; } \
    } while (0)

int main() {
    std::vector<char> store(4096 + 64);
    char* P = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(store.data()) + 63) & ~uintptr_t(63));
    uint8_t* S = reinterpret_cast<uint8_t*>(P);
    const int32_t* I = reinterpret_cast<const int32_t*>(P);
    const size_t big = size_t(1) << 40;
    const atp_cache good = {P, P, nullptr, nullptr, 10, 16, 2, 64, ATP_CACHE_SAME};
    const atp_cache codes = {P, P, S, S, 10, 16, 2, 64, ATP_CACHE_E4M3};
    const atp_batch batch = {I, I, I, 3, 5, 7};

    const auto both = [&](const atp_cache* c, const atp_batch* b, const void* x, int64_t ld) {
        const atp_dtype t = ATP_BF16;
        const atp_status w = atp_cache_write(c, b, x, x, ld, ld, t, nullptr), r = atp_cache_read(c, b, const_cast<void*>(x), const_cast<void*>(x), ld, ld, t, nullptr);
        const atp_status a = atp_attention_paged(x, c, b, const_cast<void*>(x), ld, ld, 2, 1, 0.f, 0, nullptr, 0, t, nullptr);
        EXPECT(w == r && r == a);
        return w;
    };
    // a call of no tokens does nothing, whatever the tensors are
    atp_batch none = batch;
    none.tokens = 0;
    EXPECT(both(&good, &none, nullptr, 0) == ATP_OK && both(&codes, &none, nullptr, 0) == ATP_OK);
    EXPECT(both(nullptr, &batch, P, 128) == ATP_ERR_INVALID_ARG && both(&good, nullptr, P, 128) == ATP_ERR_INVALID_ARG);
    EXPECT(both(&good, &batch, nullptr, 128) == ATP_ERR_INVALID_ARG);
    EXPECT(both(&good, &batch, P + 2, 128) == ATP_ERR_INVALID_ARG);
    EXPECT(both(&good, &batch, P, 127) == ATP_ERR_INVALID_ARG);
    EXPECT(both(&good, &batch, P, 132) == ATP_ERR_INVALID_ARG);         // rows at no multiple of 16 bytes
    EXPECT(both(&good, &batch, P, -128) == ATP_ERR_INVALID_ARG);
    EXPECT(both(&good, &batch, P, INT64_MAX) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_cache_write(&good, &batch, P, P, 128, 128, (atp_dtype)5, nullptr) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_cache_read(&good, &batch, P, P, 128, 128, (atp_dtype)5, nullptr) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_attention_paged(P, &good, &batch, P, 128, 128, 2, 1, 0.f, 0, P, big, (atp_dtype)5, nullptr) == ATP_ERR_INVALID_ARG);
    const auto bad_cache = [&](auto change) { atp_cache c = good; change(c); return both(&c, &batch, P, 128); };
    EXPECT(bad_cache([](atp_cache& c) { c.K = nullptr; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([](atp_cache& c) { c.V = nullptr; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([&](atp_cache& c) { c.V = P + 8; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([&](atp_cache& c) { c.K_scale = S; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([](atp_cache& c) { c.type = ATP_CACHE_E4M3; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([](atp_cache& c) { c.type = (atp_cache_type)9; }) == ATP_ERR_INVALID_ARG);
    for (int32_t ps : {0, -16, 24, 131072, INT32_MIN}) EXPECT(bad_cache([&](atp_cache& c) { c.page_size = ps; }) == ATP_ERR_INVALID_ARG);
    for (int64_t n : {int64_t(0), int64_t(-1), INT64_MAX}) EXPECT(bad_cache([&](atp_cache& c) { c.n_pages = n; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([](atp_cache& c) { c.kv_heads = 0; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([](atp_cache& c) { c.d_h = 0; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_cache([](atp_cache& c) { c.d_h = 60; }) == ATP_ERR_UNSUPPORTED);
    EXPECT(bad_cache([](atp_cache& c) { c.d_h = 264; }) == ATP_ERR_UNSUPPORTED);
    const auto bad_batch = [&](auto change) { atp_batch b = batch; change(b); return both(&good, &b, P, 128); };
    EXPECT(bad_batch([](atp_batch& b) { b.table = nullptr; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_batch([](atp_batch& b) { b.length = nullptr; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_batch([](atp_batch& b) { b.offsets = nullptr; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_batch([&](atp_batch& b) { b.offsets = reinterpret_cast<const int32_t*>(P + 2); }) == ATP_ERR_INVALID_ARG);
    for (int64_t n : {int64_t(0), int64_t(-3), int64_t(65537), INT64_MAX}) EXPECT(bad_batch([&](atp_batch& b) { b.n_seq = n; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_batch([](atp_batch& b) { b.max_pages = 0; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_batch([](atp_batch& b) { b.max_pages = INT64_MAX; }) == ATP_ERR_UNSUPPORTED);
    EXPECT(bad_batch([](atp_batch& b) { b.max_pages = (1 << 26) + 1; }) == ATP_ERR_UNSUPPORTED);
    EXPECT(bad_batch([](atp_batch& b) { b.tokens = -1; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_batch([](atp_batch& b) { b.tokens = INT64_MAX; }) == ATP_ERR_INVALID_ARG);
    EXPECT(bad_batch([](atp_batch& b) { b.tokens = INT32_MAX; }) == ATP_ERR_UNSUPPORTED);
    EXPECT(atp_attention_paged(P, &good, &batch, P, 192, 192, 3, 1, 0.f, 0, P, big, ATP_BF16, nullptr) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_attention_paged(P, &good, &batch, P, 128, 128, 0, 1, 0.f, 0, P, big, ATP_BF16, nullptr) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_attention_paged(P, &good, &batch, P, 128, 128, 2, 1, 0.f, -1, P, big, ATP_BF16, nullptr) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_attention_paged(P, &good, &batch, P, 128, 128, 2, 1, 0.f, 0, P + 8, big, ATP_BF16, nullptr) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_attention_paged(P, &good, &batch, P, 128, 128, INT32_MAX - 1, 1, 0.f, 0, P, big, ATP_BF16, nullptr) == ATP_ERR_UNSUPPORTED);

    const auto packed = [&](const void* Q, const void* K, int64_t ldq, int64_t ldk, const int32_t* off, int64_t n_seq, int64_t tokens, int heads,
                            int hk, int d) {
        return atp_attention_packed(Q, K, K, const_cast<void*>(Q), ldq, ldk, ldk, ldq, off, n_seq, tokens, heads, hk, d, 1, 0.f, nullptr, 0, ATP_F32, nullptr);
    };
    EXPECT(packed(nullptr, nullptr, 0, 0, nullptr, 1, 0, 4, 2, 64) == ATP_OK);
    EXPECT(packed(nullptr, P, 256, 128, I, 1, 9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, nullptr, 256, 128, I, 1, 9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 128, nullptr, 1, 9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 255, 128, I, 1, 9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 126, I, 1, 9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 128, I, 0, 9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 128, I, INT64_MAX, 9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 128, I, 1, -9, 4, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 192, I, 1, 9, 4, 3, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 128, I, 1, 9, 0, 2, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 128, I, 1, 9, 4, 0, 64) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 256, 128, I, 1, 9, 4, 2, 0) == ATP_ERR_INVALID_ARG);
    EXPECT(atp_attention_packed(P, P, P, P, 256, 128, 128, 256, I, 1, 9, 4, 2, 64, 1, 0.f, P, big, (atp_dtype)7, nullptr) == ATP_ERR_INVALID_ARG);
    EXPECT(packed(P, P, 4096, 4096, I, 1, 9, 4, 2, 320) == ATP_ERR_UNSUPPORTED);
    EXPECT(packed(P, P, 240, 120, I, 1, 9, 4, 2, 60) == ATP_ERR_UNSUPPORTED);
    EXPECT(packed(P, P, 256, 128, I, 1, INT64_MAX, 4, 2, 64) == ATP_ERR_UNSUPPORTED);

    // workspace queries over sizes up to the limits: no overflow, and enough of it is asked for where it is asked for
    for (int64_t n_seq : {1, 7, 300, 65536}) for (int64_t tokens : {0, 1, 64, 5000, INT32_MAX / 256}) for (int d : {8, 64, 128, 256}) for (int hk : {1, 3, 32})
        for (int g : {1, 8}) for (int t = 0; t < 2; ++t) {
            EXPECT(atp_attention_packed_workspace(n_seq, tokens, hk * g, hk, d, (atp_dtype)t) % 256 == 0);
            for (int64_t pages : {int64_t(1), int64_t(4096), int64_t(1) << 26}) {
                atp_cache c = {nullptr, nullptr, nullptr, nullptr, 1, 16, hk, d, ATP_CACHE_SAME};
                const atp_batch b = {nullptr, nullptr, nullptr, n_seq, pages, tokens};
                const size_t w = atp_attention_paged_workspace(&c, &b, hk * g, 1, (atp_dtype)t);
                EXPECT(w % 256 == 0 && (tokens || !w));
                if (w) {
                    c = {P, P, nullptr, nullptr, 1, 16, hk, d, ATP_CACHE_SAME};
                    const atp_batch full = {I, I, I, n_seq, pages, tokens};
                    EXPECT(atp_attention_paged(P, &c, &full, P, hk * g * d, hk * g * d, hk * g, 1, 0.f, 1, P, w - 1, (atp_dtype)t, nullptr) == ATP_ERR_WORKSPACE);
                    EXPECT(atp_attention_paged(P, &c, &full, P, hk * g * d, hk * g * d, hk * g, 1, 0.f, 1, nullptr, w, (atp_dtype)t, nullptr) == ATP_ERR_WORKSPACE);
                }
            }
        }
    EXPECT(atp_attention_packed_workspace(1, 9, 4, 3, 64, ATP_F32) == 0 && atp_attention_packed_workspace(1, 9, 4, 2, 64, (atp_dtype)5) == 0);
    EXPECT(atp_attention_paged_workspace(nullptr, &batch, 4, 1, ATP_F32) == 0 && atp_attention_paged_workspace(&good, nullptr, 4, 1, ATP_F32) == 0);
    EXPECT(atp_attention_paged_workspace(&good, &batch, 3, 1, ATP_F32) == 0);
    std::printf("%s (%d failures)\n", failures ? "FAILED" : "host checks ok", failures);
    return failures ? 1 : 0;
}
