// Sanitizer driver for the host side of decay attention and group norm (test infrastructure), beside dense_driver.cpp: calls
// qta_decay_attn* and qta_group_norm* with arguments that validation must reject and the workspace queries with valid ones over the
// whole range of sizes, so that AddressSanitizer and UndefinedBehaviorSanitizer see the validation, the rules of division and the
// layouts. Every call returns before a launch. Run by tests/test_sanitizers_decay.py.
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "qta.h"

namespace {

int failures = 0;
void expect(const char* what, long long got, long long want)
{
    if (got != want) {
        std::fprintf(stderr, "%s: %lld, expected %lld\n", what, got, want);
        ++failures;
    }
}
void* at(uintptr_t x) { return reinterpret_cast<void*>(x); }
constexpr uintptr_t kBase = 0x100000;       // aligned, never dereferenced

qta_decay_attn_args decay()
{
    qta_decay_attn_args a{};
    a.q = a.k = a.v = at(kBase);
    a.log_decay = static_cast<float*>(at(kBase));
    a.B = 2, a.heads = 4, a.N = 8, a.dk = 32, a.dv = 64;
    a.q_batch = a.k_batch = 1024, a.q_token = a.k_token = 128, a.q_head = a.k_head = 32;
    a.v_batch = 2048, a.v_token = 256, a.v_head = 64;
    return a;
}
qta_group_norm_args norm()
{
    qta_group_norm_args a{};
    a.x = at(kBase);
    a.B = 2, a.N = 10, a.C = 64, a.groups = 8;
    a.x_batch = 640, a.x_token = 64;
    a.eps = 1e-5f;
    return a;
}

template <typename Change>
void refused(const char* what, qta_status want, Change change)
{
    qta_decay_attn_args a = decay();
    change(a);
    float* const f = static_cast<float*>(at(kBase));
    expect(what, qta_decay_attn(&a, f, nullptr, nullptr, 0, nullptr), want);
    expect(what, qta_decay_attn_backward(&a, f, nullptr, f, f, f, nullptr, nullptr, 0, nullptr), want);
}
template <typename Change>
void norm_refused(const char* what, qta_status want, Change change)
{
    qta_group_norm_args a = norm();
    change(a);
    float* const f = static_cast<float*>(at(kBase));
    float* const y = static_cast<float*>(at(2 * kBase));
    expect(what, qta_group_norm(&a, y, nullptr, f, 0, nullptr), want);
    expect(what, qta_group_norm_backward(&a, f, y, static_cast<float*>(at(4 * kBase)), nullptr, nullptr, f, 0, nullptr), want);
}

}  // namespace

int main()
{
    using D = qta_decay_attn_args;
    using G = qta_group_norm_args;
    for (const int big : {0, -1, INT32_MIN}) {
        refused("B", QTA_ERR_INVALID, [=](D& a) { a.B = big; });
        refused("N", QTA_ERR_INVALID, [=](D& a) { a.N = big; });
        refused("heads", QTA_ERR_INVALID, [=](D& a) { a.heads = big; });
        refused("dk", QTA_ERR_INVALID, [=](D& a) { a.dk = big; });
        norm_refused("B", QTA_ERR_INVALID, [=](G& a) { a.B = big; });
        norm_refused("C", QTA_ERR_INVALID, [=](G& a) { a.C = big; });
        norm_refused("groups", QTA_ERR_INVALID, [=](G& a) { a.groups = big; });
    }
    refused("N", QTA_ERR_UNSUPPORTED, [](D& a) { a.N = INT32_MAX; });
    refused("B", QTA_ERR_UNSUPPORTED, [](D& a) { a.B = INT32_MAX; });
    refused("heads", QTA_ERR_UNSUPPORTED, [](D& a) { a.heads = INT32_MAX; });
    refused("token", QTA_ERR_UNSUPPORTED, [](D& a) { a.q_token = INT64_MAX / 4 * 4; });
    refused("batch", QTA_ERR_INVALID, [](D& a) { a.k_batch = INT64_MIN; });
    norm_refused("N", QTA_ERR_UNSUPPORTED, [](G& a) { a.N = INT32_MAX; });
    norm_refused("C", QTA_ERR_UNSUPPORTED, [](G& a) { a.C = INT32_MAX, a.groups = 1; });
    norm_refused("workspace", QTA_ERR_WORKSPACE, [](G&) {});
    norm_refused("eps", QTA_ERR_INVALID, [](G& a) { a.eps = -1.f; });
    long long queries = 0;
    for (const int dt : {0, 1})
        for (const int B : {1, 3, 64, 4096, 1 << 24})
            for (const int N : {1, 16, 17, 1000, 65536, 1 << 24, 1 << 30})
                for (const int n : {1, 3, 12, 32, 1 << 16}) {
                    for (const int d : {32, 64, 128}) {
                        D a = decay();
                        a.dtype = static_cast<qta_dtype>(dt);
                        a.B = B, a.N = N, a.heads = n, a.dk = d, a.dv = 160 - d > 128 ? 128 : 160 - d < 64 ? 32 : 64;
                        queries += (qta_decay_attn_workspace_bytes(&a) != 0) + (qta_decay_attn_backward_workspace_bytes(&a) != 0);
                    }
                    for (const int per : {1, 3, 8, 128, 4104})
                        for (const int token : {0, 1}) {
                            G a = norm();
                            a.dtype = static_cast<qta_dtype>(dt);
                            a.B = B, a.N = N, a.groups = n, a.per_token = token;
                            if (static_cast<long long>(n) * per > INT32_MAX) continue;
                            a.C = n * per;
                            queries += (qta_group_norm_workspace_bytes(&a) != 0) + (qta_group_norm_backward_workspace_bytes(&a) != 0);
                        }
                }
    std::printf("%lld sizes taken, %d failures\n", queries, failures);
    return failures != 0;
}
