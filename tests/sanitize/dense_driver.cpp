// Sanitizer driver for the host side of rotary positions and differential attention (test infrastructure), beside
// abi_driver.cpp: calls qta_rotary and qta_diff_attn* with arguments that validation must reject and the workspace queries
// with valid ones over the whole range of sizes, so that AddressSanitizer and UndefinedBehaviorSanitizer see the validation,
// the splitting rules and the layouts. Every call returns before a launch. Run by tests/test_sanitizers_dense.py.
#include <cmath>
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

qta_diff_attn_args valid()
{
    qta_diff_attn_args a{};
    a.q = a.k = a.v = a.lam = at(kBase);
    a.B = 2, a.heads = 4, a.kv_heads = 2, a.Nq = 8, a.Nk = 16, a.d = 32;
    a.q_batch = 2048, a.q_token = 256, a.q_head = 32;
    a.k_batch = 2048, a.k_token = 128, a.k_head = 32;
    a.v_batch = 2048, a.v_token = 128, a.v_head = 64;
    a.lam_head = 1;
    return a;
}

qta_status forward(const qta_diff_attn_args& a, size_t bytes = 0)
{
    return qta_diff_attn(&a, at(kBase), nullptr, nullptr, nullptr, bytes, nullptr);
}
qta_status backward(const qta_diff_attn_args& a, size_t bytes)
{
    float* const f = static_cast<float*>(at(kBase));
    return qta_diff_attn_backward(&a, f, f, f, f, f, f, f, 1, f, bytes, nullptr);
}

template <typename Change>
void refused(const char* what, qta_status want, Change change)
{
    qta_diff_attn_args a = valid();
    change(a);
    expect(what, forward(a), want);
    expect(what, backward(a, size_t{1} << 60), want);
}

}  // namespace

int main()
{
    using Args = qta_diff_attn_args;
    expect("null", qta_diff_attn(nullptr, at(kBase), nullptr, nullptr, nullptr, 0, nullptr), QTA_ERR_INVALID);
    expect("null query", static_cast<long long>(qta_diff_attn_workspace_bytes(nullptr)), 0);
    expect("null query", static_cast<long long>(qta_diff_attn_backward_workspace_bytes(nullptr)), 0);
    expect("small workspace", backward(valid(), 16), QTA_ERR_WORKSPACE);
    refused("batch", QTA_ERR_INVALID, [](Args& a) { a.B = 0; });
    refused("heads", QTA_ERR_INVALID, [](Args& a) { a.heads = 3; });
    refused("kv heads", QTA_ERR_INVALID, [](Args& a) { a.kv_heads = -2; });
    refused("type", QTA_ERR_INVALID, [](Args& a) { a.dtype = static_cast<qta_dtype>(9); });
    refused("weight's type", QTA_ERR_INVALID, [](Args& a) { a.lam_dtype = QTA_BF16; });
    refused("q", QTA_ERR_INVALID, [](Args& a) { a.q = at(kBase + 4); });
    refused("lens", QTA_ERR_INVALID, [](Args& a) { a.lens = static_cast<const int32_t*>(at(kBase + 2)); });
    refused("stride", QTA_ERR_INVALID, [](Args& a) { a.v_token = 130; });
    refused("negative stride", QTA_ERR_INVALID, [](Args& a) { a.lam_token = INT64_MIN; });
    refused("scale", QTA_ERR_INVALID, [](Args& a) { a.scale = NAN; });
    refused("scale", QTA_ERR_INVALID, [](Args& a) { a.scale = INFINITY; });
    refused("d", QTA_ERR_UNSUPPORTED, [](Args& a) { a.d = 128; });
    refused("far tokens", QTA_ERR_UNSUPPORTED, [](Args& a) { a.k_token = INT64_MAX / 8 * 8; });
    refused("far heads", QTA_ERR_UNSUPPORTED, [](Args& a) { a.q_head = INT64_MAX / 8 * 8; });
    refused("rows", QTA_ERR_UNSUPPORTED, [](Args& a) { a.Nq = INT32_MAX; });
    refused("keys", QTA_ERR_UNSUPPORTED, [](Args& a) { a.Nk = INT32_MAX; });
    refused("all", QTA_ERR_UNSUPPORTED, [](Args& a) { a.B = a.heads = a.kv_heads = a.Nq = a.Nk = INT32_MAX; });

    // the queries over the range of sizes: room, or zero where a launch would be too large
    const int sizes[] = {1, 5, 31, 64, 1000, 4097, 1 << 16, 1 << 20, 1 << 26, 1 << 28, INT32_MAX};
    int taken = 0;
    for (const int B : {1, 16, 1 << 12, 1 << 24})
        for (const int heads : {1, 8, 64, 1 << 16})
            for (const int Nq : sizes)
                for (const int Nk : sizes)
                    for (const int kind : {0, 1, 2, 3}) {
                        Args a = valid();
                        a.B = B, a.heads = heads, a.kv_heads = heads >= 8 && kind == 2 ? heads / 8 : heads;
                        a.Nq = Nq, a.Nk = Nk, a.d = kind & 1 ? 64 : 32, a.dtype = kind & 2 ? QTA_BF16 : QTA_F32, a.causal = kind == 3;
                        const size_t f = qta_diff_attn_workspace_bytes(&a), b = qta_diff_attn_backward_workspace_bytes(&a);
                        if (f % 256 != 0 || b % 256 != 0) expect("a multiple of 256", 1, 0);
                        taken += f != 0;
                        if (f == 0) expect("past the range", forward(a), QTA_ERR_UNSUPPORTED);
                        if (f > 256) expect("no room", forward(a, f - 1), QTA_ERR_WORKSPACE);
                        if (b == 0) expect("past the range", backward(a, size_t{1} << 60), QTA_ERR_UNSUPPORTED);
                        else expect("no room", backward(a, 16), QTA_ERR_WORKSPACE);
                    }
    if (taken == 0) expect("sizes in range", 0, 1);

    qta_rotary_tensor t{};
    t.x = at(kBase), t.y = at(kBase + 0x10000), t.heads = 4;
    t.x_batch = t.y_batch = 1536, t.x_token = t.y_token = 128, t.x_head = t.y_head = 32;
    const double* const freqs = static_cast<const double*>(at(kBase));
    auto rotary = [&](const qta_rotary_tensor* x, int count, int B, int N, int d, int rot, int axes, int width, int start) {
        return qta_rotary(x, count, B, N, d, rot, axes, width, 0, 0, QTA_F32, freqs, nullptr, 0, start, 1.f, nullptr);
    };
    expect("no tensors", rotary(nullptr, 1, 2, 12, 32, 32, 1, 0, 0), QTA_ERR_INVALID);
    expect("count", rotary(&t, 3, 2, 12, 32, 32, 1, 0, 0), QTA_ERR_INVALID);
    expect("rot", rotary(&t, 1, 2, 12, 32, 31, 1, 0, 0), QTA_ERR_INVALID);
    expect("rot", rotary(&t, 1, 2, 12, 32, INT32_MAX, 1, 0, 0), QTA_ERR_INVALID);
    expect("axes", rotary(&t, 1, 2, 12, 32, 32, 2, 5, 0), QTA_ERR_INVALID);
    expect("start on a map", rotary(&t, 1, 2, 12, 32, 32, 2, 4, 1), QTA_ERR_INVALID);
    for (const int start : {INT32_MIN, INT32_MAX, INT32_MAX - 11}) expect("start", rotary(&t, 1, 2, 12, 32, 32, 1, 0, start), QTA_ERR_INVALID);
    expect("tokens", rotary(&t, 1, INT32_MAX, INT32_MAX, 32, 32, 1, 0, -5), QTA_ERR_UNSUPPORTED);
    expect("d", rotary(&t, 1, 2, 12, INT32_MAX, 32, 1, 0, 0), QTA_ERR_UNSUPPORTED);
    qta_rotary_tensor both[2] = {t, t};
    expect("one place", rotary(both, 2, 2, 12, 32, 32, 1, 0, 0), QTA_ERR_INVALID);
    both[0].heads = both[1].heads = INT32_MAX;
    expect("heads", rotary(both, 2, 2, 12, 32, 32, 1, 0, 0), QTA_ERR_UNSUPPORTED);
    t.x_token = INT64_MIN;
    expect("stride", rotary(&t, 1, 2, 12, 32, 32, 1, 0, 0), QTA_ERR_INVALID);

    std::printf("dense validation: %d failures\n", failures);
    return failures != 0;
}
