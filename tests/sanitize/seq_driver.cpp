// Drives the C-ABI layer of the sequence operators (mfpsn_api_seq.cpp, built
// with AddressSanitizer and UndefinedBehaviorSanitizer), the GPU launchers
// replaced by counting stubs: invalid arguments must return the documented
// status and launch nothing, sizes at the limits must validate without
// overflow.  Test infrastructure only.  Prints "seq driver: OK".
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "mfpsn.h"
#include "mfpsn_delta.h"
#include "mfpsn_norm.h"

static long launches = 0;
static mfpsn::DeltaArgs last;
static int steps_launched = 0;

namespace mfpsn {
hipError_t launch_norm_forward(const NormArgs&, int, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_norm_backward(const NormArgs&, int, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_delta_forward(const DeltaArgs& a, int, hipStream_t) { ++launches; last = a; steps_launched = 0; return hipSuccess; }
hipError_t launch_delta_backward(const DeltaArgs& a, int, hipStream_t) { ++launches; last = a; return hipSuccess; }
hipError_t launch_delta_steps(const DeltaArgs& a, int, hipStream_t) { ++launches; last = a; steps_launched = 1; return hipSuccess; }
}  // namespace mfpsn

static int failures = 0;
static void expect(int line, int got, int want, long before)
{
    if (got != want || (want != MFPSN_OK && launches != before)) {
        fprintf(stderr, "line %d: status %d, expected %d, %ld launches\n", line, got, want, launches - before);
        ++failures;
    }
}
#define EXPECT(call, want)                        \
    do {                                          \
        const long before = launches;             \
        expect(__LINE__, (call), (want), before); \
    } while (0)
#define CHECK(cond)                                                      \
    do {                                                                 \
        if (!(cond)) {                                                   \
            fprintf(stderr, "line %d: %s is false\n", __LINE__, #cond);  \
            ++failures;                                                  \
        }                                                                \
    } while (0)

static mfpsn_delta_desc desc(int T, int N, int Hk, int Hv, int Dk, int Dv, int dtype)
{
    mfpsn_delta_desc d;
    memset(&d, 0, sizeof d);
    d.T = T;
    d.N = N;
    d.Hk = Hk;
    d.Hv = Hv;
    d.Dk = Dk;
    d.Dv = Dv;
    d.dtype = dtype;
    d.scale = 0.25f;
    return d;
}

int main()
{
    void* p = (void*)0x10000;
    void* odd = (void*)0x10001;
    float* f = (float*)p;
    float* fodd = (float*)0x10002;
    size_t n = 0;
    // layer norm
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, p, f, f, 1e-5f, p, f, f, nullptr), MFPSN_OK);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, p, nullptr, nullptr, 0.0f, p, nullptr, nullptr, nullptr), MFPSN_OK);
    EXPECT(mfpsn_layer_norm_forward(-1, 5, 6, MFPSN_F32, p, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_SHAPE);
    EXPECT(mfpsn_layer_norm_forward(4, -5, 6, MFPSN_F32, p, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_SHAPE);
    EXPECT(mfpsn_layer_norm_forward(INT64_MAX, INT32_MAX, INT32_MAX, MFPSN_F32, p, f, f, 1e-5f, p, f, f, nullptr),
           MFPSN_ERR_SHAPE);
    EXPECT(mfpsn_layer_norm_forward(INT64_MAX, 1, 1, MFPSN_F32, p, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_SHAPE);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_Q8_8, p, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_DTYPE);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, 9, p, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_DTYPE);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, p, f, f, -1e-5f, p, f, f, nullptr), MFPSN_ERR_PARAM);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, p, f, f, NAN, p, f, f, nullptr), MFPSN_ERR_PARAM);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, nullptr, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_NULL);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, p, f, f, 1e-5f, p, f, nullptr, nullptr), MFPSN_ERR_NULL);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, fodd, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_ALIGN);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_BF16, fodd, f, f, 1e-5f, p, f, f, nullptr), MFPSN_OK);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_BF16, odd, f, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_ALIGN);
    EXPECT(mfpsn_layer_norm_forward(4, 5, 6, MFPSN_F32, p, fodd, f, 1e-5f, p, f, f, nullptr), MFPSN_ERR_ALIGN);
    long before = launches;
    EXPECT(mfpsn_layer_norm_forward(0, 5, 6, MFPSN_F32, nullptr, nullptr, nullptr, 1e-5f, nullptr, nullptr, nullptr, nullptr),
           MFPSN_OK);
    CHECK(launches == before);
    EXPECT(mfpsn_layer_norm_workspace_size(4, 5, 6, nullptr), MFPSN_ERR_NULL);
    EXPECT(mfpsn_layer_norm_workspace_size(4, 5, -6, &n), MFPSN_ERR_SHAPE);
    EXPECT(mfpsn_layer_norm_workspace_size(1 << 30, 1000, 1, &n), MFPSN_OK);
    CHECK(n == (size_t)mfpsn::norm_blocks(1 << 30, 1000, 1) * 2 * 1000 * 4 && n <= (size_t)mfpsn::kNormMaxBlocks * 8000);
    EXPECT(mfpsn_layer_norm_workspace_size(4, 5, 6, &n), MFPSN_OK);
    const auto bwd = [&](const void* x, float* gg, void* ws, size_t bytes) {
        return mfpsn_layer_norm_backward(4, 5, 6, MFPSN_F32, x, f, f, f, p, p, gg, nullptr, ws, bytes, nullptr);
    };
    EXPECT(bwd(p, f, p, n), MFPSN_OK);
    EXPECT(bwd(p, nullptr, nullptr, 0), MFPSN_OK);
    EXPECT(bwd(p, f, p, n - 4), MFPSN_ERR_WORKSPACE);
    EXPECT(bwd(p, f, nullptr, n), MFPSN_ERR_WORKSPACE);
    EXPECT(bwd(p, f, fodd, n), MFPSN_ERR_WORKSPACE);
    EXPECT(bwd(nullptr, f, p, n), MFPSN_ERR_NULL);
    EXPECT(bwd(fodd, f, p, n), MFPSN_ERR_ALIGN);
    // gated delta rule
    const mfpsn_delta_desc good = desc(100, 3, 2, 4, 64, 48, MFPSN_BF16);
    EXPECT(mfpsn_delta_workspace_size(nullptr, &n), MFPSN_ERR_NULL);
    EXPECT(mfpsn_delta_workspace_size(&good, nullptr), MFPSN_ERR_NULL);
    const int bad[][6] = {{-1, 1, 1, 1, 1, 1}, {1, -1, 1, 1, 1, 1}, {1, 1, 0, 1, 1, 1}, {1, 1, 2, 3, 1, 1},
                          {1, 1, 1, 0, 1, 1}, {1, 1, 1, 1, 0, 1}, {1, 1, 1, 1, 129, 1}, {1, 1, 1, 1, 1, 0},
                          {1, 1, 1, 1, 1, 257}, {INT32_MAX, INT32_MAX, 1, 1, 1, 1}, {1, INT32_MAX, 1, INT32_MAX, 1, 256}};
    for (const auto& b : bad) {
        const mfpsn_delta_desc d = desc(b[0], b[1], b[2], b[3], b[4], b[5], MFPSN_F32);
        EXPECT(mfpsn_delta_workspace_size(&d, &n), MFPSN_ERR_SHAPE);
        EXPECT(mfpsn_delta_saved_size(&d, &n), MFPSN_ERR_SHAPE);
        EXPECT(mfpsn_delta_backward_workspace_size(&d, &n), MFPSN_ERR_SHAPE);
    }
    mfpsn_delta_desc d = good;
    d.dtype = MFPSN_Q8_8;
    EXPECT(mfpsn_delta_workspace_size(&d, &n), MFPSN_ERR_DTYPE);
    d = good;
    d.scale = INFINITY;
    EXPECT(mfpsn_delta_workspace_size(&d, &n), MFPSN_ERR_PARAM);
    d = good;
    d.q_row = 127;  // less than a row of 2 x 64
    EXPECT(mfpsn_delta_workspace_size(&d, &n), MFPSN_ERR_SHAPE);
    d = good;
    d.v_row = INT64_MAX;
    EXPECT(mfpsn_delta_workspace_size(&d, &n), MFPSN_ERR_SHAPE);
    d = desc(INT32_MAX, 1, 1, 1, 128, 256, MFPSN_F32);  // the longest: sizes past 32 bits
    size_t a = 0, b = 0, c = 0;
    EXPECT(mfpsn_delta_workspace_size(&d, &a), MFPSN_OK);
    EXPECT(mfpsn_delta_saved_size(&d, &b), MFPSN_OK);
    EXPECT(mfpsn_delta_backward_workspace_size(&d, &c), MFPSN_OK);
    CHECK(a > ((size_t)1 << 32) && b > a && c > ((size_t)1 << 32));
    EXPECT(mfpsn_delta_workspace_size(&good, &a), MFPSN_OK);
    EXPECT(mfpsn_delta_saved_size(&good, &b), MFPSN_OK);
    EXPECT(mfpsn_delta_backward_workspace_size(&good, &c), MFPSN_OK);
    const auto fwd = [&](const mfpsn_delta_desc* x, const void* q, void* o, void* saved, size_t sb, void* ws, size_t wb) {
        return mfpsn_delta_forward(x, q, p, p, p, p, nullptr, nullptr, o, f, saved, sb, ws, wb, nullptr);
    };
    EXPECT(fwd(&good, p, p, nullptr, 0, p, a), MFPSN_OK);
    CHECK(!steps_launched && last.S0 == nullptr && last.U == nullptr && last.vec_qk && last.q_row == 128 && last.v_row == 192);
    EXPECT(fwd(&good, p, p, p, b, nullptr, 0), MFPSN_OK);
    CHECK(last.S0 && last.U && (char*)last.S0 + c <= (char*)p + b);
    EXPECT(fwd(&good, fodd, p, nullptr, 0, p, a), MFPSN_OK);
    CHECK(!last.vec_qk);  // rows that start at no 16 bytes
    EXPECT(fwd(&good, p, p, nullptr, 0, p, a - 1), MFPSN_ERR_WORKSPACE);
    EXPECT(fwd(&good, p, p, nullptr, 0, nullptr, a), MFPSN_ERR_WORKSPACE);
    EXPECT(fwd(&good, p, p, nullptr, 0, (char*)p + 8, a), MFPSN_ERR_WORKSPACE);
    EXPECT(fwd(&good, p, p, p, b - 1, p, a), MFPSN_ERR_WORKSPACE);
    EXPECT(fwd(&good, nullptr, p, nullptr, 0, p, a), MFPSN_ERR_NULL);
    EXPECT(fwd(&good, p, nullptr, nullptr, 0, p, a), MFPSN_ERR_NULL);
    EXPECT(fwd(&good, odd, p, nullptr, 0, p, a), MFPSN_ERR_ALIGN);
    EXPECT(fwd(nullptr, p, p, nullptr, 0, p, a), MFPSN_ERR_NULL);
    d = good;
    d.N = 0;
    before = launches;
    EXPECT(mfpsn_delta_forward(&d, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                               0, nullptr, 0, nullptr),
           MFPSN_OK);
    CHECK(launches == before);
    d = good;
    d.T = 1;
    EXPECT(mfpsn_delta_workspace_size(&d, &n), MFPSN_OK);
    CHECK(n == 0);
    EXPECT(fwd(&d, p, p, nullptr, 0, nullptr, 0), MFPSN_OK);
    CHECK(steps_launched);
    const auto back = [&](const void* go, void* gk, const void* saved, size_t sb, void* ws, size_t wb) {
        return mfpsn_delta_backward(&good, p, p, p, p, p, nullptr, saved, sb, go, nullptr, p, gk, p, p, p, nullptr, ws, wb,
                                    nullptr);
    };
    EXPECT(back(p, p, p, b, p, c), MFPSN_OK);
    EXPECT(back(nullptr, p, p, b, p, c), MFPSN_ERR_NULL);
    EXPECT(back(p, nullptr, p, b, p, c), MFPSN_ERR_NULL);
    EXPECT(back(p, odd, p, b, p, c), MFPSN_ERR_ALIGN);
    EXPECT(back(p, p, p, b - 1, p, c), MFPSN_ERR_WORKSPACE);
    EXPECT(back(p, p, p, b, p, c - 1), MFPSN_ERR_WORKSPACE);
    EXPECT(back(p, p, nullptr, b, p, c), MFPSN_ERR_WORKSPACE);
    EXPECT(back(p, p, p, b, fodd, c), MFPSN_ERR_WORKSPACE);
    EXPECT(mfpsn_delta_step(nullptr, p, p, p, p, p, f, p, f, nullptr), MFPSN_ERR_NULL);
    d = good;
    d.T = -7;  // ignored
    EXPECT(mfpsn_delta_step(&d, p, p, p, p, p, f, p, f, nullptr), MFPSN_OK);
    CHECK(last.T == 1 && steps_launched);
    EXPECT(mfpsn_delta_step(&d, p, p, p, p, p, nullptr, p, f, nullptr), MFPSN_OK);
    EXPECT(mfpsn_delta_step(&d, p, p, p, p, p, f, p, nullptr, nullptr), MFPSN_ERR_NULL);
    EXPECT(mfpsn_delta_step(&d, p, p, p, p, p, fodd, p, f, nullptr), MFPSN_ERR_ALIGN);
    EXPECT(mfpsn_delta_step(&d, p, p, odd, p, p, f, p, f, nullptr), MFPSN_ERR_ALIGN);
    if (failures == 0)
        printf("seq driver: OK\n");
    return failures != 0;
}
