// The host-side paths of layer norm, dropout and log probabilities with fake device addresses.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "layer_internal.h"
#include "mics.h"

namespace mics {
extern int g_layer_launches;
extern Dropout g_dropout;
extern NormBackward g_backward;
}

#define CHECK(cond) do { if (!(cond)) { std::fprintf(stderr, "%s:%d: %s [%s]\n", __FILE__, __LINE__, #cond, mics_last_error()); std::exit(1); } } while (0)

int main()
{
    auto fake = [](size_t i) { return reinterpret_cast<char*>(0x7F0000000000ull + (i << 34)); };
    auto f32 = [&](size_t i) { return reinterpret_cast<float*>(fake(i)); };
    const size_t rows = 100, cols = 1000;
    int n = 0;

    // accepted calls reach their launcher once
    CHECK(mics_layer_norm(fake(0), f32(1), nullptr, fake(2), fake(3), nullptr, rows, cols, nullptr, 1e-5f, 0, 2, nullptr) == MICS_OK);
    CHECK(mics::g_layer_launches == ++n && mics::g_dropout.threshold == 0);
    for (float drop : {0.0f, 0.1f, 0.5f, 0.999999f}) {
        CHECK(mics_bias_dropout_add(fake(0), fake(1), nullptr, nullptr, rows, cols, nullptr, drop, 5, ~0ull, 1, 1, nullptr) == MICS_OK);
        CHECK(mics::g_layer_launches == ++n);
        const mics::Dropout d = mics::g_dropout;
        CHECK(d.threshold == (drop == 0.0f ? 0u : drop == 0.1f ? 6554u : drop == 0.5f ? 32768u : 65535u));
        CHECK(d.scale == (float)(65536.0 / (65536.0 - d.threshold)) && d.seed == 5 && d.offset == ~0ull);
    }
    // the workspace of long rows holds the rows' sums in front
    const size_t tiled = mics::kTiledCols;
    for (size_t c : {cols, tiled, tiled + 1}) {
        const size_t need = mics_column_workspace_bytes(rows, c);
        CHECK(need == 4 * (3 * rows * c + (c > tiled ? 2 * rows : 0)));
        CHECK(mics_layer_norm_backward(fake(0), fake(1), nullptr, fake(2), fake(3), f32(4), f32(5), nullptr, rows, c, nullptr, 0, 0, 0,
                                       fake(6), need, nullptr) == MICS_OK);
        CHECK(mics::g_layer_launches == ++n);
        CHECK((char*)mics::g_backward.parts - fake(6) == (c > tiled ? 8 * (long)rows : 0) && !mics::g_backward.dsum.data);
        CHECK(mics_layer_norm_backward(fake(0), fake(1), nullptr, fake(2), fake(3), f32(4), f32(5), nullptr, rows, c, nullptr, 0, 0, 0,
                                       fake(6), need - 1, nullptr) == MICS_ERR_INVALID_ARG);
    }
    // strides arrive in the order of the matrices
    const size_t strides[5] = {1001, 1002, 1003, 1004, 1005}, need = mics_column_workspace_bytes(rows, cols);
    CHECK(mics_dropout_add_layer_norm_backward(fake(0), fake(1), fake(2), fake(3), fake(4), fake(5), fake(6), fake(7), f32(8), f32(9),
                                               fake(10), rows, cols, strides, 0.1f, 0, 0, 0, 0, 0, fake(11), need, nullptr) == MICS_OK);
    const mics::NormBackward b = mics::g_backward;
    CHECK(++n && b.dx.stride == 1001 && b.dresidual.stride == 1002 && b.dy.stride == 1003 && b.dsum.stride == 1004 && b.x.stride == 1005);
    // matrices that are absent have no stride to check
    const size_t zero[4] = {cols, 0, cols, 0};
    CHECK(mics_dropout_add_layer_norm(fake(0), nullptr, nullptr, nullptr, fake(2), nullptr, nullptr, nullptr, nullptr, rows, cols, zero,
                                      0.f, 0, 0, 0.f, 0, 0, nullptr) == MICS_OK && ++n);
    // no rows: nothing is launched but what writes the parameters' gradients
    CHECK(mics_layer_norm(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, cols, nullptr, 1e-5f, 0, 0, nullptr) == MICS_OK);
    CHECK(mics_bias_dropout_add_backward(nullptr, nullptr, nullptr, 0, cols, nullptr, 0.f, 0, 0, 0, 0, nullptr, 0, nullptr) == MICS_OK);
    CHECK(mics_token_logprobs(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, cols, cols, 5, 0, nullptr, 0, nullptr) == MICS_OK);
    CHECK(mics::g_layer_launches == n);
    CHECK(mics_bias_dropout_add_backward(nullptr, fake(1), nullptr, 0, cols, nullptr, 0.f, 0, 0, 0, 0, nullptr, 0, nullptr) == MICS_OK);
    CHECK(mics::g_layer_launches == ++n);
    // a launch that fails
    int64_t* const ids = (int64_t*)fake(3);
    CHECK(mics_token_logprobs(f32(0), nullptr, nullptr, ids, f32(4), fake(5), (int64_t*)fake(6), rows, cols, cols, 64, 0, nullptr, 0, nullptr)
          == MICS_ERR_HIP && std::strstr(mics_last_error(), "HIP error 77"));
    CHECK(mics_token_logprobs_workspace_bytes(3, cols, 64) == 3 * 4 * (16 + 8 * 64));
    // every count of arguments near the ends of the range
    CHECK(mics_token_logprobs_backward(fake(0), fake(1), (int64_t*)fake(2), f32(3), nullptr, f32(4), nullptr, 1, 1, nullptr, 2, nullptr) == MICS_OK);
    CHECK(mics_layer_norm(fake(0), nullptr, nullptr, fake(0), nullptr, nullptr, SIZE_MAX / 32 / 8, 8, nullptr, 0.f, 2, 2, nullptr) == MICS_OK);
    const size_t wide[2] = {SIZE_MAX / 8, SIZE_MAX / 8};
    CHECK(mics_layer_norm(fake(0), nullptr, nullptr, fake(8), nullptr, nullptr, 2, 8, wide, 0.f, 2, 2, nullptr) == MICS_ERR_INVALID_ARG);
    std::puts("layer host checks ok");
    return 0;
}
