// The host-side paths of the linear layer and of activations with fake device addresses.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "linear_internal.h"
#include "mics.h"

namespace mics {
extern int g_linear_launches, g_linear_answer;
extern Product g_product;
extern ProductPlan g_plan;
extern ActivationPass g_activation;
extern CheckpointRead g_read;
extern ActivationBackward g_activation_backward;
}

#define CHECK(cond) do { if (!(cond)) { std::fprintf(stderr, "%s:%d: %s [%s]\n", __FILE__, __LINE__, #cond, mics_last_error()); std::exit(1); } } while (0)

int main()
{
    auto fake = [](size_t i) { return reinterpret_cast<char*>(0x7F0000000000ull + (i << 34)); };
    auto f32 = [&](size_t i) { return reinterpret_cast<float*>(fake(i)); };
    auto i8 = [&](size_t i) { return reinterpret_cast<int8_t*>(fake(i)); };
    const size_t rows = 100, in = 1000, outs = 520, most = MICS_LINEAR_MOST_WORKSPACE;
    int n = 0;

    // strides arrive in the order of the matrices, every product in its form
    const size_t six[6] = {521, 522, 523, 1001, 1002, 524}, four[4] = {1001, 521, 1002, 1003}, three[3] = {1001, 521, 1002};
    CHECK(mics_linear(fake(0), fake(1), i8(2), f32(3), fake(4), fake(5), fake(6), fake(7), rows, in, outs, six, MICS_ACT_GELU, 0, 2, fake(8), most,
                      nullptr) == MICS_OK && mics::g_linear_launches == ++n);
    mics::Product p = mics::g_product;
    CHECK(p.e.out.stride == 521 && p.e.pre.stride == 522 && p.e.codes.stride == 523 && p.a.stride == 1001 && p.b.stride == 1002 && p.e.residual.stride == 524);
    CHECK(p.m == rows && p.n == outs && p.k == in && !p.a_turned && !p.b_turned && p.e.act == MICS_ACT_GELU && p.e.param == 2 && p.e.out_kind == 0);
    CHECK(mics_linear_backward_input(fake(0), fake(1), fake(2), fake(3), rows, in, outs, four, 1, fake(8), most, nullptr) == MICS_OK && mics::g_linear_launches == ++n);
    p = mics::g_product;
    CHECK(p.e.out.stride == 1001 && p.a.stride == 521 && p.b.stride == 1002 && p.e.residual.stride == 1003 && p.m == rows && p.n == in && p.k == outs);
    CHECK(!p.a_turned && p.b_turned && p.e.act == 0 && !p.e.codes.data && !p.e.bias);
    CHECK(mics_linear_backward_weight(fake(0), fake(1), fake(2), rows, in, outs, three, 1, 2, fake(8), most, nullptr) == MICS_OK && mics::g_linear_launches == ++n);
    p = mics::g_product;
    CHECK(p.e.out.stride == 1001 && p.a.stride == 521 && p.b.stride == 1002 && p.m == outs && p.n == in && p.k == rows && p.a_turned && p.b_turned && p.e.out_kind == 2);

    // what a call needs is what its plan takes, and no more than is said beforehand
    for (size_t r : {1, 20, 33, 300, 5000})
        for (size_t skew : {0, 2}) {
            const size_t said = mics_linear_workspace_bytes(r, in, outs);
            CHECK(mics_linear(fake(0), nullptr, nullptr, nullptr, fake(4) + skew, fake(5), nullptr, nullptr, r, in, outs, nullptr, 0, 0, 0, fake(8), said,
                              nullptr) == MICS_OK && mics::g_linear_launches == ++n);
            const size_t need = mics::workspace_of(mics::g_plan);
            CHECK(need <= said);
            if (need)
                CHECK(mics_linear(fake(0), nullptr, nullptr, nullptr, fake(4) + skew, fake(5), nullptr, nullptr, r, in, outs, nullptr, 0, 0, 0, fake(8),
                                  need - 1, nullptr) == MICS_ERR_INVALID_ARG && std::strstr(mics_last_error(), "workspace_bytes"));
        }

    // activations
    const size_t acts[4] = {1001, 1002, 1003, 1004};
    CHECK(mics_activation(fake(0), i8(1), f32(2), fake(3), fake(4), rows, in, acts, MICS_ACT_SILU, 0, 1, nullptr) == MICS_OK && mics::g_linear_launches == ++n);
    CHECK(mics::g_activation.e.out.stride == 1001 && mics::g_activation.e.codes.stride == 1002 && mics::g_activation.x.stride == 1003 && mics::g_activation.e.param == 1);
    CHECK(mics_checkpoint_read(fake(0), i8(1), f32(2), rows, in, acts, MICS_ACT_RELU, 2, nullptr) == MICS_OK && mics::g_linear_launches == ++n);
    CHECK(mics::g_read.y.stride == 1001 && mics::g_read.codes.stride == 1002 && mics::g_read.act == MICS_ACT_RELU);
    const size_t need = mics_column_workspace_bytes(rows, in);
    CHECK(mics_activation_backward(fake(0), fake(1), fake(2), nullptr, i8(3), f32(4), rows, in, acts, 2, 0, 2, fake(5), need, nullptr) == MICS_OK && mics::g_linear_launches == ++n);
    CHECK(mics::g_activation_backward.dx.stride == 1001 && mics::g_activation_backward.dy.stride == 1002 && mics::g_activation_backward.codes.stride == 1004);

    // no rows: nothing is launched but what writes gradients of parameters
    CHECK(mics_linear(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, in, outs, nullptr, 0, 0, 0, nullptr, 0, nullptr) == MICS_OK);
    CHECK(mics_linear_backward_input(nullptr, nullptr, nullptr, nullptr, 0, in, outs, nullptr, 0, nullptr, 0, nullptr) == MICS_OK);
    CHECK(mics_activation(nullptr, nullptr, nullptr, nullptr, nullptr, 0, in, nullptr, 0, 0, 0, nullptr) == MICS_OK);
    CHECK(mics_checkpoint_read(nullptr, nullptr, nullptr, 0, in, nullptr, 0, 0, nullptr) == MICS_OK);
    CHECK(mics_activation_backward(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0, in, nullptr, 0, 0, 0, nullptr, 0, nullptr) == MICS_OK);
    CHECK(mics::g_linear_launches == n);
    CHECK(mics_linear_backward_weight(fake(0), nullptr, nullptr, 0, in, outs, nullptr, 0, 0, nullptr, 0, nullptr) == MICS_OK && mics::g_linear_launches == ++n);
    CHECK(mics_activation_backward(nullptr, fake(1), nullptr, nullptr, nullptr, nullptr, 0, in, nullptr, 0, 0, 0, nullptr, 0, nullptr) == MICS_OK && mics::g_linear_launches == ++n);

    // a launch that fails; sizes near the ends of the range
    mics::g_linear_answer = 77;
    CHECK(mics_checkpoint_read(fake(0), i8(1), f32(2), rows, in, nullptr, 0, 0, nullptr) == MICS_ERR_HIP && std::strstr(mics_last_error(), "HIP error 77"));
    mics::g_linear_answer = 0;
    CHECK(mics_linear(fake(0), nullptr, nullptr, nullptr, fake(1), fake(2), nullptr, nullptr, SIZE_MAX / 32 / 8, 8, 8, nullptr, 0, 2, 2, fake(3), most, nullptr)
          == MICS_ERR_INVALID_ARG);        // such a matrix reaches into the next one
    CHECK(mics_linear(fake(0), nullptr, nullptr, nullptr, (void*)16, fake(0) - 64, nullptr, nullptr, size_t{1} << 40, 1, 1, nullptr, 0, 2, 2, fake(3), most, nullptr) != MICS_OK);
    CHECK(mics_linear_workspace_bytes(SIZE_MAX / 32 / 8, 8, 8) <= most);
    std::puts("linear host checks ok");
    return 0;
}
