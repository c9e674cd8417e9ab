// Stand-ins for the launchers of linear.hip and activation.hip: they record what they were asked for and touch no pointer.
#include "linear_internal.h"

namespace mics {
int g_linear_launches = 0, g_linear_answer = 0;
Product g_product;
ProductPlan g_plan;
ActivationPass g_activation;
CheckpointRead g_read;
ActivationBackward g_activation_backward;
int launch_product(const Product& p, const ProductPlan& plan, int, void*) { g_product = p; g_plan = plan; ++g_linear_launches; return g_linear_answer; }
int launch_activation(const ActivationPass& a, int, void*) { g_activation = a; ++g_linear_launches; return g_linear_answer; }
int launch_checkpoint_read(const CheckpointRead& a, int, void*) { g_read = a; ++g_linear_launches; return g_linear_answer; }
int launch_activation_backward(const ActivationBackward& a, int, void*, int, void*) { g_activation_backward = a; ++g_linear_launches; return g_linear_answer; }
}  // namespace mics
