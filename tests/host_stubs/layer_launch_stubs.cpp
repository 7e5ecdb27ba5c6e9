// Stand-ins for the kernel launchers of the layer operators, for the host-only sanitizer build of their argument checks (csrc/layers_api.hip).
#include "layers_internal.h"

namespace ssmv {
int launch_block_norm(const BlockNormParams &, hipStream_t) { return 0; }
int launch_block_norm_backward(const BlockNormGradParams &, hipStream_t) { return 0; }
int launch_gated_recurrence(const GatedParams &, hipStream_t) { return 0; }
int launch_gated_backward(const GatedGradParams &, hipStream_t) { return 0; }
int launch_logit_rules(const RulesParams &, hipStream_t) { return 0; }
}  // namespace ssmv
