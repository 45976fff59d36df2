// Prompts of linear attention, fp32 queries, keys and values.
#include "lcsm_lin_prompt.h"

namespace lcsm {

hipError_t lin_prompt_f32(const LinCall& c, const LinCut& w, hipStream_t st) { return lin_prompt<float>(c, w, st); }

}  // namespace lcsm
