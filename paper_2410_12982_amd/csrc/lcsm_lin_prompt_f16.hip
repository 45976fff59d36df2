// Prompts of linear attention, fp16 queries, keys and values.
#include "lcsm_lin_prompt.h"

namespace lcsm {

hipError_t lin_prompt_f16(const LinCall& c, const LinCut& w, hipStream_t st) { return lin_prompt<f16_t>(c, w, st); }

}  // namespace lcsm
