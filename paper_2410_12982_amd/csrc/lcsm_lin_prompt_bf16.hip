// Prompts of linear attention, bf16 queries, keys and values.
#include "lcsm_lin_prompt.h"

namespace lcsm {

hipError_t lin_prompt_bf16(const LinCall& c, const LinCut& w, hipStream_t st) { return lin_prompt<bf16_t>(c, w, st); }

}  // namespace lcsm
