// Prompts of the state space mixer, activations of this type.
#include "lcsm_ssm_prompt.h"

namespace lcsm {

hipError_t ssm_prompt_f32(const SsmCall& c, const SsmScratch& w, hipStream_t st) {
  return ssm_prompt<float>(c, w, st);
}

}  // namespace lcsm
