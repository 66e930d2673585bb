// qmm_lora_grad_f16_rows8.cu -- the adapters' weight gradients where dY and B are fp16 and X comes as rows of 8 bits.
#include "qmm_lora.cuh"

namespace qmm {

QMM_LORA_WGRAD_TYPE(f16_rows8, __half, true)

}  // namespace qmm
