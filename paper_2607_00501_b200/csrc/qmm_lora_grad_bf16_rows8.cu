// qmm_lora_grad_bf16_rows8.cu -- the adapters' weight gradients where dY and B are bf16 and X comes as rows of 8 bits.
#include "qmm_lora.cuh"

namespace qmm {

QMM_LORA_WGRAD_TYPE(bf16_rows8, __nv_bfloat16, true)

}  // namespace qmm
