// qmm_lora_grad_f16.cu -- the adapters' weight gradients on f16 rows.
#include "qmm_lora.cuh"

namespace qmm {

QMM_LORA_WGRAD_TYPE(f16, __half, false)

}  // namespace qmm
