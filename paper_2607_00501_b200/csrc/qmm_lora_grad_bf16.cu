// qmm_lora_grad_bf16.cu -- the adapters' weight gradients on bf16 rows.
#include "qmm_lora.cuh"

namespace qmm {

QMM_LORA_WGRAD_TYPE(bf16, __nv_bfloat16, false)
QMM_LORA_JOIN

}  // namespace qmm
