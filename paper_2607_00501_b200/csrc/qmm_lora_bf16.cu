// qmm_lora_bf16.cu -- the adapters on bf16 rows.
#include "qmm_lora.cuh"

namespace qmm {

QMM_LORA_TYPE(bf16, __nv_bfloat16)

}  // namespace qmm
