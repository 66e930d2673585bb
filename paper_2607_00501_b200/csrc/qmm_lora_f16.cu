// qmm_lora_f16.cu -- the adapters on f16 rows.
#include "qmm_lora.cuh"

namespace qmm {

QMM_LORA_TYPE(f16, __half)

}  // namespace qmm
