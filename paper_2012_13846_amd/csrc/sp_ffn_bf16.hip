// The feed-forward block's products in bf16 (v_mfma_f32_16x16x32_bf16).
#include "sp_ffn.h"

namespace sp {
template int ffn_fwd<bf16_t>(const Ffn& f, hipStream_t s);
template int ffn_bwd<bf16_t>(const Ffn& f, hipStream_t s);
}  // namespace sp
