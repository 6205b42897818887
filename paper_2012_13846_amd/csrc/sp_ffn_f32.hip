// The feed-forward block's products in fp32 (v_mfma_f32_16x16x4_f32).
#include "sp_ffn.h"

namespace sp {
template int ffn_fwd<float>(const Ffn& f, hipStream_t s);
template int ffn_bwd<float>(const Ffn& f, hipStream_t s);
}  // namespace sp
