// mx_attn_decode with MX9 keys (the kernels are in mx_attn_decode.cuh; one file per key format so that they compile side by side).
#include "mx_attn_decode.cuh"

namespace bdr {
BDR_ATTN_KEY_FORMAT(8)
}  // namespace bdr
