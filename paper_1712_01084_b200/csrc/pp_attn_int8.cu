// The attention kernels of 8-bit integer caches (pp_attn.cuh).
#include "pp_attn.cuh"

namespace pp {
namespace attn {

Form form_int8(Reading reading, pp_dtype_t q_type, int dim, bool two) { return mma_form8<kInt8>(reading, q_type, dim, two); }

}  // namespace attn
}  // namespace pp
