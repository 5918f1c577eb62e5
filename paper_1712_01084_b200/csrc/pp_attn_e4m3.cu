// The attention kernels of e4m3 caches (pp_attn.cuh).
#include "pp_attn.cuh"

namespace pp {
namespace attn {

Form form_e4m3(Reading reading, pp_dtype_t q_type, int dim, bool two) { return mma_form8<kE4m3>(reading, q_type, dim, two); }

}  // namespace attn
}  // namespace pp
