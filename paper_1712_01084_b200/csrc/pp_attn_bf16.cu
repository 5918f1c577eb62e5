// The attention kernels of bf16 caches (pp_attn.cuh).
#include "pp_attn.cuh"

namespace pp {
namespace attn {

Form form_bf16(Reading reading, int dim, bool two) { return mma_form<kBf16, true, 1>(reading, dim, two); }

}  // namespace attn
}  // namespace pp
