// The attention kernels of float caches, and of caches that are read element by element (pp_attn.cuh).
#include "pp_attn.cuh"

namespace pp {
namespace attn {

Form form_scalar(Reading reading, int dim, int group) {
    return reading == kWhole ? scalar_form<kWhole>(dim, group) : reading == kRows ? scalar_form<kRows>(dim, group) : scalar_form<kElements>(dim, group);
}

}  // namespace attn
}  // namespace pp
