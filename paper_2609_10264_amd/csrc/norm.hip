// block_norm (norm.h) of rows of whole chunks of eight values, and which form a call takes.
#include "norm.h"

namespace mvk {

hipError_t launch_block_norm(const NormArgs& a, hipStream_t s) {
    if (a.n % 8) return launch_block_norm_ragged(a, s);
    if (a.out.p && a.out.type == MVK_TYPE_FIELD) return launch_norm_in<double, true>(a, s);
    return launch_norm_in<float, true>(a, s);
}

}  // namespace mvk
