#include "lp_linear_back.h"

namespace lp {
namespace linear {

hipError_t launch_back_bf16_any(int act, const BackDev& d, const Parts& p, bool skinny, hipStream_t s) { return launch_back<__bf16, false>(act, d, p, skinny, s); }

}  // namespace linear
}  // namespace lp
