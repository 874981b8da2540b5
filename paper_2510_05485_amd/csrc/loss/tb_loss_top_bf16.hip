#include "tb_loss_top.h"

namespace tb {
namespace loss {
template hipError_t top_of<BF16>(const TopCall&);
template hipError_t top_gradient_of<BF16>(const TopCall&);
}  // namespace loss
}  // namespace tb
