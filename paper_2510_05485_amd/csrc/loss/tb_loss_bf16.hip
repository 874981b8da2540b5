#include "tb_loss_rows.h"

namespace tb {
namespace loss {
template hipError_t rows_of<BF16>(Op, Call&);
template hipError_t gradient_of<BF16>(Op, const Call&);
}  // namespace loss
}  // namespace tb
