#include "tb_loss_rows.h"

namespace tb {
namespace loss {
template hipError_t rows_of<F32>(Op, Call&);
template hipError_t gradient_of<F32>(Op, const Call&);
}  // namespace loss
}  // namespace tb
