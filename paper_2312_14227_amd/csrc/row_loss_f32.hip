// Row kernels of f32 logits
#include "row_loss.h"

namespace et {
namespace rows {
ET_ROWS_OF(float)
}  // namespace rows
}  // namespace et
