// Row kernels of bf16 logits
#include "row_loss.h"

namespace et {
namespace rows {
ET_ROWS_OF(bf16)
}  // namespace rows
}  // namespace et
