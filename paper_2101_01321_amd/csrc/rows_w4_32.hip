// Products with 4-bit weights in groups of 32 values.
#include "rows_launch.h"

namespace ibert {

IBERT_ROWS_UNIT(true, 32)

}  // namespace ibert
