// Products with 4-bit weights in groups of 64 values.
#include "rows_launch.h"

namespace ibert {

IBERT_ROWS_UNIT(true, 64)

}  // namespace ibert
