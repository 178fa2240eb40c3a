// The operators along rows and the microscaled products for 32-bit numbers.
#include "plain_rows_host.h"

PLAIN_ROWS_TYPE(, float)
