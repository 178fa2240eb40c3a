// The operators along rows and the microscaled products for bfloat16 numbers.
#include "plain_rows_host.h"

PLAIN_ROWS_TYPE(, Bfloat)
