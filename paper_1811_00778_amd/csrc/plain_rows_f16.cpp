// The operators along rows and the microscaled products for binary16 numbers.
#include "plain_rows_host.h"

PLAIN_ROWS_TYPE(, Half)
