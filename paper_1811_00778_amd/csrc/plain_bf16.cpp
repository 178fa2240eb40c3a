// The training operators for bfloat16 numbers.
#include "plain_host.h"

PLAIN_TYPE(, Bfloat)
