// The training operators for 32-bit numbers.
#include "plain_host.h"

PLAIN_TYPE(, float)
