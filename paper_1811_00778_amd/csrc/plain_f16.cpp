// The training operators for binary16 numbers.
#include "plain_host.h"

PLAIN_TYPE(, Half)
