// The dense products' kernels for rows of _Float16.
#include "spdnn_linear_typed.h"

SPDNN_LINEAR_LAUNCHES(_Float16)
