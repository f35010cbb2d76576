// The dense products' kernels for rows of float.
#include "spdnn_linear_typed.h"

SPDNN_LINEAR_LAUNCHES(float)
