// The dense products' kernels for rows of __bf16.
#include "spdnn_linear_typed.h"

SPDNN_LINEAR_LAUNCHES(__bf16)
