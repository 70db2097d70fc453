// The norm of rows of fp32 values.
#define RD_NORM_ROWS F32
#include "rd_norm_kernels.h"
