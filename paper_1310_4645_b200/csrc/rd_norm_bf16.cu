// The norm of rows of bf16 values.
#define RD_NORM_ROWS B16
#include "rd_norm_kernels.h"
