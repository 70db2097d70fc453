// The norm of rows of fp16 values.
#define RD_NORM_ROWS H16
#include "rd_norm_kernels.h"
