// octo_op_product's kernels for rows of 8 bits
#define OCTO_PRODUCT_TYPE f8
#include "product.h"
