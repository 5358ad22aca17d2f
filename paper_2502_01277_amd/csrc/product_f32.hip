// octo_op_product's kernels for rows of f32
#define OCTO_PRODUCT_TYPE float
#include "product.h"
