// octo_op_product's kernels for rows of f16
#define OCTO_PRODUCT_TYPE _Float16
#include "product.h"
