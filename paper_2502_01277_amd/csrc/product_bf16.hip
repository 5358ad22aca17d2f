// octo_op_product's kernels for rows of bf16
#define OCTO_PRODUCT_TYPE __bf16
#include "product.h"
