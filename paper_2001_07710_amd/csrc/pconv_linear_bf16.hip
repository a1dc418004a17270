// The matrix products of pconv_linear_kernels.h for bf16 storage.
#define PCONV_LINEAR_DT PCONV_BF16
#include "pconv_linear_kernels.h"

namespace pconv {
int launch_product_bf16(const Product& p, void* stream) { return launch_product(p, stream); }
int launch_few_rows_bf16(const Product& p, void* stream) { return launch_few_rows(p, stream); }
}  // namespace pconv
