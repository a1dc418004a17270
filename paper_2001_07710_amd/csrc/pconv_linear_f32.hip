// The matrix products of pconv_linear_kernels.h for f32 storage.
#define PCONV_LINEAR_DT PCONV_F32
#include "pconv_linear_kernels.h"

namespace pconv {
int launch_product_f32(const Product& p, void* stream) { return launch_product(p, stream); }
int launch_few_rows_f32(const Product& p, void* stream) { return launch_few_rows(p, stream); }
}  // namespace pconv
