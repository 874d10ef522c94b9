// Shapes of the microscaled product's kernel (mx_rules.h).
#include "mx_gemm.h"

bool mx_gemm_bf16(const MxArgs& a, int kind, int* n_part) { return mx_launch_kind<SSD_MX_OUT_BF16, 0, 5>(a, kind, n_part); }
