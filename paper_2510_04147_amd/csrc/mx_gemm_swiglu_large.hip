// Shapes of the microscaled product's kernel (mx_rules.h).
#include "mx_gemm.h"

bool mx_gemm_swiglu_large(const MxArgs& a, int kind, int* n_part) { return mx_launch_kind<SSD_MX_OUT_SWIGLU, 13, 17>(a, kind, n_part); }
