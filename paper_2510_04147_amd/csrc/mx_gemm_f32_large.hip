// Shapes of the microscaled product's kernel (mx_rules.h).
#include "mx_gemm.h"

bool mx_gemm_f32_large(const MxArgs& a, int kind, int* n_part) { return mx_launch_kind<SSD_MX_OUT_F32, 6, 17>(a, kind, n_part); }
