// The microscaled product with all slices in a work-group (mx_rules.h).
#include "mx_gemm.h"

bool mx_gemm_all_bf16(const MxArgs& a, int kind) { return mx_launch_all<SSD_MX_OUT_BF16>(a, kind); }
