// The microscaled product with all slices in a work-group (mx_rules.h).
#include "mx_gemm.h"

bool mx_gemm_all(const MxArgs& a, int kind, int result) {
    int parts;
#define MX_ALL_CASE(id, tm, kc, nst, ...)                                                                                             \
    if (kind == id) return result == SSD_MX_OUT_F32 ? mx_launch_shape<1, 1, 1, tm, kc, nst, SSD_MX_OUT_F32, false, true, true>(a, &parts)   \
                                                    : mx_launch_shape<1, 1, 1, tm, kc, nst, SSD_MX_OUT_BF16, false, true, true>(a, &parts);
    MX_ALL_KINDS(MX_ALL_CASE)
#undef MX_ALL_CASE
    return false;
}
