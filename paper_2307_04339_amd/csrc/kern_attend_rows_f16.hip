// Attention for few query rows, f16.
#include "attend_rows.h"

namespace miriam {
int attend_rows_kernels_f16(int dp, const void *out[3], int *lds) {
    switch (dp) {
    case 64: rows_table<half_t, 64>(out, lds); return 0;
    case 128: rows_table<half_t, 128>(out, lds); return 0;
    case 256: rows_table<half_t, 256>(out, lds); return 0;
    default: return -1;
    }
}
}  // namespace miriam
