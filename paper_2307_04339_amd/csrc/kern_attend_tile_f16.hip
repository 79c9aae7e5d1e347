// Attention for tiles of query rows, f16.
#include "attend_tile.h"

namespace miriam {
int attend_tile_kernels_f16(int d, bool uni, const void *out[3], int *lds) {
    switch ((d + 31) / 32 * 32) {
    case 32:
    case 64: tile_table<half_t, 64>(uni, out, lds); return 0;
    case 96: tile_table<half_t, 128, 96>(uni, out, lds); return 0;
    case 128: tile_table<half_t, 128>(uni, out, lds); return 0;
    case 160:
    case 192:
    case 224:
    case 256: tile_table<half_t, 256>(uni, out, lds); return 0;
    default: return -1;
    }
}
}  // namespace miriam
