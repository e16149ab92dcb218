// The products of two matrices in 8 bits with the gated activation behind them.
#include "rows8_forms.h"

namespace sige {

int linear8_gated(const char* who, const Linear8Args& a, int rows, int form, hipStream_t st)
{
    switch (form) {
    case GATED8_FEW: return launch_few<bf16, true, 1, 2, 2>(who, a, rows, 8, st);
    case GATED8_TILE_64: return launch_tiles<bf16, true, 1, 4, 3, 1>(who, a, rows, st);
    case GATED8_TILE_128: return launch_tiles<bf16, true, 2, 4, 2, 1>(who, a, rows, st);
    case GATED8_TILE_256: return launch_tiles<bf16, true, 4, 4, 2, 1, true>(who, a, rows, st);
    }
    return fail(SIGE_ERR_UNSUPPORTED, "%s: the call has no form %d", who, form);
}

}  // namespace sige
