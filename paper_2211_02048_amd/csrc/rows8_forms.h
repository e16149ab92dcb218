// Which kernel takes a product of two matrices in 8 bits (one instantiation per file).
#pragma once

#include "rows8_few.h"
#include "rows8_tiles.h"
#include "rows8_waves.h"

namespace sige {

// The forms, also by their numbers through the knob ROWS8_FORM.  Plain: rows x output channels of a workgroup.
enum Linear8Form {
    LINEAR8_FEW = 0,            // 16 x 16, waves share the input channels (up to 8, 512 channels at a time)
    LINEAR8_WAVES_32 = 1,       // 32 x 32, four waves share them
    LINEAR8_WAVES_32X64 = 2,    // 32 x 64
    LINEAR8_WAVES_64 = 3,       // 64 x 64
    LINEAR8_TILE_128X64 = 4,
    LINEAR8_TILE_128 = 5,       // two workgroups per compute unit
    LINEAR8_TILE_128_DEEP = 6,  // one, four blocks on their way
    LINEAR8_TILE_256 = 7,       // (half types)
    LINEAR8_FORMS = 8
};
// Gated: rows x 128 output channels of a workgroup.
enum Linear8GatedForm { GATED8_FEW = 0 /* 16 rows */, GATED8_TILE_64 = 1, GATED8_TILE_128 = 2, GATED8_TILE_256 = 3, GATED8_FORMS = 4 };

int linear8_f32(const char* who, const Linear8Args& a, int rows, int form, hipStream_t st);
int linear8_f16(const char* who, const Linear8Args& a, int rows, int form, hipStream_t st);
int linear8_bf16(const char* who, const Linear8Args& a, int rows, int form, hipStream_t st);
int linear8_gated(const char* who, const Linear8Args& a, int rows, int form, hipStream_t st);

template <typename T>
inline int linear8_launch(const char* who, const Linear8Args& a, int rows, int form, hipStream_t st)
{
    switch (form) {
    case LINEAR8_FEW: return launch_few<T, false, 1, 1, 2>(who, a, rows, 8, st);
    case LINEAR8_WAVES_32: return launch_waves<T, 1, 1, 4, 4>(who, a, rows, st);
    case LINEAR8_WAVES_32X64: return launch_waves<T, 1, 2, 3, 4>(who, a, rows, st);
    case LINEAR8_WAVES_64: return launch_waves<T, 2, 2, 2, 4>(who, a, rows, st);
    case LINEAR8_TILE_128X64: return launch_tiles<T, false, 2, 1, 3, 2>(who, a, rows, st);
    case LINEAR8_TILE_128: return launch_tiles<T, false, 2, 2, 2, 2>(who, a, rows, st);
    case LINEAR8_TILE_128_DEEP: return launch_tiles<T, false, 2, 2, 4, 1>(who, a, rows, st);
    case LINEAR8_TILE_256:
        if constexpr (sizeof(T) == 2) return launch_tiles<T, false, 4, 4, 2, 1, true>(who, a, rows, st);
    }
    return fail(SIGE_ERR_UNSUPPORTED, "%s: the call has no form %d", who, form);
}

}  // namespace sige
