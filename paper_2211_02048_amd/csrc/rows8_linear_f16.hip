// The products of two matrices in 8 bits with results in fp16.
#include "rows8_forms.h"

namespace sige {
int linear8_f16(const char* who, const Linear8Args& a, int rows, int form, hipStream_t st) { return linear8_launch<f16>(who, a, rows, form, st); }
}  // namespace sige
