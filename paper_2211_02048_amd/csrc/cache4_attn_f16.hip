// The attention on the cache held in 4 bits, f16 queries (one storage type per file: they compile side by side).
#include "cache4_attn.h"

namespace sige {
int launch_cache4_f16(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st) { return launch_cache4<f16>(a, f, st); }
}  // namespace sige
