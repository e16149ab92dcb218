// The attention on the cache held in 4 bits, f32 queries (one storage type per file: they compile side by side).
#include "cache4_attn.h"

namespace sige {
int launch_cache4_f32(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st) { return launch_cache4<float>(a, f, st); }
}  // namespace sige
