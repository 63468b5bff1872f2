// Attention over a cache of e4m3 codes with a power of two for each block of rows
// and head (the kernels: attention_kernels.h).

#include "attention_kernels.h"

namespace cl {

hipError_t launch_attention8(const AttnArgs& a, void* ws, hipStream_t st) { return launch_for<true>(a, ws, st); }

}  // namespace cl
