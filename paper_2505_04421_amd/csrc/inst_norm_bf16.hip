#include "layer_norm.h"
namespace longer {
namespace ln {
void norm_bf16(Params& p, hipStream_t st) { norm<__bf16, 8>(p, st); }
}  // namespace ln
}  // namespace longer
