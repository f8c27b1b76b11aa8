#include "layer_norm.h"
namespace longer {
namespace ln {
unsigned grad_bf16(Params& p, unsigned most, float* only, hipStream_t st) { return grad<__bf16, __bf16, 8>(p, most, only, st); }
}  // namespace ln
}  // namespace longer
