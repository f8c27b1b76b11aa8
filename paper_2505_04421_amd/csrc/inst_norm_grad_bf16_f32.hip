#include "layer_norm.h"
namespace longer {
namespace ln {
unsigned grad_bf16_f32(Params& p, unsigned most, float* only, hipStream_t st) { return grad<__bf16, float, 8>(p, most, only, st); }
}  // namespace ln
}  // namespace longer
