#include "layer_norm.h"
namespace longer {
namespace ln {
unsigned grad_f32(Params& p, unsigned most, float* only, hipStream_t st) { return grad<float, float, 4>(p, most, only, st); }
}  // namespace ln
}  // namespace longer
