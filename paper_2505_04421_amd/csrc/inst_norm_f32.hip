#include "layer_norm.h"
namespace longer {
namespace ln {
void norm_f32(Params& p, hipStream_t st) { norm<float, 4>(p, st); }
}  // namespace ln
}  // namespace longer
