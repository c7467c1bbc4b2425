// gfx950 kernels of the operators around a protected classifier (compiled
// with kernels.hip, see library.hip).
#include "ops.h"

#include <type_traits>

#include "group_norm.h"
#include "fp8_quantize.h"
#include "fp8_product.h"
#include "token_scores.h"
#include "attention.h"
#include "head_norm.h"
#include "clip.h"
