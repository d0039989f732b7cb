// The product in 8 bits over tiles with an epilogue: no activation and ZI_ACT_RELU.
#include "zi_fp8_matmul_epilogue_kernels.h"

namespace zi {

ZI_EPILOGUE_TILES(ActivationKind::kFloor)

}  // namespace zi
