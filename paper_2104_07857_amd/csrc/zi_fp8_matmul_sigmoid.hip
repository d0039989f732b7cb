// The product in 8 bits over tiles with an epilogue: ZI_ACT_GELU_TANH and ZI_ACT_SILU.
#include "zi_fp8_matmul_epilogue_kernels.h"

namespace zi {

ZI_EPILOGUE_TILES(ActivationKind::kSigmoid)

}  // namespace zi
