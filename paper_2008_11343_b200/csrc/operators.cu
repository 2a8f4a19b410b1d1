// The operators beside the step (no context): the norm of a list of tensors and clipping, the root-mean-square norm at
// a residual junction and its gradient.

#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <algorithm>
#include <atomic>
#include <math.h>
#include <memory>
#include <new>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>
#include <type_traits>
#include <vector>

#include "apms.h"
#include "errors.h"

#include "op_common.cuh"
#include "op_gradients.cuh"
#include "op_rms_norm.cuh"
