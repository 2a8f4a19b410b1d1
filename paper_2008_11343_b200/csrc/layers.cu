// The operators of a network's layers (no context): the embedding lookup and its gradient, dropout, the gated linear recurrence.

#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <algorithm>
#include <atomic>
#include <math.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>
#include <type_traits>

#include "apms.h"
#include "errors.h"

#include "op_common.cuh"
#include "layer_common.cuh"
#include "layer_dropout.cuh"
#include "layer_embedding.cuh"
#include "layer_recurrence.cuh"
