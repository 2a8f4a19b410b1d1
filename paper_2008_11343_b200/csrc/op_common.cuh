// Element types, sums and error reporting of the operators beside the step.
// Part of libapms.so: included by operators.cu.
#pragma once

namespace {

// One element of type `type` (apms_grad_type) as binary32 (exact), and back (one rounding, to nearest even).
__device__ __forceinline__ float load_element(const void* p, int64_t i, int type)
{
    if (type == APMS_GRAD_F32) return static_cast<const float*>(p)[i];
    if (type == APMS_GRAD_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_element(void* p, int64_t i, int type, float v)
{
    if (type == APMS_GRAD_F32) static_cast<float*>(p)[i] = v;
    else if (type == APMS_GRAD_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p)[i] = __float2half_rn(v);
}

// Sum over the block's threads in a fixed order; valid in every thread.  smem: one T per warp.  May be called again
// with the same smem.
template <class T>
__device__ __forceinline__ T block_total(T v, T* smem)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int warps = (blockDim.x + 31) / 32;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    T t = smem[0];
    for (int w = 1; w < warps; ++w) t += smem[w];
    return t;
}

inline size_t element_size(int type) { return type == APMS_GRAD_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == APMS_GRAD_F32 || type == APMS_GRAD_BF16 || type == APMS_GRAD_F16; }

apms_status operator_fail(apms_status st, const char* fmt, ...)
{
    va_list a;
    va_start(a, fmt);
    vsnprintf(apms_thread_error(), kThreadErrorBytes, fmt, a);
    va_end(a);
    return st;
}

#define OPERATOR_CUDA(name, call)                                                                            \
    do {                                                                                                     \
        const cudaError_t e__ = (call);                                                                      \
        if (e__ != cudaSuccess) return operator_fail(APMS_ERR_CUDA, name ": %s", cudaGetErrorString(e__));   \
    } while (0)

}  // namespace
