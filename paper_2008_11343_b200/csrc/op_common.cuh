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

// Two 16-bit elements in a word, the first in the low half.
template <int TYPE>
__device__ __forceinline__ float2 unpack16(uint32_t w)
{
    if (TYPE == APMS_GRAD_BF16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <int TYPE>
__device__ __forceinline__ uint32_t pack16(float a, float b)
{
    if (TYPE == APMS_GRAD_BF16) { const __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&v); }
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

template <int TYPE>
__device__ __forceinline__ uint32_t pack16(float2 v) { return pack16<TYPE>(v.x, v.y); }

// Two binary32 operations in one instruction (each half rounded to nearest as the scalar one is).
__device__ __forceinline__ float2 from_pair(unsigned long long v) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ unsigned long long to_pair(float2 a) { unsigned long long r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a.x), "f"(a.y)); return r; }
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(to_pair(a)), "l"(to_pair(b)));
    return from_pair(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(to_pair(a)), "l"(to_pair(b)));
    return from_pair(r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(to_pair(a)), "l"(to_pair(b)), "l"(to_pair(c)));
    return from_pair(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// 32 bytes in one access (sm_100's widest); p is 32-byte aligned.
__device__ __forceinline__ void load32(uint32_t* w, const void* p)
{
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint32_t* w)
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void load16(uint32_t* w, const void* p)
{
    const uint4 v = *static_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}

// Sums in a fixed order, valid in every thread: over a warp, and over the block's threads (smem: one T per warp; may be
// used again by the next call).
template <class T>
__device__ __forceinline__ T warp_total(T v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <class T>
__device__ __forceinline__ T block_total(T v, T* smem)
{
    v = warp_total(v);
    const int warps = (blockDim.x + 31) / 32;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    T t = smem[0];
    for (int w = 1; w < warps; ++w) t += smem[w];
    return t;
}

// Programmatic dependent launch: the stream's next kernel may start its CTAs once all of this one's have come here, and reads
// what this one leaves only after its own wait_for_last_kernel(), which returns when this kernel is complete.
__device__ __forceinline__ void allow_next_kernel() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void wait_for_last_kernel() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// early: the kernel calls wait_for_last_kernel() and the stream's last kernel was launched by the same call of the library.
template <class... Params, class... Args>
cudaError_t launch(void (*kernel)(Params...), dim3 grid, dim3 threads, size_t shared, cudaStream_t stream, bool early, const Args&... args)
{
    cudaLaunchAttribute attribute = {};
    attribute.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = threads;
    config.dynamicSmemBytes = shared;
    config.stream = stream;
    config.attrs = &attribute;
    config.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&config, kernel, Params(args)...);
}

constexpr size_t kMostShared = 220 * 1024;         // of a CTA's dynamic shared memory, with room for a kernel's fixed arrays
constexpr int kMostDevices = 64;
struct Resident { std::atomic<int> ctas{0}; };

// How many CTAs of a kernel the current device holds at once (at least one per SM); raises the kernel's limit of dynamic shared memory.
cudaError_t resident_ctas(Resident* known, const void* kernel, int threads, size_t shared, int* ctas)
{
    int device = 0, sms = 0, each = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= kMostDevices) return cudaErrorInvalidDevice;
    *ctas = known[device].ctas.load(std::memory_order_relaxed);
    if (*ctas) return cudaSuccess;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, threads, shared);
    if (e != cudaSuccess) return e;
    *ctas = sms * std::max(1, each);
    known[device].ctas.store(*ctas, std::memory_order_relaxed);
    return cudaSuccess;
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
