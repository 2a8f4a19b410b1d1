// What the operators of a network's layers share: eight elements at a time, clusters of CTAs.
// Part of libapms.so: included by layers.cu.
#pragma once

namespace {

template <int TYPE> struct Element;
template <> struct Element<APMS_GRAD_F32> { using T = float; };
template <> struct Element<APMS_GRAD_BF16> { using T = __nv_bfloat16; };
template <> struct Element<APMS_GRAD_F16> { using T = __half; };
template <int TYPE> constexpr int kBytes = (int)sizeof(typename Element<TYPE>::T);

template <int TYPE>
__device__ __forceinline__ float load1(const void* p, int64_t i) { return (float)static_cast<const typename Element<TYPE>::T*>(p)[i]; }
template <int TYPE>
__device__ __forceinline__ void store1(void* p, int64_t i, float v) { store_element(p, i, TYPE, v); }

// Elements i to i + 7 as they lie in memory, in one access: of 16 bytes for 16-bit types, of 32 for binary32 (two of 16 would write half sectors); p + i lies on such a boundary.
template <int TYPE> struct Eight { uint32_t w[2 * kBytes<TYPE>]; };
template <int TYPE>
__device__ __forceinline__ Eight<TYPE> load8(const void* p, int64_t i)
{
    const char* q = static_cast<const char*>(p) + i * kBytes<TYPE>;
    Eight<TYPE> e;
    if constexpr (TYPE == APMS_GRAD_F32) load32(e.w, q); else load16(e.w, q);
    return e;
}
template <int TYPE>
__device__ __forceinline__ void values8(float* v, const Eight<TYPE>& e)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (TYPE == APMS_GRAD_F32) {
            v[2 * k] = __uint_as_float(e.w[2 * k]); v[2 * k + 1] = __uint_as_float(e.w[2 * k + 1]);
        } else {
            const float2 a = unpack16<TYPE>(e.w[k]);
            v[2 * k] = a.x; v[2 * k + 1] = a.y;
        }
    }
}
template <int TYPE>
__device__ __forceinline__ void store8(void* p, int64_t i, const float* v)
{
    char* q = static_cast<char*>(p) + i * kBytes<TYPE>;
    if constexpr (TYPE == APMS_GRAD_F32) {
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(v[k]);
        store32(q, w);
    } else {
        *reinterpret_cast<uint4*>(q) = make_uint4(pack16<TYPE>(v[0], v[1]), pack16<TYPE>(v[2], v[3]), pack16<TYPE>(v[4], v[5]), pack16<TYPE>(v[6], v[7]));
    }
}

// The barrier of all threads of a cluster's CTAs, in two halves and whole: what each wrote before (to global memory or to the others' shared memory) the others may read after,
// and what each read before has been read.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() { cluster_arrive(); cluster_wait(); }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
// The address in CTA `rank` of what this CTA has at shared-memory address `a`.
__device__ __forceinline__ uint32_t cluster_address(uint32_t a, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// As launch(), by clusters of `cluster` CTAs.
template <class... Params, class... Args>
cudaError_t launch_clusters(void (*kernel)(Params...), int cluster, dim3 grid, dim3 threads, size_t shared, cudaStream_t stream, const Args&... args)
{
    cudaLaunchAttribute attribute = {};
    attribute.id = cudaLaunchAttributeClusterDimension;
    attribute.val.clusterDim.x = (unsigned)cluster;
    attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = threads;
    config.dynamicSmemBytes = shared;
    config.stream = stream;
    config.attrs = &attribute;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, Params(args)...);
}

// Raises, once per device, a kernel's limits of shared memory and of the cluster's size.
struct Raised { std::atomic<bool> done{false}; };
cudaError_t raise_limits(Raised* known, const void* kernel, size_t shared, bool large_cluster)
{
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= kMostDevices) return cudaErrorInvalidDevice;
    if (known[device].done.load(std::memory_order_relaxed)) return cudaSuccess;
    if (shared) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared);
    if (e == cudaSuccess && large_cluster) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) known[device].done.store(true, std::memory_order_relaxed);
    return e;
}

inline bool on_element(const void* p, int type) { return (uintptr_t)p % element_size(type) == 0; }
inline bool on_16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
// What load8 and store8 need of an address, and of rows `stride` elements apart.
inline bool on_eight(const void* p, int type) { return (uintptr_t)p % (8 * element_size(type)) == 0; }
inline bool rows_of_eight(const void* p, int64_t rows, int64_t stride, int64_t width, int type)
{
    return !p || (on_eight(p, type) && width % 8 == 0 && (rows <= 1 || stride % 8 == 0));
}

}  // namespace
