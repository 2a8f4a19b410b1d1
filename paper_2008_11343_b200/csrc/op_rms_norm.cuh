// Root-mean-square norm at a residual junction, with 8-bit output, and its gradient.
// Part of libapms.so: included by operators.cu.
//
//   h = x + r,  rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd w                      (per row)
//   xh = h rstd,  a = w dy,  dx = rstd (a - xh mean(a xh)) + dh,  dw = sum_rows dy xh
#pragma once

namespace {

constexpr int kRmsThreads = 256;
constexpr float kE4m3Max = 448.0f;
constexpr float kScaleFloor = 0x1p-100f;       // a group whose largest |y| is below this counts as zero: 448 / a stays finite

struct RmsArgs {
    int64_t width, x_stride, r_stride;
    const void *x, *r, *w;
    void *h, *y;
    float *scales, *rstd;
    int64_t group, groups;
    int x_type, r_type, w_type;
    float eps;
};

// |v| as bits: ordered like the magnitudes, with infinity and then NaN above every number, so a maximum keeps NaN
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// A group's scale and what its elements are multiplied by.
__device__ __forceinline__ void group_scale(uint32_t most_bits, float* scale, float* inverse)
{
    const float a = __uint_as_float(most_bits);
    const bool none = a < kScaleFloor;
    *scale = none ? 0.0f : __fdiv_rn(a, kE4m3Max);
    *inverse = none ? 0.0f : __fdiv_rn(kE4m3Max, a);
}

// One CTA per row, any width, stride and alignment: the row is read again for each of the passes.
__global__ void __launch_bounds__(kRmsThreads)
k_rms_rows(const RmsArgs a)
{
    __shared__ float red[kRmsThreads / 32];
    __shared__ uint32_t most;
    const int64_t row = blockIdx.x;
    const int64_t x0 = row * a.x_stride, r0 = row * a.r_stride, o0 = row * a.width;
    auto h_of = [&](int64_t c) {
        float h = load_element(a.x, x0 + c, a.x_type);
        return a.r ? h + load_element(a.r, r0 + c, a.r_type) : h;
    };
    float acc = 0.0f;
    for (int64_t c = threadIdx.x; c < a.width; c += kRmsThreads) {
        const float h = h_of(c);
        acc = fmaf(h, h, acc);
    }
    const float rstd = __frsqrt_rn(block_total(acc, red) / (float)a.width + a.eps);
    if (threadIdx.x == 0) a.rstd[row] = rstd;
    if (!a.scales) {
        for (int64_t c = threadIdx.x; c < a.width; c += kRmsThreads) {
            const float h = h_of(c);
            if (a.r) store_element(a.h, o0 + c, a.r_type, h);
            store_element(a.y, o0 + c, a.x_type, h * rstd * load_element(a.w, c, a.w_type));
        }
        return;
    }
    for (int64_t g = 0; g < a.groups; ++g) {
        const int64_t c1 = min(a.width, (g + 1) * a.group);
        if (threadIdx.x == 0) most = 0;
        __syncthreads();
        uint32_t m = 0;
        for (int64_t c = g * a.group + threadIdx.x; c < c1; c += kRmsThreads) m = max(m, magnitude_bits(h_of(c) * rstd * load_element(a.w, c, a.w_type)));
        atomicMax(&most, m);
        __syncthreads();
        float scale, inverse;
        group_scale(most, &scale, &inverse);
        if (threadIdx.x == 0) a.scales[row * a.groups + g] = scale;
        for (int64_t c = g * a.group + threadIdx.x; c < c1; c += kRmsThreads) {
            const float h = h_of(c);
            if (a.r) store_element(a.h, o0 + c, a.r_type, h);
            static_cast<uint8_t*>(a.y)[o0 + c] = __nv_cvt_float_to_fp8(h * rstd * load_element(a.w, c, a.w_type) * inverse, __NV_SATFINITE, __NV_E4M3);
        }
        __syncthreads();
    }
}

struct RmsBackArgs {
    int64_t rows, width, dy_stride, h_stride, dh_stride;
    const void *dy, *h, *w, *dh;
    const float* rstd;
    void *dx, *dr, *dw;
    float* partial;
    int dy_type, h_type, w_type;
};

__global__ void __launch_bounds__(kRmsThreads)
k_rms_back_rows(const RmsBackArgs a)
{
    __shared__ float red[kRmsThreads / 32];
    const int64_t row = blockIdx.x;
    const float rstd = a.rstd[row];
    float acc = 0.0f;
    for (int64_t c = threadIdx.x; c < a.width; c += kRmsThreads) {
        const float xh = load_element(a.h, row * a.h_stride + c, a.h_type) * rstd;
        acc = fmaf(load_element(a.w, c, a.w_type) * load_element(a.dy, row * a.dy_stride + c, a.dy_type), xh, acc);
    }
    const float mean = block_total(acc, red) / (float)a.width;
    for (int64_t c = threadIdx.x; c < a.width; c += kRmsThreads) {
        const float xh = load_element(a.h, row * a.h_stride + c, a.h_type) * rstd;
        const float v = load_element(a.w, c, a.w_type) * load_element(a.dy, row * a.dy_stride + c, a.dy_type);
        float dx = rstd * (v - xh * mean);
        if (a.dh) dx += load_element(a.dh, row * a.dh_stride + c, a.h_type);
        store_element(a.dx, row * a.width + c, a.dy_type, dx);
        if (a.dr) store_element(a.dr, row * a.width + c, a.h_type, dx);
    }
}

// dweight in two stages: strips of rows into partial sums, then the strips.
constexpr int kStrips = 64;

__global__ void __launch_bounds__(kRmsThreads)
k_rms_back_weight(const RmsBackArgs a)
{
    const int64_t c = (int64_t)blockIdx.x * kRmsThreads + threadIdx.x;
    if (c >= a.width) return;
    const int64_t per = (a.rows + kStrips - 1) / kStrips, row0 = blockIdx.y * per, row1 = min(a.rows, row0 + per);
    float acc = 0.0f;
    for (int64_t row = row0; row < row1; ++row)
        acc = fmaf(load_element(a.dy, row * a.dy_stride + c, a.dy_type), load_element(a.h, row * a.h_stride + c, a.h_type) * a.rstd[row], acc);
    a.partial[blockIdx.y * a.width + c] = acc;
}

__global__ void __launch_bounds__(kRmsThreads)
k_rms_back_strips(const RmsBackArgs a)
{
    const int64_t c = (int64_t)blockIdx.x * kRmsThreads + threadIdx.x;
    if (c >= a.width) return;
    float acc = 0.0f;
    for (int s = 0; s < kStrips; ++s) acc += a.partial[s * a.width + c];
    store_element(a.dw, c, a.w_type, acc);
}

bool aligned_to(const void* p, int type) { return (uintptr_t)p % element_size(type) == 0; }
// The statistics stay in the activations' own type or in binary32.
bool type_pair(int narrow, int wide) { return known_type(narrow) && known_type(wide) && (wide == narrow || wide == APMS_GRAD_F32); }

constexpr int64_t kMostRows = 0x7fffffff, kMostWidth = (int64_t)1 << 24;

}  // namespace

extern "C" {

apms_status apms_rms_norm(const apms_rms_norm_args* args, void* cuda_stream)
{
    const char* who = "apms_rms_norm";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_rms_norm_args& g = *args;
    if (g.rows < 0 || g.rows > kMostRows || g.width < 1 || g.width > kMostWidth)
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld rows of %lld: needs 0 <= rows < 2^31 and 1 <= width <= 2^24", who, (long long)g.rows, (long long)g.width);
    if (!type_pair(g.x_type, g.weight_type) || (g.residual && !type_pair(g.x_type, g.residual_type)))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: the weight and the residual have x's type or binary32", who);
    if (!(g.eps >= 0.0f)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: eps must be >= 0, got %g", who, (double)g.eps);
    if (g.scales && g.group != 0 && g.group != 128) return operator_fail(APMS_ERR_INVALID_ARG, "%s: group must be 0 (a row) or 128, got %lld", who, (long long)g.group);
    if (g.rows == 0) return APMS_OK;
    if (!g.x || !g.weight || !g.y || !g.rstd || (g.residual && !g.h)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: x, weight, y, rstd, or h beside a residual is NULL", who);
    if ((g.rows > 1 && g.x_stride < g.width) || (g.residual && g.rows > 1 && g.residual_stride < g.width)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: rows overlap: a stride is below the width", who);
    if (!aligned_to(g.x, g.x_type) || !aligned_to(g.weight, g.weight_type) || (!g.scales && !aligned_to(g.y, g.x_type)) || !aligned_to(g.rstd, APMS_GRAD_F32) ||
        !aligned_to(g.scales, APMS_GRAD_F32) || (g.residual && (!aligned_to(g.residual, g.residual_type) || !aligned_to(g.h, g.residual_type))))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    RmsArgs a = {};
    a.width = g.width; a.x_stride = g.x_stride; a.r_stride = g.residual_stride;
    a.x = g.x; a.r = g.residual; a.w = g.weight; a.h = g.h; a.y = g.y; a.scales = g.scales; a.rstd = g.rstd;
    a.group = g.group ? g.group : g.width;
    a.groups = (g.width + a.group - 1) / a.group;
    a.x_type = g.x_type; a.r_type = g.residual_type; a.w_type = g.weight_type; a.eps = g.eps;
    k_rms_rows<<<(unsigned)g.rows, kRmsThreads, 0, (cudaStream_t)cuda_stream>>>(a);
    OPERATOR_CUDA("apms_rms_norm", cudaGetLastError());
    return APMS_OK;
}

size_t apms_rms_norm_backward_workspace_bytes(int64_t rows, int64_t width)
{
    if (rows < 0 || rows > kMostRows || width < 1 || width > kMostWidth) return 0;
    return (size_t)kStrips * (size_t)width * sizeof(float);
}

apms_status apms_rms_norm_backward(const apms_rms_norm_backward_args* args, void* cuda_stream)
{
    const char* who = "apms_rms_norm_backward";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_rms_norm_backward_args& g = *args;
    if (g.rows < 0 || g.rows > kMostRows || g.width < 1 || g.width > kMostWidth)
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld rows of %lld: needs 0 <= rows < 2^31 and 1 <= width <= 2^24", who, (long long)g.rows, (long long)g.width);
    if (!type_pair(g.dy_type, g.h_type) || !type_pair(g.dy_type, g.weight_type))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: h and the weight have dy's type or binary32", who);
    if (!g.dweight || !g.weight || (g.rows && (!g.dy || !g.h || !g.rstd || !g.dx)))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: dy, h, weight, rstd, dx or dweight is NULL", who);
    if (g.rows > 1 && (g.dy_stride < g.width || g.h_stride < g.width || (g.dh && g.dh_stride < g.width))) return operator_fail(APMS_ERR_INVALID_ARG, "%s: rows overlap: a stride is below the width", who);
    if (!aligned_to(g.dy, g.dy_type) || !aligned_to(g.h, g.h_type) || !aligned_to(g.weight, g.weight_type) || !aligned_to(g.rstd, APMS_GRAD_F32) || !aligned_to(g.dh, g.h_type) ||
        !aligned_to(g.dx, g.dy_type) || !aligned_to(g.dresidual, g.h_type) || !aligned_to(g.dweight, g.weight_type))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    if (!g.workspace_dev || ((uintptr_t)g.workspace_dev & 15u) || g.workspace_bytes < apms_rms_norm_backward_workspace_bytes(g.rows, g.width))
        return operator_fail(APMS_ERR_OOM, "%s: needs apms_rms_norm_backward_workspace_bytes() of 16-byte aligned workspace", who);
    RmsBackArgs a = {};
    a.rows = g.rows; a.width = g.width; a.dy_stride = g.dy_stride; a.h_stride = g.h_stride; a.dh_stride = g.dh_stride;
    a.dy = g.dy; a.h = g.h; a.w = g.weight; a.dh = g.dh; a.rstd = g.rstd; a.dx = g.dx; a.dr = g.dresidual; a.dw = g.dweight;
    a.partial = (float*)g.workspace_dev;
    a.dy_type = g.dy_type; a.h_type = g.h_type; a.w_type = g.weight_type;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (g.rows) {
        k_rms_back_rows<<<(unsigned)g.rows, kRmsThreads, 0, stream>>>(a);
        OPERATOR_CUDA("apms_rms_norm_backward", cudaGetLastError());
    }
    const unsigned columns = (unsigned)((g.width + kRmsThreads - 1) / kRmsThreads);
    k_rms_back_weight<<<dim3(columns, kStrips), kRmsThreads, 0, stream>>>(a);
    OPERATOR_CUDA("apms_rms_norm_backward", cudaGetLastError());
    k_rms_back_strips<<<columns, kRmsThreads, 0, stream>>>(a);
    OPERATOR_CUDA("apms_rms_norm_backward", cudaGetLastError());
    return APMS_OK;
}

}  // extern "C"
