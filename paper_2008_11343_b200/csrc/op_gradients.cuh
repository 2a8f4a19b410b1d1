// The norm of a list of tensors, and clipping in place or into one flat gradient.
// Part of libapms.so: included by operators.cu.
//
//   S_t = sum_j g_tj^2 (binary64),  norm = sqrt(sum_t S_t),  c = norm <= max ? 1 : max / norm,  out = g * c
//
// The list is cut into tiles; a tile lies in one tensor and is one CTA.  Both kernels are HBM streams: 2 operations per
// element read.
#pragma once

namespace {

constexpr int kGradThreads = 256;
constexpr int kTileBytes = 32768;        // of a tensor's elements
constexpr int kListPointers = 500;       // tensors' addresses in a launch's arguments

struct TileRecord {
    int64_t first;                       // first element, counted inside its tensor
    int64_t out;                         // ... and inside the whole list (its place in the flat gradient)
    int32_t length;
    int32_t tensor;
};
struct TensorRecord {
    int64_t cols, stride;                // rows of `cols` consecutive elements, `stride` apart
    int32_t type;
    int32_t contiguous;
    int32_t tile0, tiles;
};
struct TensorPointers { const void* p[kListPointers]; };

// Where element e of a tensor lies.
__device__ __forceinline__ int64_t element_place(const TensorRecord& t, int64_t e)
{
    return t.contiguous ? e : e / t.cols * t.stride + e % t.cols;
}

__global__ void __launch_bounds__(kGradThreads)
k_tile_squares(const __grid_constant__ TensorPointers ptrs, int tensor0, const TileRecord* __restrict__ tiles, int64_t tile0,
               const TensorRecord* __restrict__ tensors, double* __restrict__ partial)
{
    __shared__ double red[kGradThreads / 32];
    const TileRecord tile = tiles[tile0 + blockIdx.x];
    const TensorRecord t = tensors[tile.tensor];
    const void* p = ptrs.p[tile.tensor - tensor0];
    double acc = 0.0;
    for (int k = threadIdx.x; k < tile.length; k += kGradThreads) {
        const double g = (double)load_element(p, element_place(t, tile.first + k), t.type);
        acc = fma(g, g, acc);
    }
    acc = block_total(acc, red);
    if (threadIdx.x == 0) partial[tile0 + blockIdx.x] = acc;
}

__device__ __forceinline__ float clip_factor(double squares, float max_norm)
{
    const double norm = sqrt(squares);
    return (isinf(max_norm) || (float)norm <= max_norm) ? 1.0f : (float)((double)max_norm / norm);
}

// One CTA: the tensors' sums, then the list's.
__global__ void __launch_bounds__(kGradThreads)
k_list_norm(const TensorRecord* __restrict__ tensors, int count, const double* __restrict__ partial, float* __restrict__ norm,
            float* __restrict__ norms, float max_norm, float* __restrict__ factor)
{
    __shared__ double red[kGradThreads / 32];
    double total = 0.0;
    for (int t = threadIdx.x; t < count; t += kGradThreads) {
        double s = 0.0;
        for (int k = 0; k < tensors[t].tiles; ++k) s += partial[tensors[t].tile0 + k];
        if (norms) norms[t] = (float)sqrt(s);
        total += s;
    }
    total = block_total(total, red);
    if (threadIdx.x == 0) {
        *norm = (float)sqrt(total);
        *factor = clip_factor(total, max_norm);
    }
}

__global__ void __launch_bounds__(kGradThreads)
k_scale_tiles(const __grid_constant__ TensorPointers ptrs, int tensor0, const TileRecord* __restrict__ tiles, int64_t tile0,
              const TensorRecord* __restrict__ tensors, void* flat, int flat_type, const float* __restrict__ factor)
{
    const TileRecord tile = tiles[tile0 + blockIdx.x];
    const TensorRecord t = tensors[tile.tensor];
    void* p = const_cast<void*>(ptrs.p[tile.tensor - tensor0]);
    const float c = *factor;
    for (int k = threadIdx.x; k < tile.length; k += kGradThreads) {
        const int64_t at = element_place(t, tile.first + k);
        const float g = load_element(p, at, t.type) * c;
        if (flat) store_element(flat, tile.out + k, flat_type, g);
        else store_element(p, at, t.type, g);
    }
}

}  // namespace

struct apms_tensors {
    std::vector<TensorRecord> tensors;
    std::vector<TileRecord> tiles;
    std::vector<int64_t> numel;
    int64_t total;
    TileRecord* d_tiles;
    TensorRecord* d_tensors;
    double* d_partial;
    float* d_factor;

    size_t place(size_t* tensors_at, size_t* partial_at, size_t* factor_at) const
    {
        auto up = [](size_t v) { return (v + 255) / 256 * 256; };
        *tensors_at = up(tiles.size() * sizeof(TileRecord));
        *partial_at = *tensors_at + up(tensors.size() * sizeof(TensorRecord));
        *factor_at = *partial_at + up(tiles.size() * sizeof(double));
        return *factor_at + 256;
    }
};

extern "C" {

apms_status apms_tensors_create(apms_tensors** out, int count, const int64_t* numel, const apms_grad_type* types,
                                const int64_t* cols, const int64_t* row_strides)
{
    if (!out) return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_create: out is NULL");
    *out = nullptr;
    if (count < 1 || !numel || !types || (!cols) != (!row_strides))
        return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_create: needs count >= 1, numel and types, and cols and row_strides together");
    for (int t = 0; t < count; ++t) {
        if (numel[t] < 0 || numel[t] > ((int64_t)1 << 40)) return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_create: tensor %d has %lld elements", t, (long long)numel[t]);
        if (!known_type(types[t])) return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_create: tensor %d has an unknown element type", t);
        if (cols && numel[t] && (cols[t] < 1 || numel[t] % cols[t] || row_strides[t] < cols[t]))
            return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_create: tensor %d: %lld elements are no rows of %lld, %lld apart", t,
                                 (long long)numel[t], (long long)cols[t], (long long)row_strides[t]);
    }
    try {
        apms_tensors* list = new apms_tensors();
        int64_t at = 0;
        for (int t = 0; t < count; ++t) {
            TensorRecord r = {};
            r.type = types[t];
            r.contiguous = !cols || row_strides[t] == cols[t] || cols[t] == numel[t];
            r.cols = r.contiguous ? numel[t] : cols[t];
            r.stride = r.contiguous ? numel[t] : row_strides[t];
            r.tile0 = (int32_t)list->tiles.size();
            const int64_t per_tile = kTileBytes / (int64_t)element_size(types[t]);
            for (int64_t e = 0; e < numel[t]; e += per_tile) {
                if (list->tiles.size() >= 0x7fffffff) { delete list; return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_create: the list is too long"); }
                list->tiles.push_back({e, at + e, (int32_t)std::min(per_tile, numel[t] - e), t});
            }
            r.tiles = (int32_t)list->tiles.size() - r.tile0;
            list->tensors.push_back(r);
            list->numel.push_back(numel[t]);
            at += numel[t];
        }
        list->total = at;
        *out = list;
    } catch (const std::bad_alloc&) {
        return operator_fail(APMS_ERR_OOM, "apms_tensors_create: host allocation failed");
    }
    return APMS_OK;
}

size_t apms_tensors_workspace_bytes(const apms_tensors* list)
{
    size_t a, b, c;
    return list ? list->place(&a, &b, &c) : 0;
}

apms_status apms_tensors_bind(apms_tensors* list, void* workspace_dev, size_t bytes, void* cuda_stream)
{
    if (!list || !workspace_dev || ((uintptr_t)workspace_dev & 255u)) return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_bind: needs a list and a 256-byte aligned workspace");
    size_t tensors_at, partial_at, factor_at;
    if (bytes < list->place(&tensors_at, &partial_at, &factor_at)) return operator_fail(APMS_ERR_OOM, "apms_tensors_bind: workspace smaller than apms_tensors_workspace_bytes()");
    char* ws = (char*)workspace_dev;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    OPERATOR_CUDA("apms_tensors_bind", cudaMemcpyAsync(ws, list->tiles.data(), list->tiles.size() * sizeof(TileRecord), cudaMemcpyHostToDevice, stream));
    OPERATOR_CUDA("apms_tensors_bind", cudaMemcpyAsync(ws + tensors_at, list->tensors.data(), list->tensors.size() * sizeof(TensorRecord), cudaMemcpyHostToDevice, stream));
    OPERATOR_CUDA("apms_tensors_bind", cudaStreamSynchronize(stream));
    list->d_tiles = (TileRecord*)ws;
    list->d_tensors = (TensorRecord*)(ws + tensors_at);
    list->d_partial = (double*)(ws + partial_at);
    list->d_factor = (float*)(ws + factor_at);
    return APMS_OK;
}

void apms_tensors_destroy(apms_tensors* list) { delete list; }

}  // extern "C"

namespace {

apms_status check_addresses(const apms_tensors* list, const void* const* tensors_dev, const char* who)
{
    if (!list || !list->d_tiles) return operator_fail(APMS_ERR_BAD_STATE, "%s: the list has no workspace (apms_tensors_bind)", who);
    if (!tensors_dev) return operator_fail(APMS_ERR_INVALID_ARG, "%s: tensors_dev is NULL", who);
    for (size_t t = 0; t < list->tensors.size(); ++t)
        if (list->numel[t] && (!tensors_dev[t] || (uintptr_t)tensors_dev[t] % element_size(list->tensors[t].type)))
            return operator_fail(APMS_ERR_INVALID_ARG, "%s: tensor %zu is at a NULL or misaligned address", who, t);
    return APMS_OK;
}

// The bytes tensor t spans, from its first element to behind its last.
int64_t spanned_bytes(const apms_tensors* list, size_t t)
{
    const TensorRecord& r = list->tensors[t];
    if (!list->numel[t]) return 0;
    return ((list->numel[t] / r.cols - 1) * r.stride + r.cols) * (int64_t)element_size(r.type);
}

// Launches `kernel(pointers, first tensor, tiles, first tile, tensors, ...)` over the list's tiles, as many tensors at a
// time as a launch's arguments hold addresses.
template <class Kernel, class... Args>
cudaError_t over_tiles(const apms_tensors* list, const void* const* tensors_dev, cudaStream_t stream, Kernel kernel, Args... args)
{
    const int count = (int)list->tensors.size();
    for (int t0 = 0; t0 < count; t0 += kListPointers) {
        const int t1 = std::min(count, t0 + kListPointers);
        const int64_t first = list->tensors[t0].tile0, last = list->tensors[t1 - 1].tile0 + list->tensors[t1 - 1].tiles;
        if (first == last) continue;
        TensorPointers ptrs;
        memcpy(ptrs.p, tensors_dev + t0, (t1 - t0) * sizeof(void*));
        kernel<<<(unsigned)(last - first), kGradThreads, 0, stream>>>(ptrs, t0, list->d_tiles, first, list->d_tensors, args...);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

apms_status list_norm(apms_tensors* list, const void* const* tensors_dev, float* norm_dev, float* norms_dev, float max_norm,
                      cudaStream_t stream, const char* who)
{
    cudaError_t e = over_tiles(list, tensors_dev, stream, k_tile_squares, list->d_partial);
    if (e == cudaSuccess) {
        k_list_norm<<<1, kGradThreads, 0, stream>>>(list->d_tensors, (int)list->tensors.size(), list->d_partial, norm_dev, norms_dev, max_norm, list->d_factor);
        e = cudaGetLastError();
    }
    return e == cudaSuccess ? APMS_OK : operator_fail(APMS_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
}

}  // namespace

extern "C" {

apms_status apms_grad_norm(apms_tensors* list, const void* const* tensors_dev, float* norm_dev, float* norms_dev, void* cuda_stream)
{
    const apms_status st = check_addresses(list, tensors_dev, "apms_grad_norm");
    if (st != APMS_OK) return st;
    if (!norm_dev) return operator_fail(APMS_ERR_INVALID_ARG, "apms_grad_norm: norm_dev is NULL");
    return list_norm(list, tensors_dev, norm_dev, norms_dev, INFINITY, (cudaStream_t)cuda_stream, "apms_grad_norm");
}

apms_status apms_clip_grads(apms_tensors* list, void* const* tensors_dev, float max_norm, void* flat_dev, apms_grad_type flat_type,
                            float* norm_dev, void* cuda_stream)
{
    apms_status st = check_addresses(list, tensors_dev, "apms_clip_grads");
    if (st != APMS_OK) return st;
    if (!norm_dev) return operator_fail(APMS_ERR_INVALID_ARG, "apms_clip_grads: norm_dev is NULL");
    if (!(max_norm >= 0.0f)) return operator_fail(APMS_ERR_INVALID_ARG, "apms_clip_grads: max_norm must be >= 0, got %g", (double)max_norm);
    const size_t count = list->tensors.size();
    if (flat_dev) {
        if (!known_type(flat_type) || ((uintptr_t)flat_dev & 15u)) return operator_fail(APMS_ERR_INVALID_ARG, "apms_clip_grads: flat_dev must be 16-byte aligned, of a known type");
        const uintptr_t f0 = (uintptr_t)flat_dev, es = element_size(flat_type), f1 = f0 + (uintptr_t)list->total * es;
        int64_t at = 0;
        for (size_t t = 0; t < count; at += list->numel[t], ++t) {
            const uintptr_t a0 = (uintptr_t)tensors_dev[t], a1 = a0 + (uintptr_t)spanned_bytes(list, t);
            if (a0 == a1 || a1 <= f0 || a0 >= f1) continue;
            if (!list->tensors[t].contiguous || list->tensors[t].type != (int)flat_type || a0 != f0 + (uintptr_t)at * es)
                return operator_fail(APMS_ERR_INVALID_ARG, "apms_clip_grads: tensor %zu overlaps the flat gradient without being in its place there", t);
        }
    } else {
        try {
            // of a tensor in rows its first row only: column slices of one matrix interleave without sharing elements
            std::vector<std::pair<uintptr_t, uintptr_t>> spans;
            for (size_t t = 0; t < count; ++t)
                if (list->numel[t]) spans.push_back({(uintptr_t)tensors_dev[t], (uintptr_t)tensors_dev[t] + (uintptr_t)list->tensors[t].cols * element_size(list->tensors[t].type)});
            std::sort(spans.begin(), spans.end());
            for (size_t k = 1; k < spans.size(); ++k)
                if (spans[k].first < spans[k - 1].second) return operator_fail(APMS_ERR_INVALID_ARG, "apms_clip_grads: two tensors of the list overlap in memory; clip into a flat gradient instead");
        } catch (const std::bad_alloc&) {
            return operator_fail(APMS_ERR_OOM, "apms_clip_grads: host allocation failed");
        }
    }
    st = list_norm(list, tensors_dev, norm_dev, nullptr, max_norm, (cudaStream_t)cuda_stream, "apms_clip_grads");
    if (st != APMS_OK) return st;
    const cudaError_t e = over_tiles(list, tensors_dev, (cudaStream_t)cuda_stream, k_scale_tiles, flat_dev, (int)flat_type, (const float*)list->d_factor);
    return e == cudaSuccess ? APMS_OK : operator_fail(APMS_ERR_CUDA, "apms_clip_grads: %s", cudaGetErrorString(e));
}

}  // extern "C"
