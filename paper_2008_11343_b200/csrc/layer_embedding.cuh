// The embedding lookup with scaling, and its gradient by sorted tokens.
// Part of libapms.so: included by layers.cu.
#pragma once

namespace {

struct Tokens {
    const void* p;
    int wide;                                                       // 64-bit numbers
    int64_t vocab;
    // The token's row, or `vocab` where it has none.
    __device__ __forceinline__ uint32_t row(int64_t i) const
    {
        const long long t = wide ? static_cast<const long long*>(p)[i] : static_cast<const int*>(p)[i];
        return t >= 0 && t < vocab ? (uint32_t)t : (uint32_t)vocab;
    }
};

struct EmbedArgs {
    Tokens tokens;
    int64_t count, width, w_stride;
    const void* w;
    void* out;
    float scale;
};

// ------------------------------------------------------------------------------------------ lookup

// out = round(scale * w[token]), by groups of eight elements (rows on 16-byte boundaries), UNITS groups a thread so that as many chains of
// token -> row are in flight.  Bound by HBM: the distinct rows once (repeats come from L2), the output once.
template <int WT, int OT, int UNITS>
__global__ void __launch_bounds__(256) k_embed(EmbedArgs a)
{
    const int64_t per_row = a.width / 8, units = a.count * per_row, first = (int64_t)blockIdx.x * (256 * UNITS) + threadIdx.x;
    uint32_t from[UNITS];
    int64_t col[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const int64_t u = first + k * 256;
        if (u >= units) break;
        const int64_t row = units <= 0xffffffffll ? (uint32_t)u / (uint32_t)per_row : u / per_row;
        col[k] = (u - row * per_row) * 8;
        from[k] = a.tokens.row(row);
    }
    Eight<WT> w[UNITS];
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        if (first + k * 256 >= units) break;
        if (from[k] < a.tokens.vocab) w[k] = load8<WT>(a.w, from[k] * a.w_stride + col[k]);
    }
#pragma unroll
    for (int k = 0; k < UNITS; ++k) {
        const int64_t u = first + k * 256;
        if (u >= units) break;
        float v[8] = {};
        if (from[k] < a.tokens.vocab) {
            values8<WT>(v, w[k]);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= a.scale;
        }
        store8<OT>(a.out, u * 8, v);
    }
}

// Any width and alignment, element by element, eight a thread.
template <int WT, int OT>
__global__ void __launch_bounds__(256) k_embed_any(EmbedArgs a)
{
    const int64_t numel = a.count * a.width, first = (int64_t)blockIdx.x * 2048 + threadIdx.x;
    float v[8] = {};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t i = first + k * 256;
        if (i >= numel) break;
        const int64_t row = numel <= 0xffffffffll ? (uint32_t)i / (uint32_t)a.width : i / a.width;
        const uint32_t from = a.tokens.row(row);
        if (from < a.tokens.vocab) v[k] = load1<WT>(a.w, from * a.w_stride + (i - row * a.width)) * a.scale;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (first + k * 256 < numel) store1<OT>(a.out, first + k * 256, v[k]);
}

// ------------------------------------------------------------------------------------------ gradient
//
// dw[v] = round(scale * sum of dout[i] over the i with tokens[i] = v), rows without a token 0.  Three kernels:
//   k_embed_sort   the first cluster of CTAs sorts (token, position) by token, positions in order; the other clusters meanwhile write the zeros, so that
//                  the sort costs no time of its own where the table is large
//   k_embed_sums   `length` sorted entries a group of threads, eight rows of dout in flight: runs of one token that lie within are written,
//                  what belongs to a run that goes on to the left or the right is left as a partial sum
//   k_embed_joins  adds up the partial sums of the runs over several groups
// The sums are binary32, in an order that the sizes fix.  Bound by HBM: dout read once, dw written once.

constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortBits = 8, kSortBins = 1 << kSortBits;
constexpr int kMostClearing = 16;                                   // clusters that write zeros
constexpr int kClearRows = 1 << 16;                                 // rows whose bits a CTA of them holds at once

struct EmbedBackArgs {
    Tokens tokens;
    int64_t count, width, d_stride;
    const void* d;
    void* dw;
    uint2 *sorted, *other;                                          // (token, position): the result, and the other buffer of the sort
    float *head, *tail;                                             // partial sums of each group: of the run that came from the left, of the one that goes on
    int64_t padded;                                                 // floats a partial sum's row takes
    int length, passes, digit;                                      // entries a group; of the sort, bits a pass
    int64_t groups;
    float scale;
};

// Which of the warp's lanes hold the same digit.
__device__ __forceinline__ uint32_t same_digit(uint32_t d) { return __match_any_sync(0xffffffffu, d); }

// Stable radix sort, least significant digit first, by one cluster: each warp owns a run of consecutive entries and counts its digits, the CTAs read
// one another's counts through shared memory, and each warp's entries move to their places in order.  Entries live in global memory (L2).
__device__ void embed_sort(const EmbedBackArgs& a, uint32_t (*counts)[kSortBins], uint32_t* total, uint32_t* base, uint32_t* warp_sums)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), bins = 1u << a.digit, mask = bins - 1;
    const int64_t share = ((a.count + kSortCtas * kSortWarps - 1) / (kSortCtas * kSortWarps) + 31) / 32 * 32;
    const int64_t begin = min(a.count, ((int64_t)rank * kSortWarps + warp) * share), end = min(a.count, begin + share);
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit;
        const uint2* from = pass & 1 ? ((a.passes & 1) ? a.sorted : a.other) : ((a.passes & 1) ? a.other : a.sorted);
        uint2* to = pass & 1 ? ((a.passes & 1) ? a.other : a.sorted) : ((a.passes & 1) ? a.sorted : a.other);
        auto entry = [&](int64_t i) { return pass == 0 ? make_uint2(a.tokens.row(i), (uint32_t)i) : __ldcg(from + i); };
        for (uint32_t d = lane; d < bins; d += 32) counts[warp][d] = 0;
        __syncwarp();
        for (int64_t i0 = begin; i0 < end; i0 += 32) {
            const bool here = i0 + lane < end;
            const uint32_t d = here ? (entry(i0 + lane).x >> shift) & mask : bins;
            const uint32_t same = same_digit(d);
            if (here && lane == __ffs(same) - 1) counts[warp][d] += __popc(same);
            __syncwarp();
        }
        __syncthreads();
        if (threadIdx.x < bins) {                                   // each warp's entries of a digit come after those of the warps before it
            uint32_t sum = 0;
            for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = counts[w][threadIdx.x]; counts[w][threadIdx.x] = sum; sum += c; }
            total[threadIdx.x] = sum;
        }
        cluster_barrier();
        uint32_t before = 0, all = 0;
        if (threadIdx.x < bins) {
            for (uint32_t r = 0; r < kSortCtas; ++r) {
                uint32_t c;
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(cluster_address(shared_address(total + threadIdx.x), r)));
                if (r < rank) before += c;
                all += c;
            }
        }
        uint32_t upto = all;                                        // digits in order: an inclusive scan over the CTA's first 256 threads
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
        if (lane == 31) warp_sums[warp] = upto;
        __syncthreads();
        if (threadIdx.x < bins) {
            for (int w = 0; w < warp; ++w) before += warp_sums[w];
            base[threadIdx.x] = before + upto - all;
        }
        __syncthreads();
        for (int64_t i0 = begin; i0 < end; i0 += 32) {
            const bool here = i0 + lane < end;
            const uint2 e = here ? entry(i0 + lane) : make_uint2(0, 0);
            const uint32_t d = here ? (e.x >> shift) & mask : bins;
            const uint32_t same = same_digit(d);
            if (here) {
                const uint32_t at = base[d] + counts[warp][d] + __popc(same & ((1u << lane) - 1));
                __stcg(to + at, e);
            }
            __syncwarp();
            if (here && lane == __ffs(same) - 1) counts[warp][d] += __popc(same);
            __syncwarp();
        }
        cluster_barrier();                                          // the entries are in place, and no CTA's counts are read any more
    }
}

// Zeros into the rows of [begin, end) that no token has.  Each CTA of a cluster looks at a share of the tokens; the rows' bits are joined through shared memory.
template <int OT>
__device__ void embed_clear(const EmbedBackArgs& a, int64_t begin, int64_t end, uint32_t* bits, uint32_t* own, bool vector)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    for (int64_t at = begin; at < end; at += kClearRows) {
        const int64_t rows = min((int64_t)kClearRows, end - at);
        const int words = (int)((rows + 31) / 32);
        for (int w = threadIdx.x; w < words; w += kSortThreads) bits[w] = 0;
        __syncthreads();
        for (int64_t i = (int64_t)rank * kSortThreads + threadIdx.x; i < a.count; i += kSortCtas * kSortThreads) {
            const int64_t r = (int64_t)a.tokens.row(i) - at;
            if (r >= 0 && r < rows) atomicOr(bits + (r >> 5), 1u << (r & 31));
        }
        cluster_barrier();
        const int mine = (words - (int)rank + kSortCtas - 1) / kSortCtas;                             // every eighth word's rows
        for (int k = threadIdx.x; k < mine; k += kSortThreads) {
            uint32_t taken = 0;
            for (uint32_t r = 0; r < kSortCtas; ++r) {
                uint32_t v;
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_address(shared_address(bits + rank + k * kSortCtas), r)));
                taken |= v;
            }
            own[k] = taken;
        }
        __syncthreads();
        const int64_t row_bytes = a.width * kBytes<OT>;
        for (int i = warp; i < mine * 32; i += kSortWarps) {
            const int64_t r = ((int64_t)rank + (i >> 5) * kSortCtas) * 32 + (i & 31);
            if (r >= rows || (own[i >> 5] >> (i & 31) & 1)) continue;
            char* row = static_cast<char*>(a.dw) + (at + r) * row_bytes;
            if (vector) {
                for (int64_t c = lane * 16; c < row_bytes; c += 512) *reinterpret_cast<uint4*>(row + c) = make_uint4(0, 0, 0, 0);
            } else {
                for (int64_t c = lane; c < a.width; c += 32) store1<OT>(row, c, 0.0f);
            }
        }
        cluster_barrier();
    }
}

template <int OT>
__global__ void __launch_bounds__(kSortThreads) k_embed_sort(EmbedBackArgs a, int clearing, int vector)
{
    __shared__ union {
        struct { uint32_t counts[kSortWarps][kSortBins], total[kSortBins], base[kSortBins], warp_sums[kSortWarps]; } sort;
        struct { uint32_t bits[kClearRows / 32], own[kClearRows / 32 / kSortCtas]; } clear;
    } s;
    allow_next_kernel();
    const int cluster = blockIdx.x / kSortCtas;
    if (cluster == 0) {
        embed_sort(a, s.sort.counts, s.sort.total, s.sort.base, s.sort.warp_sums);
    } else {
        const int64_t share = ((a.tokens.vocab + clearing - 1) / clearing + 31) / 32 * 32, begin = min(a.tokens.vocab, (cluster - 1) * share);
        embed_clear<OT>(a, begin, min(a.tokens.vocab, begin + share), s.clear.bits, s.clear.own, vector);
    }
}

// Columns of the groups of eight that a thread holds: consecutive where rows lie on 16-byte boundaries, else `lanes` apart.
template <int DT, bool VECTOR>
struct Columns {
    int64_t first;
    int lanes;
    __device__ __forceinline__ int64_t at(int j) const { return VECTOR ? first + j : first + (int64_t)j * lanes; }
};

// A group: `lanes` threads (a power of two up to 128) hold 8 columns each of a slice of 8 * lanes; blockIdx.y is the slice.
template <int DT, int OT, bool VECTOR>
__global__ void __launch_bounds__(128) k_embed_sums(EmbedBackArgs a, int lanes)
{
    constexpr int FLIGHT = 8;
    const int lane = threadIdx.x & (lanes - 1), per_cta = 128 / lanes;
    const int64_t group = (int64_t)blockIdx.x * per_cta + threadIdx.x / lanes;
    const Columns<DT, VECTOR> columns = {(int64_t)blockIdx.y * 8 * lanes + (VECTOR ? lane * 8 : lane), lanes};
    wait_for_last_kernel();
    allow_next_kernel();
    if (group >= a.groups || columns.first >= a.width) return;
    const int64_t begin = group * a.length, end = min(a.count, begin + a.length);
    const uint32_t vocab = (uint32_t)a.tokens.vocab;
    const uint32_t left = begin ? a.sorted[begin - 1].x : vocab, right = end < a.count ? a.sorted[end].x : vocab;
    float sum[8];
    uint32_t run = vocab;                                           // the running token; `vocab`: none yet
    bool from_left = false;

    auto write = [&](bool goes_on) {
        if (run == vocab) return;
        float* partial = from_left ? a.head + group * a.padded : goes_on ? a.tail + group * a.padded : nullptr;
        if (VECTOR) {
            if (partial) { store8<APMS_GRAD_F32>(partial, columns.first, sum); return; }
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = sum[j] * a.scale;
            store8<OT>(a.dw, run * a.width + columns.first, v);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (columns.at(j) >= a.width) break;
                if (partial) partial[columns.at(j)] = sum[j];
                else store1<OT>(a.dw, run * a.width + columns.at(j), sum[j] * a.scale);
            }
        }
    };

    for (int64_t i0 = begin; i0 < end; i0 += FLIGHT) {
        uint2 e[FLIGHT];
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) e[k] = i0 + k < end ? a.sorted[i0 + k] : make_uint2(vocab, 0);
        float v[VECTOR ? 1 : FLIGHT][8];
        Eight<DT> raw[VECTOR ? FLIGHT : 1];
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            if (e[k].x == vocab) continue;
            if constexpr (VECTOR) {
                raw[k] = load8<DT>(a.d, e[k].y * a.d_stride + columns.first);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[k][j] = columns.at(j) < a.width ? load1<DT>(a.d, e[k].y * a.d_stride + columns.at(j)) : 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            if (e[k].x == vocab) continue;                          // behind the group's entries, or no row (sorted last)
            float one[8];
            if constexpr (VECTOR) values8<DT>(one, raw[k]);
            if (e[k].x != run) {
                write(false);
                from_left = run == vocab && e[k].x == left;
                run = e[k].x;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = VECTOR ? one[j] : v[VECTOR ? 0 : k][j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += VECTOR ? one[j] : v[VECTOR ? 0 : k][j];
            }
        }
    }
    write(run == right);
}

// The runs over several groups: 256 columns a CTA, four a thread, its four strips of threads taking every fourth partial sum.
template <int OT>
__global__ void __launch_bounds__(256) k_embed_joins(EmbedBackArgs a)
{
    __shared__ float4 sums[3][64];
    const int64_t group = blockIdx.x, end = (group + 1) * a.length;
    const int lane = threadIdx.x & 63, strip = threadIdx.x >> 6;
    wait_for_last_kernel();
    const uint32_t run = a.sorted[end - 1].x, before = group ? a.sorted[end - a.length - 1].x : (uint32_t)a.tokens.vocab;
    // launched for all groups but the last, so end < count
    if (a.sorted[end].x != run || before == run || run == (uint32_t)a.tokens.vocab) return;               // none goes on, or it began further left
    int64_t low = group + 1, high = a.groups;                       // the last group that begins with the run: in [low, high)
    while (high - low > 1) {
        const int64_t middle = (low + high) / 2;
        if (a.sorted[middle * a.length].x == run) low = middle; else high = middle;
    }
    for (int64_t c0 = (int64_t)blockIdx.y * 256; c0 < a.width; c0 += (int64_t)gridDim.y * 256) {
        const int64_t c = c0 + lane * 4;                            // padded rows: whole groups of four
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto add = [&](const float4& v) { sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w; };
        if (c < a.width) {
            if (strip == 0) sum = *reinterpret_cast<const float4*>(a.tail + group * a.padded + c);
            int64_t g = group + 1 + strip;
            for (; g + 28 <= low; g += 32) {
                float4 v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const float4*>(a.head + (g + 4 * k) * a.padded + c);
#pragma unroll
                for (int k = 0; k < 8; ++k) add(v[k]);
            }
            for (; g <= low; g += 4) add(*reinterpret_cast<const float4*>(a.head + g * a.padded + c));
        }
        __syncthreads();
        if (strip) sums[strip - 1][lane] = sum;
        __syncthreads();
        if (strip == 0 && c < a.width) {
            for (int s = 0; s < 3; ++s) add(sums[s][lane]);
            const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < a.width) store1<OT>(a.dw, run * a.width + c + j, v[j] * a.scale);
        }
    }
}

// ------------------------------------------------------------------------------------------ host

template <int WT, int OT>
cudaError_t launch_embed(const EmbedArgs& a, bool vector, cudaStream_t stream)
{
    const int64_t numel = a.count * a.width, units = numel / 8;
    if (!vector) return launch(k_embed_any<WT, OT>, dim3((unsigned)((numel + 2047) / 2048)), 256, 0, stream, false, a);
    constexpr int MANY = WT == APMS_GRAD_F32 ? 2 : 4;
    if (units < (int64_t)1024 * 256 * MANY) return launch(k_embed<WT, OT, 1>, dim3((unsigned)((units + 255) / 256)), 256, 0, stream, false, a);
    return launch(k_embed<WT, OT, MANY>, dim3((unsigned)((units + 256 * MANY - 1) / (256 * MANY))), 256, 0, stream, false, a);
}

template <int WT>
cudaError_t launch_embed_to(const EmbedArgs& a, int out_type, bool vector, cudaStream_t stream)
{
    return out_type == APMS_GRAD_F32 ? launch_embed<WT, APMS_GRAD_F32>(a, vector, stream)
         : out_type == APMS_GRAD_BF16 ? launch_embed<WT, APMS_GRAD_BF16>(a, vector, stream) : launch_embed<WT, APMS_GRAD_F16>(a, vector, stream);
}

// How the work is cut: by the sizes alone, so that the order of the sums is the same on every GPU.
struct EmbedPlan { int lanes, length, passes, digit; int64_t slices, groups, padded; size_t entries, bytes; };
EmbedPlan embed_plan(int64_t count, int64_t vocab, int64_t width)
{
    EmbedPlan p = {};
    p.lanes = 1;
    while (p.lanes < 128 && p.lanes * 8 < width) p.lanes *= 2;
    p.slices = (width + 8 * p.lanes - 1) / (8 * p.lanes);
    // about 1024 CTAs of 128 threads, of 8 to 128 entries: fewer partial sums with long groups, more in flight with many
    const int64_t per_cta = 128 / p.lanes;
    p.length = (int)std::min<int64_t>(128, std::max<int64_t>(8, (count * p.slices + 1024 * per_cta - 1) / (1024 * per_cta)));
    p.groups = (count + p.length - 1) / p.length;
    int bits = 1;                                                   // of the numbers 0 to vocab
    while ((vocab >> bits) > 0) ++bits;
    p.passes = (bits + kSortBits - 1) / kSortBits;
    p.digit = (bits + p.passes - 1) / p.passes;
    p.padded = (width + 7) / 8 * 8;
    p.entries = ((size_t)count * sizeof(uint2) + 255) / 256 * 256;
    p.bytes = 2 * p.entries + 2 * (size_t)p.groups * (size_t)p.padded * sizeof(float);
    return p;
}

template <int DT, int OT>
cudaError_t launch_embed_back(const EmbedBackArgs& a, const EmbedPlan& p, bool vector, cudaStream_t stream)
{
    const int64_t bytes = a.tokens.vocab * a.width * kBytes<OT>;
    const int clearing = (int)std::min<int64_t>(kMostClearing, std::max<int64_t>(1, bytes >> 19));       // half a megabyte a cluster at least
    const bool clear16 = on_16(a.dw) && a.width * kBytes<OT> % 16 == 0;
    cudaError_t e = launch_clusters(k_embed_sort<OT>, kSortCtas, dim3(kSortCtas * (1 + clearing)), kSortThreads, 0, stream, a, clearing, (int)clear16);
    if (e != cudaSuccess) return e;
    const int64_t per_cta = 128 / p.lanes;
    const dim3 grid((unsigned)((p.groups + per_cta - 1) / per_cta), (unsigned)p.slices);
    e = vector ? launch(k_embed_sums<DT, OT, true>, grid, 128, 0, stream, true, a, p.lanes) : launch(k_embed_sums<DT, OT, false>, grid, 128, 0, stream, true, a, p.lanes);
    if (e != cudaSuccess || p.groups < 2) return e;
    return launch(k_embed_joins<OT>, dim3((unsigned)(p.groups - 1), (unsigned)std::min<int64_t>(4, (a.width + 255) / 256)), 256, 0, stream, true, a);
}

template <int DT>
cudaError_t launch_embed_back_to(const EmbedBackArgs& a, const EmbedPlan& p, int out_type, bool vector, cudaStream_t stream)
{
    return out_type == APMS_GRAD_F32 ? launch_embed_back<DT, APMS_GRAD_F32>(a, p, vector, stream)
         : out_type == APMS_GRAD_BF16 ? launch_embed_back<DT, APMS_GRAD_BF16>(a, p, vector, stream) : launch_embed_back<DT, APMS_GRAD_F16>(a, p, vector, stream);
}

constexpr int64_t kMostTokens = 0x7fffffff, kMostVocab = 0x7fffffff, kMostEmbedWidth = (int64_t)1 << 19;

bool embed_sizes(int64_t count, int64_t vocab, int64_t width)
{
    return count >= 0 && count <= kMostTokens && vocab >= 1 && vocab <= kMostVocab && width >= 1 && width <= kMostEmbedWidth;
}

}  // namespace

extern "C" {

apms_status apms_embedding(const apms_embedding_args* args, void* cuda_stream)
{
    const char* who = "apms_embedding";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_embedding_args& g = *args;
    if (!embed_sizes(g.count, g.vocab, g.width) || g.count > APMS_EMBEDDING_MAX / g.width)
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld tokens, %lld rows of %lld: needs 0 <= count < 2^31, 1 <= vocab < 2^31, 1 <= width <= 2^19 and at most 2^40 elements", who,
                             (long long)g.count, (long long)g.vocab, (long long)g.width);
    if (g.token_bytes != 4 && g.token_bytes != 8) return operator_fail(APMS_ERR_INVALID_ARG, "%s: tokens have 4 or 8 bytes, not %d", who, g.token_bytes);
    if (!known_type(g.weight_type) || !known_type(g.out_type)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: unknown element type", who);
    if (g.count == 0) return APMS_OK;
    if (!g.tokens || !g.weight || !g.out) return operator_fail(APMS_ERR_INVALID_ARG, "%s: tokens, weight or out is NULL", who);
    if (g.vocab > 1 && g.weight_stride < g.width) return operator_fail(APMS_ERR_INVALID_ARG, "%s: rows overlap: the stride is below the width", who);
    if ((uintptr_t)g.tokens % g.token_bytes || !on_element(g.weight, g.weight_type) || !on_element(g.out, g.out_type))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    EmbedArgs a = {};
    a.tokens = {g.tokens, g.token_bytes == 8, g.vocab};
    a.count = g.count; a.width = g.width; a.w_stride = g.weight_stride; a.w = g.weight; a.out = g.out; a.scale = g.scale;
    const bool vector = rows_of_eight(a.w, g.vocab, a.w_stride, a.width, g.weight_type) && on_16(a.out);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    OPERATOR_CUDA("apms_embedding", g.weight_type == APMS_GRAD_F32 ? launch_embed_to<APMS_GRAD_F32>(a, g.out_type, vector, stream)
                                  : g.weight_type == APMS_GRAD_BF16 ? launch_embed_to<APMS_GRAD_BF16>(a, g.out_type, vector, stream)
                                                                    : launch_embed_to<APMS_GRAD_F16>(a, g.out_type, vector, stream));
    return APMS_OK;
}

size_t apms_embedding_backward_workspace_bytes(int64_t count, int64_t vocab, int64_t width)
{
    return embed_sizes(count, vocab, width) ? embed_plan(count, vocab, width).bytes : 0;
}

apms_status apms_embedding_backward(const apms_embedding_backward_args* args, void* cuda_stream)
{
    const char* who = "apms_embedding_backward";
    if (!args) return operator_fail(APMS_ERR_INVALID_ARG, "%s: args is NULL", who);
    const apms_embedding_backward_args& g = *args;
    if (!embed_sizes(g.count, g.vocab, g.width))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: %lld tokens, %lld rows of %lld: needs 0 <= count < 2^31, 1 <= vocab < 2^31 and 1 <= width <= 2^19", who,
                             (long long)g.count, (long long)g.vocab, (long long)g.width);
    if (g.token_bytes != 4 && g.token_bytes != 8) return operator_fail(APMS_ERR_INVALID_ARG, "%s: tokens have 4 or 8 bytes, not %d", who, g.token_bytes);
    if (!known_type(g.dout_type) || !known_type(g.dweight_type)) return operator_fail(APMS_ERR_INVALID_ARG, "%s: unknown element type", who);
    if (!g.dweight || (g.count && (!g.tokens || !g.dout))) return operator_fail(APMS_ERR_INVALID_ARG, "%s: tokens, dout or dweight is NULL", who);
    if (g.count > 1 && g.dout_stride < 0) return operator_fail(APMS_ERR_INVALID_ARG, "%s: the stride is below 0", who);
    if ((uintptr_t)g.tokens % g.token_bytes || !on_element(g.dout, g.dout_type) || !on_element(g.dweight, g.dweight_type))
        return operator_fail(APMS_ERR_INVALID_ARG, "%s: an address is not aligned to its element size", who);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (g.count == 0) {
        OPERATOR_CUDA("apms_embedding_backward", cudaMemsetAsync(g.dweight, 0, (size_t)g.vocab * (size_t)g.width * element_size(g.dweight_type), stream));
        return APMS_OK;
    }
    const EmbedPlan p = embed_plan(g.count, g.vocab, g.width);
    if (!g.workspace_dev || ((uintptr_t)g.workspace_dev & 255u) || g.workspace_bytes < p.bytes)
        return operator_fail(APMS_ERR_OOM, "%s: needs apms_embedding_backward_workspace_bytes() of 256-byte aligned workspace", who);
    EmbedBackArgs a = {};
    a.tokens = {g.tokens, g.token_bytes == 8, g.vocab};
    a.count = g.count; a.width = g.width; a.d_stride = g.dout_stride; a.d = g.dout; a.dw = g.dweight; a.scale = g.scale;
    a.length = p.length; a.passes = p.passes; a.digit = p.digit; a.groups = p.groups; a.padded = p.padded;
    char* w = static_cast<char*>(g.workspace_dev);
    a.sorted = reinterpret_cast<uint2*>(w); a.other = reinterpret_cast<uint2*>(w + p.entries);
    a.head = reinterpret_cast<float*>(w + 2 * p.entries); a.tail = a.head + p.groups * p.padded;
    const bool vector = rows_of_eight(a.d, a.count, a.d_stride, a.width, g.dout_type) && on_16(a.dw);
    OPERATOR_CUDA("apms_embedding_backward", g.dout_type == APMS_GRAD_F32 ? launch_embed_back_to<APMS_GRAD_F32>(a, p, g.dweight_type, vector, stream)
                                           : g.dout_type == APMS_GRAD_BF16 ? launch_embed_back_to<APMS_GRAD_BF16>(a, p, g.dweight_type, vector, stream)
                                                                           : launch_embed_back_to<APMS_GRAD_F16>(a, p, g.dweight_type, vector, stream));
    return APMS_OK;
}

}  // extern "C"
