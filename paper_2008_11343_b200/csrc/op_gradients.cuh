// The norm of a list of tensors, and clipping in place or into one flat gradient.
// Part of libapms.so: included by operators.cu.
//
//   S_t = sum_j g_tj^2 (binary64),  norm = sqrt(sum_t S_t),  c = norm <= max ? 1 : max / norm,  out = g * c
//
// The list is cut into tiles; a tile lies in one tensor and is one CTA.  Both readings are HBM streams, 2 operations per element: on a
// list of 1.34 GB (391 tensors, binary32) the norm takes 192 us = 7.0 TB/s, clipping into the flat gradient 580 us = 6.9 TB/s over its two
// readings and one writing; what bounds lists below some 100 MB is the launches and the ramp of one wave of CTAs (50 MB: 14 us).
#pragma once

namespace {

constexpr int kTileBytes = 32768;        // of a tensor's elements
constexpr int kNormThreads = 128;        // 256 bytes a thread (64 to 512 threads, tiles of 8 to 64 KB: 192 to 206 us on 1.34 GB, 128 and 32 KB the fastest)
constexpr int kScaleThreads = 256;       // 128 bytes a thread (with 128 threads the values in registers leave too few CTAs: 675 against 600 us)
constexpr int kGroupTiles = 1024;        // consecutive tiles of one tensor whose sums one warp adds up
constexpr int kTotalThreads = 512;
constexpr int kAloneTiles = kNormThreads;      // lists this short (4 MB): the CTA that finishes last adds up, a launch less (a call on six small
                                         // tensors 9.8 -> 8.2 us; on the GPU the ticket costs what the second kernel did)
constexpr int kOneTiles = 8192, kOneThreads = 1024;      // lists this short: one CTA adds up, from shared memory
constexpr int kTickets = 1024;           // of a list: one for its plain calls, one for each captured call (4 KB)
constexpr int kListPointers = 500;       // tensors' addresses in a launch's arguments

struct __align__(16) TileRecord {
    int64_t first;                       // first element, counted inside its tensor
    int64_t out;                         // ... and inside the whole list (its place in the flat gradient)
    int64_t numel;                       // the tensor's
    int32_t length;
    int32_t tensor;
    int32_t type, contiguous;            // the tensor's, here too: one load tells a CTA all it needs
};
struct GroupRecord { int32_t tile0, tiles; };      // a group: up to kGroupTiles consecutive tiles of one tensor
struct TensorRecord {
    int64_t numel, cols, stride;                // rows of `cols` consecutive elements, `stride` apart
    int32_t type;
    int32_t contiguous;
    int32_t group0, groups;
    int32_t tile0, tiles;
};
struct TensorPointers { const void* p[kListPointers]; };

// The list's tables and sums in its workspace.
struct ListMemory {
    const TileRecord* tiles;
    const TensorRecord* tensors;
    const GroupRecord* group;
    double *tile_sum, *group_sum;
    unsigned* ticket;                    // zero between calls: the CTA that draws the last one puts it back
    float* factor;
    int count, groups;
};

// Where the elements of a tile of a tensor in rows lie; one 64-bit division a thread, then 32-bit ones.
struct RowWalk {
    int64_t row0, col0, cols, stride;
    __device__ RowWalk(const TensorRecord& t, int64_t first) : row0(first / t.cols), col0(first - row0 * t.cols), cols(t.cols), stride(t.stride) {}
    __device__ int64_t place(int k) const
    {
        const int64_t x = col0 + k;
        const int64_t q = cols > (1 << 30) ? (int64_t)(x >= cols) : (int64_t)((uint32_t)x / (uint32_t)cols);
        return (row0 + q) * stride + (x - q * cols);
    }
};

// Square of the elements in a word, added to acc.  In binary64, so that nothing a finite gradient holds over- or underflows;
// joining products in binary32 first was no faster for binary32 and slower for the 16-bit types (the checks it needs).
template <int TYPE>
__device__ __forceinline__ void add_squares(double& acc, uint32_t w)
{
    if (TYPE == APMS_GRAD_F32) {
        const double g = (double)__uint_as_float(w);
        acc = fma(g, g, acc);
    } else {
        const float2 g = unpack16<TYPE>(w);
        acc = fma((double)g.x, (double)g.x, acc);
        acc = fma((double)g.y, (double)g.y, acc);
    }
}

template <int TYPE>
__device__ __forceinline__ double tile_squares(const void* tensor, const TensorRecord* tensors, const TileRecord& tile)
{
    constexpr int ES = TYPE == APMS_GRAD_F32 ? 4 : 2, V = 32 / ES, LOADS = kTileBytes / 32 / kNormThreads;
    double acc = 0.0;
    if (!tile.contiguous) {
        const RowWalk walk(tensors[tile.tensor], tile.first);
        for (int k = threadIdx.x; k < tile.length; k += kNormThreads) {
            const double g = (double)load_element(tensor, walk.place(k), TYPE);
            acc = fma(g, g, acc);
        }
        return acc;
    }
    const char* p = static_cast<const char*>(tensor) + tile.first * ES;
    const int head = min(tile.length, (int)((32 - ((uintptr_t)p & 31)) & 31) / ES);       // elements up to the first 32-byte boundary
    const int vectors = (tile.length - head) / V;
    const char* body = p + head * ES;
    uint32_t w[LOADS][8];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
        const int at = k * kNormThreads + threadIdx.x;
        if (at < vectors) load32(w[k], body + at * 32);
        else for (int j = 0; j < 8; ++j) w[k][j] = 0;
    }
    const int loose = tile.length - vectors * V;                                          // before and behind the body, below 2 V
    if (threadIdx.x < loose) {
        const int k = threadIdx.x < head ? threadIdx.x : threadIdx.x + vectors * V;
        const double g = (double)load_element(p, k, TYPE);
        acc = g * g;
    }
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
#pragma unroll
        for (int j = 0; j < 8; ++j) add_squares<TYPE>(acc, w[k][j]);
    }
    return acc;
}

__device__ __forceinline__ float clip_factor(double squares, float max_norm)
{
    const double norm = sqrt(squares);
    return (isinf(max_norm) || (float)norm <= max_norm) ? 1.0f : (float)((double)max_norm / norm);
}

struct NormOut {
    float *norm, *norms;                 // norms may be null
    float max_norm;
};

// What the norm kernels end with; `total` valid in thread 0.
__device__ __forceinline__ void put_norm(const ListMemory& m, const NormOut& out, double total)
{
    if (threadIdx.x) return;
    *out.norm = (float)sqrt(total);
    *m.factor = clip_factor(total, out.max_norm);
}

// True in every thread of the CTA that is last to come here; what the others wrote before is then visible to it.
__device__ __forceinline__ bool last_cta(unsigned* ticket, bool* smem)
{
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        *smem = atomicAdd(ticket, 1u) == gridDim.x - 1;
        if (*smem) *ticket = 0;
        __threadfence();
    }
    __syncthreads();
    return *smem;
}

// Sums of squares of the tiles.  A CTA holds one tile in registers and leaves: nothing is counted and nobody is waited for (a ticket per
// tile, by which the last CTA would know to add up, kept the CTAs on the SMs for the fence and the atomic's round trip: 256 us
// instead of 197 us on 1.34 GB).  ALONE: the shortest lists, which do count.
// All the sums of these kernels run in an order fixed by the list, whoever forms them.
template <bool ALONE>
__global__ void __launch_bounds__(kNormThreads)
k_tile_squares(const __grid_constant__ TensorPointers ptrs, int tensor0, int64_t tile0, const __grid_constant__ ListMemory m, const __grid_constant__ NormOut out)
{
    __shared__ double red[kNormThreads / 32];
    allow_next_kernel();
    const TileRecord tile = m.tiles[tile0 + blockIdx.x];
    const void* p = ptrs.p[tile.tensor - tensor0];
    double acc = tile.type == APMS_GRAD_F32 ? tile_squares<APMS_GRAD_F32>(p, m.tensors, tile)
               : tile.type == APMS_GRAD_BF16 ? tile_squares<APMS_GRAD_BF16>(p, m.tensors, tile) : tile_squares<APMS_GRAD_F16>(p, m.tensors, tile);
    acc = warp_total(acc);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kNormThreads / 32; ++w) acc += red[w];
        m.tile_sum[tile0 + blockIdx.x] = acc;
    }
    if (!ALONE) return;
    __shared__ double sums[kAloneTiles];
    __shared__ bool last;
    int2 mine = make_int2(0, 0);                     // tiles of this thread's first tensor, read before the wait
    if (threadIdx.x < m.count) mine = make_int2(m.tensors[threadIdx.x].tile0, m.tensors[threadIdx.x].tiles);
    if (!last_cta(m.ticket, &last)) return;
    if (threadIdx.x < gridDim.x) sums[threadIdx.x] = __ldcg(m.tile_sum + threadIdx.x);
    __syncthreads();
    double total = 0.0;
    for (int t = threadIdx.x; t < m.count; t += kNormThreads) {
        if (t >= kNormThreads) mine = make_int2(m.tensors[t].tile0, m.tensors[t].tiles);
        double s = 0.0;
        for (int k = 0; k < mine.y; ++k) s += sums[mine.x + k];
        if (out.norms) out.norms[t] = (float)sqrt(s);
        total += s;
    }
    put_norm(m, out, block_total(total, red));
}

// Lists of up to 8192 tiles (256 MB): all tile sums come to one CTA's shared memory, a thread adds a tensor's, a warp those of a tensor of many.
__global__ void __launch_bounds__(kOneThreads)
k_one_norm(const __grid_constant__ ListMemory m, const __grid_constant__ NormOut out, int tiles)
{
    extern __shared__ double sums[];
    __shared__ double red[kOneThreads / 32];
    constexpr int FEW = 32;
    allow_next_kernel();
    const int lane = threadIdx.x & 31, mine_first = lane * 32 + (threadIdx.x >> 5);        // consecutive tensors go to different warps
    int2 mine = make_int2(0, 0);                     // tiles of this thread's first tensor
    if (mine_first < m.count) mine = make_int2(m.tensors[mine_first].tile0, m.tensors[mine_first].tiles);
    wait_for_last_kernel();
#pragma unroll 8
    for (int k = threadIdx.x; k < tiles; k += kOneThreads) sums[k] = m.tile_sum[k];
    __syncthreads();
    double total = 0.0;
    for (int t0 = 0; t0 < m.count; t0 += kOneThreads) {
        const int t = t0 + mine_first;
        if (t0) mine = t < m.count ? make_int2(m.tensors[t].tile0, m.tensors[t].tiles) : make_int2(0, 0);
        double s = 0.0;
        if (mine.y <= FEW)
            for (int k = 0; k < mine.y; ++k) s += sums[mine.x + k];
        for (unsigned many = __ballot_sync(0xffffffffu, mine.y > FEW); many; many &= many - 1) {        // the warp together
            const int who = __ffs(many) - 1, first = __shfl_sync(0xffffffffu, mine.x, who), count = __shfl_sync(0xffffffffu, mine.y, who);
            double part = 0.0;
            for (int k = lane; k < count; k += 32) part += sums[first + k];
            part = warp_total(part);
            if (lane == who) s = part;
        }
        if (t < m.count && out.norms) out.norms[t] = (float)sqrt(s);
        total += s;
    }
    put_norm(m, out, block_total(total, red));
}

// Longer lists: a warp adds the tiles of a group, the CTA that is last (a ticket each) adds the groups, tensor by tensor, and the tensors.
__global__ void __launch_bounds__(kTotalThreads)
k_list_norm(const __grid_constant__ ListMemory m, const __grid_constant__ NormOut out)
{
    __shared__ double red[kTotalThreads / 32];
    __shared__ bool last;
    allow_next_kernel();
    const int group = blockIdx.x * (kTotalThreads / 32) + threadIdx.x / 32, lane = threadIdx.x & 31;
    GroupRecord g = {0, 0};
    if (group < m.groups) g = m.group[group];
    int g0 = 0, groups = 0;                          // of this thread's first tensor, for the last CTA
    if (threadIdx.x < m.count) { g0 = m.tensors[threadIdx.x].group0; groups = m.tensors[threadIdx.x].groups; }
    wait_for_last_kernel();
    double acc = 0.0;
#pragma unroll 8
    for (int k = lane; k < g.tiles; k += 32) acc += m.tile_sum[g.tile0 + k];
    acc = warp_total(acc);
    if (lane == 0 && group < m.groups) m.group_sum[group] = acc;
    if (!last_cta(m.ticket, &last)) return;
    double total = 0.0;
    for (int k = threadIdx.x; k < m.count; k += kTotalThreads) {
        if (k >= kTotalThreads) { g0 = m.tensors[k].group0; groups = m.tensors[k].groups; }
        double s = 0.0;
#pragma unroll 8
        for (int j = 0; j < groups; ++j) s += __ldcg(m.group_sum + g0 + j);
        if (out.norms) out.norms[k] = (float)sqrt(s);
        total += s;
    }
    put_norm(m, out, block_total(total, red));
}

// ELEMENTS consecutive elements at p as they lie in memory: 16 between 16-bit types, 8 where a type is binary32, so that the wider of
// source and output is 32 bytes a lane.  p is aligned to the piece's bytes, or to 16, or `shift` bytes behind such a boundary,
// the same for the whole tile: a shifted read takes the aligned 16-byte pieces around it and puts the bytes together (a thread's last
// piece is its neighbour's first, so it comes from L1).
template <int TYPE, int ELEMENTS>
struct Piece {
    static constexpr int WORDS = ELEMENTS * (TYPE == APMS_GRAD_F32 ? 4 : 2) / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const char* p, int shift)
    {
        if (WORDS == 8 && shift == 0 && ((uintptr_t)p & 16) == 0) {
            load32(w, p);
            return;
        }
        if (shift == 0) {
#pragma unroll
            for (int k = 0; k < WORDS; k += 4) load16(w + k, p + 4 * k);
            return;
        }
        uint32_t a[WORDS + 4];
#pragma unroll
        for (int k = 0; k < WORDS + 4; k += 4) load16(a + k, p - shift + 4 * k);
        const int words = shift >> 2, bits = (shift & 3) * 8;
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            const uint32_t lo = words == 0 ? a[k] : words == 1 ? a[k + 1] : words == 2 ? a[k + 2] : a[k + 3];
            const uint32_t hi = words == 0 ? a[k + 1] : words == 1 ? a[k + 2] : words == 2 ? a[k + 3] : a[k + 4];
            w[k] = __funnelshift_r(lo, hi, bits);
        }
    }
    __device__ __forceinline__ void values(float* f) const
    {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            if (TYPE == APMS_GRAD_F32) f[k] = __uint_as_float(w[k]);
            else { const float2 g = unpack16<TYPE>(w[k]); f[2 * k] = g.x; f[2 * k + 1] = g.y; }
        }
    }
    // f rounded to TYPE, at p aligned to the piece's bytes
    static __device__ __forceinline__ void store(char* p, const float* f)
    {
        uint32_t v[WORDS];
#pragma unroll
        for (int k = 0; k < WORDS; ++k) v[k] = TYPE == APMS_GRAD_F32 ? __float_as_uint(f[k]) : pack16<TYPE == APMS_GRAD_F32 ? APMS_GRAD_BF16 : TYPE>(f[(2 * k) % ELEMENTS], f[(2 * k + 1) % ELEMENTS]);
        if (WORDS == 8) store32(p, v);
        else *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
    }
};

__device__ __forceinline__ float factor_when_ready(const float* factor)
{
    wait_for_last_kernel();
    return __ldcg(factor);
}

// One tile times the factor, from SRC to DST elements at `out`.  The elements are loaded before the factor is waited for.
template <int SRC, int DST>
__device__ __forceinline__ void scale_tile(const void* tensor, const TensorRecord* tensors, const TileRecord& tile, char* out, const float* factor, bool in_place)
{
    constexpr int SS = SRC == APMS_GRAD_F32 ? 4 : 2, DS = DST == APMS_GRAD_F32 ? 4 : 2;
    constexpr int N = SS == 2 && DS == 2 ? 16 : 8, PIECES = kTileBytes / SS / N / kScaleThreads;
    if (!tile.contiguous) {
        const RowWalk walk(tensors[tile.tensor], tile.first);
        const float c = factor_when_ready(factor);
        if (in_place && c == 1.0f) return;
        for (int k = threadIdx.x; k < tile.length; k += kScaleThreads) {
            const int64_t at = walk.place(k);
            const float g = load_element(tensor, at, SRC) * c;
            if (in_place) store_element(const_cast<void*>(tensor), at, SRC, g);
            else store_element(out, k, DST, g);
        }
        return;
    }
    const char* p = static_cast<const char*>(tensor) + tile.first * SS;
    const int head = min(tile.length, (int)((32 - ((uintptr_t)out & 31)) & 31) / DS);     // elements up to the output's first 32-byte boundary
    const char* from = p + head * SS;
    const int shift = (int)((uintptr_t)from & 15);
    int pieces = (tile.length - head) / N, skip = 0;
    if (shift) {                                   // shifted reads inside the tensor only; the pieces at its ends go one by one
        const char* lo = static_cast<const char*>(tensor);
        const char* hi = lo + tile.numel * SS;
        if (pieces && from - shift < lo) skip = 1;
        if (pieces && from - shift + (int64_t)pieces * (N * SS) + 16 > hi) --pieces;
        if (skip > pieces) skip = pieces;
    }
    Piece<SRC, N> v[PIECES];
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int at = k * kScaleThreads + threadIdx.x;
        if (at >= skip && at < pieces) v[k].load(from + at * (N * SS), shift);
    }
    const float c = factor_when_ready(factor);
    if (in_place && c == 1.0f) return;
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
        const int at = k * kScaleThreads + threadIdx.x;
        if (at >= skip && at < pieces) {
            float f[N];
            v[k].values(f);
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] *= c;
            Piece<DST, N>::store(out + (head + at * N) * DS, f);
        }
    }
    const int before = head + skip * N, behind = head + pieces * N;                       // one by one: [0, before) and [behind, length)
    for (int k = threadIdx.x; k < before + tile.length - behind; k += kScaleThreads) {
        const int e = k < before ? k : k - before + behind;
        store_element(out, e, DST, load_element(p, e, SRC) * c);
    }
}

// DST < 0: in place.  The tiles are taken in the norm's order backwards: its last ones may still be in L2.
template <int DST>
__global__ void __launch_bounds__(kScaleThreads)
k_scale_tiles(const __grid_constant__ TensorPointers ptrs, int tensor0, int64_t tile0, const __grid_constant__ ListMemory m, char* flat)
{
    const TileRecord tile = m.tiles[tile0 + gridDim.x - 1 - blockIdx.x];
    const void* p = ptrs.p[tile.tensor - tensor0];
    if (DST < 0) {
        char* out = static_cast<char*>(const_cast<void*>(p)) + tile.first * (tile.type == APMS_GRAD_F32 ? 4 : 2);
        if (tile.type == APMS_GRAD_F32) scale_tile<APMS_GRAD_F32, APMS_GRAD_F32>(p, m.tensors, tile, out, m.factor, true);
        else if (tile.type == APMS_GRAD_BF16) scale_tile<APMS_GRAD_BF16, APMS_GRAD_BF16>(p, m.tensors, tile, out, m.factor, true);
        else scale_tile<APMS_GRAD_F16, APMS_GRAD_F16>(p, m.tensors, tile, out, m.factor, true);
    } else {
        constexpr int D = DST < 0 ? 0 : DST;
        char* out = flat + tile.out * (D == APMS_GRAD_F32 ? 4 : 2);
        if (tile.type == APMS_GRAD_F32) scale_tile<APMS_GRAD_F32, D>(p, m.tensors, tile, out, m.factor, false);
        else if (tile.type == APMS_GRAD_BF16) scale_tile<APMS_GRAD_BF16, D>(p, m.tensors, tile, out, m.factor, false);
        else scale_tile<APMS_GRAD_F16, D>(p, m.tensors, tile, out, m.factor, false);
    }
}

}  // namespace

struct apms_tensors {
    std::vector<TensorRecord> tensors;
    std::vector<TileRecord> tiles;
    std::vector<GroupRecord> groups;
    std::vector<int> tile0;              // first tile of each tensor, and behind the last
    int64_t total;
    ListMemory m;                        // m.tiles == nullptr: no workspace yet

    // Which kernels form the norm: the tiles' last CTA adds up / one CTA does / the groups' CTAs do, the last of them the rest.
    enum class Route { alone, one, groups };
    Route route() const
    {
        if (!tiles.empty() && tiles.size() <= (size_t)kAloneTiles && tensors.size() <= (size_t)kListPointers) return Route::alone;
        return tiles.size() <= (size_t)kOneTiles ? Route::one : Route::groups;
    }

    // Byte offsets of the tables, the tickets and, from tile_sum on, of what a call writes before it reads it in the workspace.
    struct Places { size_t tensors, groups, tickets, tile_sum, group_sum, last, bytes; };
    Places places() const
    {
        auto up = [](size_t v) { return (v + 255) / 256 * 256; };
        Places p;
        p.tensors = up(tiles.size() * sizeof(TileRecord));
        p.groups = p.tensors + up(tensors.size() * sizeof(TensorRecord));
        p.tickets = p.groups + up(groups.size() * sizeof(GroupRecord));
        p.tile_sum = p.tickets + kTickets * sizeof(unsigned);
        p.group_sum = p.tile_sum + up(tiles.size() * sizeof(double));
        p.last = p.group_sum + up(groups.size() * sizeof(double));       // the factor, and a ticket beside it
        p.bytes = p.last + 256;
        return p;
    }
    int tickets_taken = 1;               // the first is the plain calls'

    // The calls' sums and factor at `p`, laid out as from tile_sum on, and their ticket.
    void write_at(char* p, unsigned* ticket)
    {
        const Places at = places();
        m.tile_sum = (double*)p;
        m.group_sum = (double*)(p + (at.group_sum - at.tile_sum));
        m.factor = (float*)(p + (at.last - at.tile_sum));
        m.ticket = ticket;
    }
    unsigned* tickets() const { return (unsigned*)((char*)m.tiles + places().tickets); }
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
        std::unique_ptr<apms_tensors> list(new apms_tensors());
        int64_t at = 0;
        for (int t = 0; t < count; ++t) {
            TensorRecord r = {};
            r.numel = numel[t];
            r.type = types[t];
            r.contiguous = !cols || row_strides[t] == cols[t] || cols[t] == numel[t];
            r.cols = r.contiguous ? numel[t] : cols[t];
            r.stride = r.contiguous ? numel[t] : row_strides[t];
            const int64_t per_tile = kTileBytes / (int64_t)element_size(types[t]);
            const int64_t tiles = (numel[t] + per_tile - 1) / per_tile;
            if ((int64_t)list->tiles.size() + tiles > 0x7fffffff) return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_create: the list is too long");
            r.group0 = (int32_t)list->groups.size();
            r.tile0 = (int32_t)list->tiles.size();
            r.tiles = (int32_t)tiles;
            list->tile0.push_back((int)list->tiles.size());
            for (int64_t k = 0; k < tiles; ++k) {
                if (k % kGroupTiles == 0) list->groups.push_back({(int32_t)list->tiles.size(), (int32_t)std::min<int64_t>(kGroupTiles, tiles - k)});
                list->tiles.push_back({k * per_tile, at + k * per_tile, numel[t], (int32_t)std::min(per_tile, numel[t] - k * per_tile), t, r.type, r.contiguous});
            }
            r.groups = (int32_t)list->groups.size() - r.group0;
            list->tensors.push_back(r);
            at += numel[t];
        }
        list->total = at;
        list->tile0.push_back((int)list->tiles.size());
        *out = list.release();
    } catch (const std::bad_alloc&) {
        return operator_fail(APMS_ERR_OOM, "apms_tensors_create: host allocation failed");
    }
    return APMS_OK;
}

size_t apms_tensors_workspace_bytes(const apms_tensors* list) { return list ? list->places().bytes : 0; }

apms_status apms_tensors_bind(apms_tensors* list, void* workspace_dev, size_t bytes, void* cuda_stream)
{
    if (!list || !workspace_dev || ((uintptr_t)workspace_dev & 255u)) return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_bind: needs a list and a 256-byte aligned workspace");
    const apms_tensors::Places at = list->places();
    if (bytes < at.bytes) return operator_fail(APMS_ERR_OOM, "apms_tensors_bind: workspace smaller than apms_tensors_workspace_bytes()");
    char* ws = (char*)workspace_dev;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    OPERATOR_CUDA("apms_tensors_bind", cudaMemcpyAsync(ws, list->tiles.data(), list->tiles.size() * sizeof(TileRecord), cudaMemcpyHostToDevice, stream));
    OPERATOR_CUDA("apms_tensors_bind", cudaMemcpyAsync(ws + at.tensors, list->tensors.data(), list->tensors.size() * sizeof(TensorRecord), cudaMemcpyHostToDevice, stream));
    OPERATOR_CUDA("apms_tensors_bind", cudaMemcpyAsync(ws + at.groups, list->groups.data(), list->groups.size() * sizeof(GroupRecord), cudaMemcpyHostToDevice, stream));
    OPERATOR_CUDA("apms_tensors_bind", cudaMemsetAsync(ws + at.tickets, 0, kTickets * sizeof(unsigned), stream));
    OPERATOR_CUDA("apms_tensors_bind", cudaStreamSynchronize(stream));
    ListMemory& m = list->m;
    m.tiles = (const TileRecord*)ws;
    m.tensors = (const TensorRecord*)(ws + at.tensors);
    m.group = (const GroupRecord*)(ws + at.groups);
    m.count = (int)list->tensors.size();
    m.groups = (int)list->groups.size();
    list->tickets_taken = 1;
    list->write_at(ws + at.tile_sum, list->tickets());
    return APMS_OK;
}

size_t apms_tensors_scratch_bytes(const apms_tensors* list)
{
    if (!list) return 0;
    const apms_tensors::Places at = list->places();
    return at.bytes - at.tile_sum;
}

apms_status apms_tensors_use_scratch(apms_tensors* list, void* scratch_dev, size_t bytes, void* cuda_stream)
{
    if (!list || !list->m.tiles) return operator_fail(APMS_ERR_BAD_STATE, "apms_tensors_use_scratch: the list has no workspace (apms_tensors_bind)");
    if (!scratch_dev) {
        list->write_at((char*)list->m.tiles + list->places().tile_sum, list->tickets());
        return APMS_OK;
    }
    if ((uintptr_t)scratch_dev & 255u) return operator_fail(APMS_ERR_INVALID_ARG, "apms_tensors_use_scratch: the scratch memory must be 256-byte aligned");
    if (bytes < apms_tensors_scratch_bytes(list)) return operator_fail(APMS_ERR_OOM, "apms_tensors_use_scratch: scratch memory smaller than apms_tensors_scratch_bytes()");
    const apms_tensors::Places at = list->places();
    unsigned* ticket = nullptr;
    if (list->route() != apms_tensors::Route::one) {
        // A ticket has to be zero before its call, which leaves it so.  The list's own are, so the call need not clear one (3.6 us more in a graph of
        // a 5.6 us call); when they have run out, the one beside the factor is cleared on the stream.
        if (list->tickets_taken < kTickets) {
            ticket = list->tickets() + list->tickets_taken++;
        } else {
            ticket = (unsigned*)((char*)scratch_dev + (at.last - at.tile_sum)) + 1;
            OPERATOR_CUDA("apms_tensors_use_scratch", cudaMemsetAsync(ticket, 0, sizeof(unsigned), (cudaStream_t)cuda_stream));
        }
    }
    list->write_at((char*)scratch_dev, ticket);
    return APMS_OK;
}

void apms_tensors_destroy(apms_tensors* list) { delete list; }

}  // extern "C"

namespace {

apms_status check_addresses(const apms_tensors* list, const void* const* tensors_dev, const char* who)
{
    if (!list || !list->m.tiles) return operator_fail(APMS_ERR_BAD_STATE, "%s: the list has no workspace (apms_tensors_bind)", who);
    if (!tensors_dev) return operator_fail(APMS_ERR_INVALID_ARG, "%s: tensors_dev is NULL", who);
    for (size_t t = 0; t < list->tensors.size(); ++t)
        if (list->tensors[t].numel && (!tensors_dev[t] || (uintptr_t)tensors_dev[t] % element_size(list->tensors[t].type)))
            return operator_fail(APMS_ERR_INVALID_ARG, "%s: tensor %zu is at a NULL or misaligned address", who, t);
    return APMS_OK;
}

// The bytes a tensor spans, from its first element to behind its last.
int64_t spanned_bytes(const TensorRecord& r)
{
    if (!r.numel) return 0;
    return ((r.numel / r.cols - 1) * r.stride + r.cols) * (int64_t)element_size(r.type);
}

// A tensor's bytes: `rows` rows of `length` bytes, `stride` apart.
struct ByteRows {
    int64_t first, rows, length, stride;
    int64_t end() const { return first + (rows - 1) * stride + length; }
};
ByteRows byte_rows(const TensorRecord& r, uintptr_t p)
{
    const int64_t es = (int64_t)element_size(r.type);
    return {(int64_t)p, r.contiguous ? 1 : r.numel / r.cols, r.cols * es, r.stride * es};
}

// Whether two tensors share a byte, exactly: column slices of one matrix interleave without sharing any.
bool share_bytes(const ByteRows& a, const ByteRows& b)
{
    if (a.end() <= b.first || b.end() <= a.first) return false;
    if (a.rows == 1 && b.rows == 1) return true;
    if (a.rows > 1 && b.rows > 1 && a.stride != b.stride) {       // row by row of the shorter one
        const ByteRows& few = a.rows <= b.rows ? a : b;
        for (int64_t k = 0; k < few.rows; ++k)
            if (share_bytes({few.first + k * few.stride, 1, few.length, few.stride}, a.rows <= b.rows ? b : a)) return true;
        return false;
    }
    // Row i of a and row j of b share a byte where k = i - j has  k S < d + b.length  and  k S > d - a.length;  k lies between 1 - b.rows and a.rows - 1.
    const int64_t S = a.rows > 1 ? a.stride : b.stride, d = b.first - a.first;
    auto floor_div = [S](int64_t v) { return v / S - (v % S < 0); };
    const int64_t least = floor_div(d - a.length) + 1, most = floor_div(d + b.length - 1);
    return std::max(least, 1 - b.rows) <= std::min(most, a.rows - 1);
}

// Whether no two tensors of `all` share a byte.  Slices of one matrix mostly lie side by side in its rows, which one pass over their
// columns shows (300 of them: 45,000 pairs otherwise, 260 us); what that leaves open is asked pair by pair.
bool lie_apart(const std::vector<ByteRows>& all)
{
    if (all.size() < 2) return true;
    int64_t S = 0;
    bool matrix = true;
    for (const ByteRows& r : all)
        if (r.rows > 1) { matrix = matrix && (!S || S == r.stride); S = r.stride; }
    if (matrix && S) {
        std::vector<std::pair<int64_t, int64_t>> columns;
        columns.reserve(all.size());
        for (const ByteRows& r : all) columns.push_back({r.first % S, r.length});
        std::sort(columns.begin(), columns.end());
        bool side_by_side = columns.back().first + columns.back().second <= columns.front().first + S;
        for (size_t k = 1; k < columns.size(); ++k) side_by_side = side_by_side && columns[k - 1].first + columns[k - 1].second <= columns[k].first;
        if (side_by_side) return true;
    }
    for (size_t k = 1; k < all.size(); ++k)
        for (size_t j = 0; j < k; ++j)
            if (share_bytes(all[j], all[k])) return false;
    return true;
}

// Launches `kernel(addresses, first tensor, first tile, memory, ...)` over the list's tiles, as many tensors at a time as a
// launch's arguments hold addresses.  `early`: the first launch may begin while the kernel before it drains.
template <class... Params, class... Args>
cudaError_t over_tiles(const apms_tensors* list, const void* const* tensors_dev, cudaStream_t stream, int threads, bool early,
                       void (*kernel)(TensorPointers, int, int64_t, ListMemory, Params...), Args... args)
{
    const int count = (int)list->tensors.size();
    for (int t0 = 0; t0 < count; t0 += kListPointers) {
        const int t1 = std::min(count, t0 + kListPointers);
        const int64_t first = list->tile0[t0], last = list->tile0[t1];
        if (first == last) continue;
        TensorPointers ptrs;
        memcpy(ptrs.p, tensors_dev + t0, (t1 - t0) * sizeof(void*));
        const cudaError_t e = launch(kernel, dim3((unsigned)(last - first)), threads, 0, stream, early, ptrs, t0, first, list->m, Params(args)...);
        if (e != cudaSuccess) return e;
        early = false;
    }
    return cudaSuccess;
}

cudaError_t list_norm(const apms_tensors* list, const void* const* tensors_dev, cudaStream_t stream, float* norm, float* norms, float max_norm)
{
    const NormOut out = {norm, norms, max_norm};
    const int tiles = (int)list->tiles.size();
    const apms_tensors::Route route = list->route();
    if (route == apms_tensors::Route::alone) return over_tiles(list, tensors_dev, stream, kNormThreads, false, k_tile_squares<true>, out);
    cudaError_t e = over_tiles(list, tensors_dev, stream, kNormThreads, false, k_tile_squares<false>, out);
    if (e != cudaSuccess) return e;
    if (route == apms_tensors::Route::one) {
        static Resident resident[kMostDevices];
        int ctas = 0;
        e = resident_ctas(resident, reinterpret_cast<const void*>(k_one_norm), kOneThreads, kOneTiles * sizeof(double), &ctas);
        return e != cudaSuccess ? e : launch(k_one_norm, dim3(1), kOneThreads, tiles * sizeof(double), stream, tiles > 0, list->m, out, tiles);
    }
    const unsigned ctas = (unsigned)((list->groups.size() + kTotalThreads / 32 - 1) / (kTotalThreads / 32));
    return launch(k_list_norm, dim3(ctas), kTotalThreads, 0, stream, true, list->m, out);
}

}  // namespace

extern "C" {

apms_status apms_grad_norm(apms_tensors* list, const void* const* tensors_dev, float* norm_dev, float* norms_dev, void* cuda_stream)
{
    const apms_status st = check_addresses(list, tensors_dev, "apms_grad_norm");
    if (st != APMS_OK) return st;
    if (!norm_dev) return operator_fail(APMS_ERR_INVALID_ARG, "apms_grad_norm: norm_dev is NULL");
    const cudaError_t e = list_norm(list, tensors_dev, (cudaStream_t)cuda_stream, norm_dev, norms_dev, INFINITY);
    return e == cudaSuccess ? APMS_OK : operator_fail(APMS_ERR_CUDA, "apms_grad_norm: %s", cudaGetErrorString(e));
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
        for (size_t t = 0; t < count; at += list->tensors[t].numel, ++t) {
            const uintptr_t a0 = (uintptr_t)tensors_dev[t], a1 = a0 + (uintptr_t)spanned_bytes(list->tensors[t]);
            if (a0 == a1 || a1 <= f0 || a0 >= f1) continue;
            if (!list->tensors[t].contiguous || list->tensors[t].type != (int)flat_type || a0 != f0 + (uintptr_t)at * es)
                return operator_fail(APMS_ERR_INVALID_ARG, "apms_clip_grads: tensor %zu overlaps the flat gradient without being in its place there", t);
        }
    } else {
        try {
            std::vector<std::pair<uintptr_t, size_t>> by_address;
            by_address.reserve(count);
            for (size_t t = 0; t < count; ++t)
                if (list->tensors[t].numel) by_address.push_back({(uintptr_t)tensors_dev[t], t});
            if (!std::is_sorted(by_address.begin(), by_address.end())) std::sort(by_address.begin(), by_address.end());
            std::vector<ByteRows> knot;                  // consecutive ones, each beginning before the end of those before it
            int64_t reach = 0;
            bool apart = true;
            for (const auto& [address, t] : by_address) {
                const ByteRows r = byte_rows(list->tensors[t], address);
                if (r.first >= reach) {
                    apart = apart && lie_apart(knot);
                    knot.clear();
                }
                knot.push_back(r);
                reach = std::max(reach, r.end());
            }
            if (!apart || !lie_apart(knot)) return operator_fail(APMS_ERR_INVALID_ARG, "apms_clip_grads: two tensors of the list overlap in memory; clip into a flat gradient instead");
        } catch (const std::bad_alloc&) {
            return operator_fail(APMS_ERR_OOM, "apms_clip_grads: host allocation failed");
        }
    }
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    cudaError_t e = list_norm(list, tensors_dev, stream, norm_dev, nullptr, max_norm);
    if (e == cudaSuccess) {
        char* flat = (char*)flat_dev;
        e = !flat ? over_tiles(list, tensors_dev, stream, kScaleThreads, true, k_scale_tiles<-1>, flat)
          : flat_type == APMS_GRAD_F32 ? over_tiles(list, tensors_dev, stream, kScaleThreads, true, k_scale_tiles<APMS_GRAD_F32>, flat)
          : flat_type == APMS_GRAD_BF16 ? over_tiles(list, tensors_dev, stream, kScaleThreads, true, k_scale_tiles<APMS_GRAD_BF16>, flat)
          : over_tiles(list, tensors_dev, stream, kScaleThreads, true, k_scale_tiles<APMS_GRAD_F16>, flat);
    }
    return e == cudaSuccess ? APMS_OK : operator_fail(APMS_ERR_CUDA, "apms_clip_grads: %s", cudaGetErrorString(e));
}

}  // extern "C"
