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

// out = round(scale * w[token]), by groups of eight elements (rows that load8 can read), UNITS groups a thread so that as many chains of
// token -> row are in flight.  Bound by HBM: the distinct rows once (repeats come from L2), the output once; 16384 x 1024 binary32 into bfloat16 13.7 us.
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

// Any width and alignment: a warp a row and 256 columns of it at a time, eight elements a lane; PAIRS: two at a time, where width and addresses are even.
template <int WT, int OT, bool PAIRS>
__global__ void __launch_bounds__(256) k_embed_any(EmbedArgs a)
{
    constexpr int EACH = PAIRS ? 2 : 1, N = 8 / EACH;
    const int lane = threadIdx.x & 31;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < a.count; row += (int64_t)gridDim.x * 8) {
        const uint32_t from = a.tokens.row(row);
        const auto* w = static_cast<const typename Element<WT>::T*>(a.w) + from * a.w_stride;
        auto* out = static_cast<typename Element<OT>::T*>(a.out) + row * a.width;
        for (int64_t c0 = lane * EACH; c0 < a.width; c0 += 256) {
            float2 v[N];
            if (from < a.tokens.vocab) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int64_t c = c0 + k * 32 * EACH;
                    v[k] = make_float2(0.0f, 0.0f);
                    if (c >= a.width) continue;
                    if constexpr (!PAIRS) v[k].x = (float)w[c];
                    else if constexpr (WT == APMS_GRAD_F32) v[k] = *reinterpret_cast<const float2*>(w + c);
                    else v[k] = unpack16<WT>(*reinterpret_cast<const uint32_t*>(w + c));
                }
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) v[k] = make_float2(0.0f, 0.0f);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int64_t c = c0 + k * 32 * EACH;
                if (c >= a.width) break;
                const float2 s = make_float2(v[k].x * a.scale, v[k].y * a.scale);
                if constexpr (!PAIRS) store1<OT>(out, c, from < a.tokens.vocab ? s.x : 0.0f);
                else if (from >= a.tokens.vocab) *reinterpret_cast<std::conditional_t<OT == APMS_GRAD_F32, uint2, uint32_t>*>(out + c) = {};
                else if constexpr (OT == APMS_GRAD_F32) *reinterpret_cast<float2*>(out + c) = s;
                else *reinterpret_cast<uint32_t*>(out + c) = pack16<OT>(s);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ gradient
//
// dw[v] = round(scale * sum of dout[i] over the i with tokens[i] = v), rows without a token 0.  Four kernels:
//   k_embed_sort   one cluster of CTAs sorts (token, position) by token, positions in order
//   k_embed_zeros  meanwhile zeros into all of dw (into the rows that no token has alone: they have to be found first, which every CTA for its own rows takes 41 us for 65,536
//                  tokens where the zeros take 31, clusters that share the looking, and that the hardware puts on half of the SMs, 28 us for 512 tokens where this takes 15)
//   k_embed_sums   `length` sorted entries a group of threads, up to eight rows of dout in flight: runs of one token within are written, as are those that end in the next group;
//                  what belongs to a longer run is left as a partial sum
//   k_embed_joins  adds up the partial sums of the longer runs, which k_embed_sums has listed
// Up to 1024 tokens need no sort: k_embed_few, a CTA a token, finds its equals itself (and leaves the work to the first of them).
// The sums are binary32, in an order that the sizes fix.  Bound by HBM: dout read once, dw written once and, for the rows with tokens, twice; by the four kernels' latency where that
// is little.  65,536 tokens, 1024 wide, bfloat16 into binary32: 88 us (sort 21 beside the zeros' 32, sums 44, joins 9); 512 tokens, 768 wide, binary32: 21 us.

constexpr int kSortCtas = 16, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortBits = 9, kSortBins = 1 << kSortBits;

struct EmbedBackArgs {
    Tokens tokens;
    int64_t count, width, d_stride;
    const void* d;
    void* dw;
    uint2 *sorted, *other;                                          // (token, position): the result, and the other buffer of the sort
    float *head, *tail;                                             // partial sums of each group: of the run that came from the left, of the one that goes on
    uint32_t *listed, *list;                                        // how many groups have a longer run's beginning, and which (in any order)
    int64_t padded;                                                 // floats a partial sum's row takes
    int length, passes, digit;                                      // entries a group; of the sort, bits a pass
    int64_t groups;
    float scale;
};

// Which of the warp's lanes hold the same digit of `bits` bits (and are `here`).
__device__ __forceinline__ uint32_t same_digit(uint32_t d, int bits, bool here)
{
    uint32_t same = __ballot_sync(0xffffffffu, here);
    for (int b = 0; b < bits; ++b) {
        const uint32_t ones = __ballot_sync(0xffffffffu, d >> b & 1);
        same &= d >> b & 1 ? ones : ~ones;
    }
    return same;
}

// Stable radix sort, least significant digit first, by one cluster: each warp owns a run of consecutive entries and counts its digits, the CTAs read
// one another's counts through shared memory, and each warp's entries move to their places in order.  Entries live in global memory (L2) and come eight a lane at a time,
// so that a pass over them waits for memory a few times only.  21 us for 65,536 tokens of a vocabulary of 30,522, hidden behind the zeros where the table is large.
constexpr int kAhead = 8;
struct SortShared { uint32_t counts[kSortWarps][kSortBins], total[kSortBins], base[kSortBins], warp_sums[kSortWarps]; };
__device__ void embed_sort(const EmbedBackArgs& a, SortShared& s)
{
    auto& counts = s.counts;
    uint32_t *total = s.total, *base = s.base, *warp_sums = s.warp_sums;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), bins = 1u << a.digit, mask = bins - 1;
    const int64_t share = ((a.count + kSortCtas * kSortWarps - 1) / (kSortCtas * kSortWarps) + 31) / 32 * 32;
    const int64_t begin = min(a.count, ((int64_t)rank * kSortWarps + warp) * share), end = min(a.count, begin + share);
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit;
        const bool last_first = (a.passes & 1) != (pass & 1);       // into `sorted` in the last pass, and every second one before it
        const uint2* from = last_first ? a.other : a.sorted;
        uint2* to = last_first ? a.sorted : a.other;
        uint2 e[kAhead] = {};
        auto load = [&](int64_t i0) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t i = i0 + k * 32 + lane;
                if (i < end) e[k] = pass == 0 ? make_uint2(a.tokens.row(i), (uint32_t)i) : __ldcg(from + i);
            }
        };
        for (uint32_t d = lane; d < bins; d += 32) counts[warp][d] = 0;
        __syncwarp();
        for (int64_t i0 = begin; i0 < end; i0 += kAhead * 32) {
            load(i0);
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (i0 + k * 32 + lane < end) atomicAdd(&counts[warp][(e[k].x >> shift) & mask], 1u);
        }
        __syncthreads();
        if (threadIdx.x < bins) {                                   // each warp's entries of a digit come after those of the warps before it
            uint32_t sum = 0;
#pragma unroll 8
            for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = counts[w][threadIdx.x]; counts[w][threadIdx.x] = sum; sum += c; }
            total[threadIdx.x] = sum;
        }
        cluster_barrier();
        uint32_t before = 0, all = 0;
        if (threadIdx.x < bins) {
#pragma unroll
            for (uint32_t r = 0; r < kSortCtas; ++r) {
                uint32_t c;
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(cluster_address(shared_address(total + threadIdx.x), r)));
                if (r < rank) before += c;
                all += c;
            }
        }
        const bool last = pass == a.passes - 1;
        if (last) cluster_arrive();                                 // no CTA ends before all have read its counts
        uint32_t upto = all;                                        // digits in order: an inclusive scan over the CTA's first threads
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += v; }
        if (lane == 31) warp_sums[warp] = upto;
        __syncthreads();
        if (threadIdx.x < bins) {
            for (int w = 0; w < warp; ++w) before += warp_sums[w];
            base[threadIdx.x] = before + upto - all;
        }
        __syncthreads();
        for (uint32_t d = lane; d < bins; d += 32) counts[warp][d] += base[d];
        __syncwarp();
        for (int64_t i0 = begin; i0 < end; i0 += kAhead * 32) {
            if (end - begin > kAhead * 32) load(i0);                // else they are still there
            uint32_t same[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (i0 + k * 32 >= end) break;
                same[k] = same_digit(e[k].x >> shift & mask, a.digit, i0 + k * 32 + lane < end);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (i0 + k * 32 >= end) break;
                const bool here = i0 + k * 32 + lane < end;
                uint32_t* count = &counts[warp][(e[k].x >> shift) & mask];
                const uint32_t rank_in = __popc(same[k] & ((1u << lane) - 1)), at = here ? *count + rank_in : 0u;
                if (here) __stcg(to + at, e[k]);
                __syncwarp();
                if (here && rank_in == 0) *count = at + __popc(same[k]);
                __syncwarp();
            }
        }
        if (last) cluster_wait();
        else cluster_barrier();                                     // the entries are in place, and no CTA's counts are read any more
    }
}

__global__ void __launch_bounds__(kSortThreads) k_embed_sort(EmbedBackArgs a)
{
    extern __shared__ float4 room[];
    allow_next_kernel();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.listed = 0;
    embed_sort(a, *reinterpret_cast<SortShared*>(room));
}

// Ends after the sort (the kernel launched before it), so that what waits for this kernel has waited for both.
template <int OT>
__global__ void __launch_bounds__(512) k_embed_zeros(EmbedBackArgs a)
{
    allow_next_kernel();
    const int64_t bytes = a.tokens.vocab * a.width * kBytes<OT>, threads = (int64_t)gridDim.x * 512, first = (int64_t)blockIdx.x * 512 + threadIdx.x;
    char* p = static_cast<char*>(a.dw);
    const int64_t head = min(bytes, (int64_t)(-(uintptr_t)p & 15)), whole = (bytes - head) / 16, tail = bytes - head - whole * 16;       // whole elements: p lies on one
    if (first < head / kBytes<OT>) store1<OT>(p, first, 0.0f);
    if (first < tail / kBytes<OT>) store1<OT>(p + head + whole * 16, first, 0.0f);
    uint4* q = reinterpret_cast<uint4*>(p + head);
#pragma unroll 4
    for (int64_t i = first; i < whole; i += threads) q[i] = make_uint4(0, 0, 0, 0);
    wait_for_last_kernel();
}

// Columns of the groups of eight that a thread holds: consecutive where load8 can read the rows, else `lanes` apart.
template <bool VECTOR>
struct Columns {
    int64_t first;
    int lanes;
    __device__ __forceinline__ int64_t at(int j) const { return VECTOR ? first + j : first + (int64_t)j * lanes; }
};

// A group: `lanes` threads (a power of two up to 128) hold 8 columns each of a slice of 8 * lanes; blockIdx.y is the slice.
template <int DT, int OT, bool VECTOR>
__global__ void __launch_bounds__(128, 4) k_embed_sums(EmbedBackArgs a, int lanes)
{
    constexpr int FLIGHT = VECTOR && DT != APMS_GRAD_F32 ? 8 : 4;
    const int lane = threadIdx.x & (lanes - 1), per_cta = 128 / lanes;
    const int64_t group = (int64_t)blockIdx.x * per_cta + threadIdx.x / lanes;
    const Columns<VECTOR> columns = {(int64_t)blockIdx.y * 8 * lanes + (VECTOR ? lane * 8 : lane), lanes};
    wait_for_last_kernel();
    allow_next_kernel();
    if (group >= a.groups || columns.first >= a.width) return;
    const int64_t begin = group * a.length, end = min(a.count, begin + a.length);
    const uint32_t vocab = (uint32_t)a.tokens.vocab;
    auto token = [&](int64_t i) { return i >= 0 && i < a.count ? a.sorted[i].x : vocab; };
    // The run over the border to the left, and the one over that to the right, where they are short: each begins in the group before the border and ends in the one behind it,
    // and is that one's whole work.  Longer runs leave partial sums.
    const uint32_t last = token(end - 1), right = token(end), left = token(begin - 1);
    const bool takes_right = right == last && last != vocab && left != last && token(end + a.length) != last;
    const bool skips_left = left != vocab && left == token(begin) && token(begin - a.length - 1) != left && right != left;
    const int64_t limit = takes_right ? min(a.count, end + a.length) : end;
    float sum[8];
    uint32_t run = vocab;                                           // the running token; `vocab`: none yet
    bool from_left = false;

    auto write = [&](bool goes_on) {
        if (run == vocab) return;
        if (goes_on && !from_left && lane == 0 && blockIdx.y == 0) a.list[atomicAdd(a.listed, 1u)] = (uint32_t)group;
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

    // Rolling: as a row is added its place is loaded with the row FLIGHT entries on, whose entry came FLIGHT entries before that, so that FLIGHT rows are always in flight.
    uint32_t key[FLIGHT];                                           // of the rows in flight; `vocab`: none
    uint2 next[FLIGHT];
    typename Element<DT>::T v[VECTOR ? 1 : FLIGHT][8];              // as loaded: a conversion would wait for its load
    Eight<DT> raw[VECTOR ? FLIGHT : 1];
    auto entry = [&](int64_t i) { return i < limit ? a.sorted[i] : make_uint2(vocab, 0); };
    auto load = [&](int k, const uint2& e, int64_t i) {             // i: the entry's place (looked at here, so that nothing waits for an entry when it is asked for)
        key[k] = (skips_left && e.x == left) || (i >= end && e.x != last) ? vocab : e.x;
        if (key[k] == vocab) return;
        if constexpr (VECTOR) {
            raw[k] = load8<DT>(a.d, e.y * a.d_stride + columns.first);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (columns.at(j) < a.width) v[k][j] = static_cast<const typename Element<DT>::T*>(a.d)[e.y * a.d_stride + columns.at(j)];
        }
    };
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) next[k] = entry(begin + k);
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
        load(k, next[k], begin + k);
        next[k] = entry(begin + FLIGHT + k);
    }
    for (int64_t i0 = begin; i0 < limit; i0 += FLIGHT) {
        if (i0 >= end && key[0] == vocab) break;                    // behind the run that goes on
#pragma unroll
        for (int k = 0; k < FLIGHT; ++k) {
            if (key[k] != vocab) {                                  // else behind the group's entries, or no row (sorted last)
                float one[8];
                if constexpr (VECTOR) values8<DT>(one, raw[k]);
                else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) one[j] = columns.at(j) < a.width ? (float)v[k][j] : 0.0f;
                }
                if (key[k] != run) {
                    write(false);
                    from_left = run == vocab && key[k] == left;
                    run = key[k];
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] = one[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += one[j];
                }
            }
            load(k, next[k], i0 + FLIGHT + k);
            next[k] = entry(i0 + 2 * FLIGHT + k);
        }
    }
    write(run == right && !takes_right);
}

// The longer runs, one a time and 256 columns of it: four columns a thread, eight strips of threads each with an eighth of the partial sums.
constexpr int kStrips = 8, kJoinCtas = 296;
template <int OT>
__global__ void __launch_bounds__(kStrips * 64, 2) k_embed_joins(EmbedBackArgs a)
{
    __shared__ float4 sums[kStrips - 1][64];
    const int lane = threadIdx.x & 63, strip = threadIdx.x >> 6;
    wait_for_last_kernel();
    const int64_t slices = (a.width + 255) / 256, items = (int64_t)*a.listed * slices;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t group = a.list[item / slices], c = (item % slices) * 256 + lane * 4;       // padded rows: whole groups of four
        const uint32_t run = a.sorted[(group + 1) * a.length].x;
        int64_t low = group + 1;                                    // the last group that begins with the run: as many probes as threads at a time
        for (int more = kStrips * 64; more == kStrips * 64; low += more) {
            const int64_t probe = low + 1 + threadIdx.x;
            more = __syncthreads_count(probe < a.groups && a.sorted[probe * a.length].x == run);
        }
        const int64_t partials = low - group, share = (partials + kStrips - 1) / kStrips, first = group + 1 + strip * share, end = min(low + 1, first + share);
        float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto add = [&](const float4& v) { sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w; };
        if (c < a.width) {
            if (strip == 0) sum = *reinterpret_cast<const float4*>(a.tail + group * a.padded + c);
            for (int64_t g = first; g < end; g += 8) {
                float4 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (g + i < end) v[i] = *reinterpret_cast<const float4*>(a.head + (g + i) * a.padded + c);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (g + i < end) add(v[i]);
            }
        }
        __syncthreads();
        if (strip) sums[strip - 1][lane] = sum;
        __syncthreads();
        if (strip == 0 && c < a.width) {
            for (int s = 0; s < kStrips - 1; ++s) add(sums[s][lane]);
            const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j < a.width) store1<OT>(a.dw, run * a.width + c + j, v[j] * a.scale);
        }
    }
}

// Up to kFew tokens: a CTA a token and slice of columns, its `kFewThreads / lanes` strips of threads each a share of the rows of its equals, in order.
constexpr int kFew = 1024, kFewThreads = 512, kFewWarps = kFewThreads / 32;
template <int DT, int OT, bool VECTOR>
__global__ void __launch_bounds__(kFewThreads, 2) k_embed_few(EmbedBackArgs a, int lanes)
{
    __shared__ uint32_t rows[kFew];
    __shared__ int upto[kFew / 32];
    __shared__ float sums[kFewThreads * 8];
    const int thread = threadIdx.x, lane = thread & (lanes - 1), strip = thread / lanes, strips = kFewThreads / lanes, me = blockIdx.x;
    const uint32_t vocab = (uint32_t)a.tokens.vocab, mine = a.tokens.row(me);
    uint32_t equals[kFew / kFewThreads];                            // of the warp's 32 tokens, 512 apart
    bool earlier = false;
#pragma unroll
    for (int q = 0; q < kFew / kFewThreads; ++q) {
        const int i = q * kFewThreads + thread;
        const bool equal = i < a.count && a.tokens.row(i) == mine;
        earlier |= equal && i < me;
        equals[q] = __ballot_sync(0xffffffffu, equal);
        if ((thread & 31) == 0) upto[q * kFewWarps + (thread >> 5)] = __popc(equals[q]);
    }
    if (__syncthreads_or(mine == vocab || earlier)) {               // no row, or an earlier token's work
        wait_for_last_kernel();                                     // even if all CTAs end here, the grid must not end before the zeros are written
        return;
    }
    int count = 0;
#pragma unroll
    for (int w = 0; w < kFew / 32; ++w) {
        if (w / kFewWarps * kFewThreads >= a.count) break;
        const uint32_t own = equals[w / kFewWarps];
        if (w % kFewWarps == thread >> 5 && (own >> (thread & 31) & 1)) rows[count + __popc(own & ((1u << (thread & 31)) - 1))] = (uint32_t)(w / kFewWarps * kFewThreads + thread);
        count += upto[w];
    }
    __syncthreads();
    const Columns<VECTOR> columns = {(int64_t)blockIdx.y * 8 * lanes + (VECTOR ? lane * 8 : lane), lanes};
    const int share = (count + strips - 1) / strips, begin = min(count, strip * share), end = min(count, begin + share);
    float sum[8] = {};
    if (columns.first < a.width) {
        for (int i0 = begin; i0 < end; i0 += 4) {
            float v[4][8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (i0 + k >= end) break;
                const int64_t row = rows[i0 + k] * a.d_stride;
                if constexpr (VECTOR) {
                    const Eight<DT> raw = load8<DT>(a.d, row + columns.first);
                    values8<DT>(v[k], raw);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[k][j] = columns.at(j) < a.width ? load1<DT>(a.d, row + columns.at(j)) : 0.0f;
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (i0 + k >= end) break;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += v[k][j];
            }
        }
    }
    if (share < count) {                                            // more strips than one had rows
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[j * kFewThreads + thread] = sum[j];
        __syncthreads();
        if (strip == 0)
            for (int s = 1; s * share < count; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] += sums[j * kFewThreads + s * lanes + lane];
    }
    wait_for_last_kernel();                                         // the zeros
    if (strip || columns.first >= a.width) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] *= a.scale;
    if (VECTOR) {
        store8<OT>(a.dw, mine * a.width + columns.first, sum);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (columns.at(j) < a.width) store1<OT>(a.dw, mine * a.width + columns.at(j), sum[j]);
    }
}

// ------------------------------------------------------------------------------------------ host

template <int WT, int OT>
cudaError_t launch_embed(const EmbedArgs& a, bool vector, cudaStream_t stream)
{
    const int64_t numel = a.count * a.width, units = numel / 8;
    if (!vector) {
        const bool pairs = a.width % 2 == 0 && a.w_stride % 2 == 0 && (uintptr_t)a.w % (2 * kBytes<WT>) == 0 && (uintptr_t)a.out % (2 * kBytes<OT>) == 0;
        return launch(pairs ? k_embed_any<WT, OT, true> : k_embed_any<WT, OT, false>, dim3((unsigned)std::min<int64_t>(1 << 20, (a.count + 7) / 8)), 256, 0, stream, false, a);
    }
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
struct EmbedPlan { int lanes, length, passes, digit; int64_t slices, groups, padded; size_t entries, listed, bytes; };
EmbedPlan embed_plan(int64_t count, int64_t vocab, int64_t width)
{
    EmbedPlan p = {};
    p.lanes = 1;
    while (p.lanes < 128 && p.lanes * 8 < width) p.lanes *= 2;
    p.slices = (width + 8 * p.lanes - 1) / (8 * p.lanes);
    // about 1024 CTAs of 128 threads, of 8 to 256 entries: several waves, since a group can take on as many entries again; the fewer, the more partial sums
    const int64_t per_cta = 128 / p.lanes;
    p.length = (int)std::min<int64_t>(256, std::max<int64_t>(8, (count * p.slices + 1024 * per_cta * 8 - 1) / (1024 * per_cta * 8) * 8));
    p.groups = (count + p.length - 1) / p.length;
    int bits = 1;                                                   // of the numbers 0 to vocab
    while ((vocab >> bits) > 0) ++bits;
    p.passes = (bits + kSortBits - 1) / kSortBits;
    p.digit = (bits + p.passes - 1) / p.passes;
    p.padded = (width + 7) / 8 * 8;
    p.entries = ((size_t)count * sizeof(uint2) + 255) / 256 * 256;
    p.listed = 2 * p.entries + 2 * (size_t)p.groups * (size_t)p.padded * sizeof(float);
    p.bytes = count <= kFew ? 0 : p.listed + (1 + (size_t)p.groups) * sizeof(uint32_t);
    return p;
}

template <int DT, int OT>
cudaError_t launch_embed_back(const EmbedBackArgs& a, const EmbedPlan& p, bool vector, cudaStream_t stream)
{
    const int64_t bytes = a.tokens.vocab * a.width * kBytes<OT>, per_cta = 128 / p.lanes;
    const dim3 zeros((unsigned)std::min<int64_t>(1024, bytes / 32768 + 1)), grid((unsigned)((p.groups + per_cta - 1) / per_cta), (unsigned)p.slices), few((unsigned)a.count, (unsigned)p.slices);
    if (a.count <= kFew) {
        const cudaError_t e = launch(k_embed_zeros<OT>, zeros, 512, 0, stream, false, a);
        if (e != cudaSuccess) return e;
        return vector ? launch(k_embed_few<DT, OT, true>, few, kFewThreads, 0, stream, true, a, p.lanes) : launch(k_embed_few<DT, OT, false>, few, kFewThreads, 0, stream, true, a, p.lanes);
    }
    static Raised raised[kMostDevices];
    cudaError_t e = raise_limits(raised, reinterpret_cast<const void*>(k_embed_sort), sizeof(SortShared), true);
    if (e == cudaSuccess) e = launch_clusters(k_embed_sort, kSortCtas, dim3(kSortCtas), kSortThreads, sizeof(SortShared), stream, a);
    if (e == cudaSuccess) e = launch(k_embed_zeros<OT>, zeros, 512, 0, stream, true, a);
    if (e == cudaSuccess) e = vector ? launch(k_embed_sums<DT, OT, true>, grid, 128, 0, stream, true, a, p.lanes) : launch(k_embed_sums<DT, OT, false>, grid, 128, 0, stream, true, a, p.lanes);
    if (e == cudaSuccess) e = launch(k_embed_joins<OT>, dim3(kJoinCtas), kStrips * 64, 0, stream, true, a);
    return e;
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
    const bool vector = rows_of_eight(a.w, g.vocab, a.w_stride, a.width, g.weight_type) && on_eight(a.out, g.out_type);
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
    if (p.bytes && (!g.workspace_dev || ((uintptr_t)g.workspace_dev & 255u) || g.workspace_bytes < p.bytes))
        return operator_fail(APMS_ERR_OOM, "%s: needs apms_embedding_backward_workspace_bytes() of 256-byte aligned workspace", who);
    EmbedBackArgs a = {};
    a.tokens = {g.tokens, g.token_bytes == 8, g.vocab};
    a.count = g.count; a.width = g.width; a.d_stride = g.dout_stride; a.d = g.dout; a.dw = g.dweight; a.scale = g.scale;
    a.length = p.length; a.passes = p.passes; a.digit = p.digit; a.groups = p.groups; a.padded = p.padded;
    char* w = static_cast<char*>(g.workspace_dev);
    a.sorted = reinterpret_cast<uint2*>(w); a.other = reinterpret_cast<uint2*>(w + p.entries);
    a.head = reinterpret_cast<float*>(w + 2 * p.entries); a.tail = a.head + p.groups * p.padded;
    a.listed = reinterpret_cast<uint32_t*>(w + p.listed); a.list = a.listed + 1;
    const bool vector = rows_of_eight(a.d, a.count, a.d_stride, a.width, g.dout_type) && on_eight(a.dw, g.dweight_type);
    OPERATOR_CUDA("apms_embedding_backward", g.dout_type == APMS_GRAD_F32 ? launch_embed_back_to<APMS_GRAD_F32>(a, p, g.dweight_type, vector, stream)
                                           : g.dout_type == APMS_GRAD_BF16 ? launch_embed_back_to<APMS_GRAD_BF16>(a, p, g.dweight_type, vector, stream)
                                                                           : launch_embed_back_to<APMS_GRAD_F16>(a, p, g.dweight_type, vector, stream));
    return APMS_OK;
}

}  // extern "C"
